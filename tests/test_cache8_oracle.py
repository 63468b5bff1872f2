"""Pins of the oracle of the 8-bit cache against torch's e4m3 type and hand-worked blocks."""

import numpy as np
import torch

from oracle import cache8


def test_decode_is_torchs_type():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = cache8.decode(codes.numpy())
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    assert np.isnan(got).sum() == 2 and cache8._VALUES[-1] == 448


def test_encode_is_torchs_rounding():
    g = np.random.default_rng(0)
    x = np.concatenate([g.standard_normal(4000) * 2.0 ** g.integers(-12, 8, 4000), (cache8._VALUES[1:] + cache8._VALUES[:-1]) / 2,
                        [0.0, -0.0, 2.0 ** -10, -2.0 ** -10, 3 * 2.0 ** -10, 448, 464, -460]]).clip(-464, 464)
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(cache8.encode(x), want)
    assert cache8.encode(np.nan) == 127


def test_blocks_by_hand():
    # 448 fits 2^0, a hair more does not; the range's ends hold
    assert cache8.exponent(448.0, "bf16") == 0 and cache8.exponent(448.0000001, "bf16") == 1
    assert cache8.exponent(0.0, "fp16") == -15 and cache8.exponent(1e-30, "fp16") == -15 and cache8.exponent(65504, "fp16") == 8
    assert cache8.exponent(3.3e38, "bf16") == 120
    # 1 under 2^-8 is 256 (code 0x78); a row of 8 lifts the exponent to -5: 1 becomes 32 (0x60), exactly
    codes, e = cache8.append(np.zeros((0, 2)), 0, [[1.0, -0.25]], "fp16")
    assert e == -8 and codes.tolist() == [[0x78, 0xe8]]
    codes, e = cache8.append(codes, e, [[8.0, np.inf]], "fp16")
    assert e == -5 and codes.tolist() == [[0x60, 0xd0], [0x78, 0x7f]]
    # a smaller one leaves it
    codes, e = cache8.append(codes, e, [[0.001, 0.0]], "fp16")
    assert e == -5 and codes[2].tolist() == [cache8.encode(0.032), 0]
    # every value of a held block is finite in the type
    assert np.float16(cache8.decode(cache8.append(np.zeros((0, 1)), 0, [[65504.0]], "fp16")[0])[0, 0] * 2.0 ** 8) == 61440
