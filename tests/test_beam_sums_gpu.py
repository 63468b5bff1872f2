"""How near a beam's log-sum is: rows with one large logit and many equal small ones, whose roundings are all alike, at
places where an exponent's own rounding is largest.

The bound: an exponential is off by 2^-23.5 of itself at most (the instruction, measured over its range; what its
argument's rounding leaves out is added to first order), eight of them are added in fp32 (three roundings of 2^-24 of
the sum, ordered as a tree), all else is fp64: 2^-23.5 + 3 x 2^-24 < 2^-21.9 of the sum, so that much of its logarithm.
The scores here are made to come out near 0, where their own rounding to fp32 is below 2^-27: 2^-21.8 in all."""

import numpy as np
import pytest
import torch

from paper_2605_05819_amd import cl

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
# rows' largest logit, the others, how many
ROWS = [(0.25, -5.327, 8192), (0.25, -10.904, 128000), (5.47, -1.148, 8192), (6.758, -4.47, 128000), (0.0, -6.1, 2048), (-3.3, -14.2, 32000),
        (31.9, 24.7, 9000), (64.5, 55.25, 50000), (140.2, 131.9, 8192), (-31.8, -38.3, 8193), (-33.1, -41.4, 70000), (-900.0, -905.3, 8192),
        (2.0 ** 25, 2.0 ** 25 - 8, 8192), (16.0, 15.99, 128000), (3.0, 3.0, 1000), (1.0, -20.6, 1 << 19)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("row", range(len(ROWS)))
def test_equal_small_logits(row, dtype):
    top, low, V = ROWS[row]
    if dtype == F16 and top > 60000:
        pytest.skip("past fp16")
    x = torch.full((3, V), low, dtype=dtype)
    x[0, V // 3], x[1, V - 1], x[2, 0] = top, top, top
    x[2, 1::2] = -torch.finfo(dtype).max if row % 2 else float("-inf")     # half of them masked
    y = x.double().numpy()
    m = y.max(1)
    best = -np.log(np.exp(y - m[:, None]).sum(1))
    before = torch.from_numpy(-best).float()
    s, t, _, _, _ = cl.beam_select(cl.Beams(1), x.cuda(), before.cuda())
    torch.cuda.synchronize()
    off = np.abs(s.double().cpu().numpy()[:, 0] - (before.double().numpy() + best))
    assert (off <= 2.0 ** -21.8).all(), np.log2(off.max())
    assert (x[torch.arange(3), t.cpu().long()[:, 0]].double().numpy() == m).all()


@pytest.mark.parametrize("shift", [0.0, -20.0, -31.0, -40.0, 50.0, 70.0, 1e5])
def test_one_row_at_many_levels(shift):
    """A constant added to a row's logits changes nothing but what their own rounding to fp32 does."""
    g = torch.Generator().manual_seed(3)
    x = (2 * torch.randn((2, 40000), generator=g)).clamp(-20, 12) + shift
    x[1, ::7] = float("-inf")
    y = x.double()
    best = torch.log_softmax(y, 1).max(1).values
    before = (-best).float()
    s, t, _, _, _ = cl.beam_select(cl.Beams(1), x.cuda(), before.cuda())
    assert ((s.double().cpu()[:, 0] - (before.double() + best)).abs() <= 2.0 ** -21.8).all()
