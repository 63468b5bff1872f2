"""Chunks whose best logits do not fit a list: many equal ones (masks, constants), and more large ones in some waves' parts
than the list holds above the others'.  Order is by value, then by token, whichever way they are found."""

import numpy as np
import pytest
import torch

from oracle import beam
from paper_2605_05819_amd import cl

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def check(x, n, picks, scores=None):
    rows = x.shape[0]
    s0 = torch.zeros(rows) if scores is None else scores
    s, t, p, _, _ = cl.beam_select(cl.Beams(n, picks=picks), x.cuda(), s0.cuda())
    want = beam.select(x.double().numpy(), s0.numpy(), n, picks)
    torch.cuda.synchronize()
    assert np.array_equal(t.cpu().numpy(), want[1].astype(int)) and np.array_equal(p.cpu().numpy(), want[2].astype(int))
    assert np.allclose(s.double().cpu().numpy(), want[0], rtol=2.0 ** -22, atol=2.0 ** -20)


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("V,rows", [(2048, 1), (5000, 3), (8192, 70), (40001, 40)])
@pytest.mark.parametrize("kept", [0, 3, 40])
def test_masked_but_for_a_few(V, rows, kept, dtype):
    """All tokens at one value but for a few above it and a few below: as many picks as are above, fewer and more."""
    g = torch.Generator().manual_seed(V + kept)
    for fill in (0.0, -0.0, -100.0, -torch.finfo(dtype).max):
        x = torch.full((rows, V), fill, dtype=dtype)
        for r in range(rows):
            at = torch.randperm(V, generator=g)[:2 * kept]
            x[r, at[:kept]] = (fill / 2 + 1 + torch.rand(kept, generator=g)).to(dtype)
            x[r, at[kept:]] = float("-inf")
        for picks in (1, 3, 5, 64):
            check(x, 1, picks)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V,rows,part", [(2048, 1, 512), (8192, 70, 1024), (16384, 80, 2048)])
def test_more_above_the_least_than_the_list_holds(V, rows, part, dtype):
    """One wave's part of a chunk is constant, the others' lie above it, with ties of their own."""
    g = torch.Generator().manual_seed(V)
    x = (torch.rand((rows, V), generator=g) * 3 + 1).to(dtype)
    x.view(rows, -1, part)[:, ::4] = 0.0
    for picks in (1, 4, 33, 64):
        check(x, 1, picks)
    check(x[:rows // 5 * 5] if rows > 4 else x, 5 if rows > 4 else 1, 20, torch.zeros(rows // 5 * 5 if rows > 4 else rows))


def test_a_rows_end_of_equal_values():
    """Fewer values than picks in a row's last chunk, all of them equal."""
    x = torch.zeros((2, 2048 + 7))
    x[:, :2048] = -5.0
    check(x, 2, 64)
    check(torch.zeros((1, 40)), 1, 40)
