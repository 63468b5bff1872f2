"""Beam selection against fp64.  Tokens, parents, lengths and flags are equal wherever ranks of different beams are
further apart than the sums' error (2^-20 here: fp32 terms of 2^-23 each, added in lanes of 32 and in fp64 beyond), which the
inputs' seeds were not chosen for: groups with a smaller gap are left out, and few may be.  Scores: that and their rounding."""

import numpy as np
import pytest
import torch

from oracle import beam
from paper_2605_05819_amd import cl

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(x, scores, beams, picks=None, lengths=None, finished=None, eos=-1, alpha=0.0, logits=None, most_left_out=0):
    """x: logits on the CPU, as a tensor; logits: the device's view of them."""
    picks = beams if picks is None else picks
    rule = cl.Beams(beams, picks=picks, eos=eos, alpha=alpha)
    dev = lambda v, t: None if v is None else torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    got = cl.beam_select(rule, x.cuda() if logits is None else logits, dev(scores, F32), dev(lengths, torch.int32),
                         dev(finished, torch.int32))
    torch.cuda.synchronize()
    s32 = torch.tensor(scores, dtype=F32).double().numpy()
    *want, gap = beam.select(x.double().numpy(), s32, beams, picks, lengths, finished, eos, alpha)
    n = 1 if lengths is None else max(1, min(lengths))
    scale = max(1.0, 1.0 / n ** alpha, (max(lengths or [1]) + 1) ** -alpha)
    sure = gap > 2.0 ** -20 * scale
    assert (~sure).sum() <= most_left_out, gap.min()
    s = got[0].double().cpu().numpy()
    with np.errstate(over="ignore"):                 # a score past fp32's range (lowest less highest logit) is -inf
        same = (s == want[0].astype(np.float32)) | (np.isnan(s) & np.isnan(want[0]))
    with np.errstate(invalid="ignore"):
        near = np.abs(s - want[0]) <= 2.0 ** -24 * np.abs(want[0]) * 1.01 + 2.0 ** -20
    assert (same | near)[sure].all()
    for i, g in enumerate(got[1:], 1):
        if g is None:
            assert i == 3 and lengths is None
            continue
        assert np.array_equal(g.cpu().numpy()[sure], want[i][sure]), (i, np.argwhere(g.cpu().numpy() != want[i])[:4])
    return got


SHAPES = [(1, 1, 1, 1), (1, 2, 3, 2), (1, 4, 4, 5), (2, 3, 6, 7), (1, 4, 4, 2047), (1, 4, 4, 2049), (3, 5, 10, 8193), (2, 2, 64, 40),
          (1, 64, 64, 300), (1, 8, 16, 50257), (4, 4, 4, 32000), (9, 8, 8, 16001), (40, 8, 12, 33333), (2, 3, 5, 1 << 19)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_oracle(shape, dtype):
    G, n, k, V = SHAPES[shape]
    g = torch.Generator().manual_seed(shape)
    x = (torch.randn((G * n, V), generator=g) * 3).to(dtype)
    scores = (-5 * torch.rand(G * n, generator=g)).tolist()
    lengths = torch.randint(1, 50, (G * n,), generator=g).tolist()
    check(x, scores, n, k, most_left_out=G // 10)
    check(x, scores, n, k, lengths=lengths, alpha=0.7, eos=V // 2, finished=(torch.rand(G * n, generator=g) < 0.3).int().tolist(),
          most_left_out=G // 10)


@pytest.mark.parametrize("V", [10, 3000, 20000])
def test_ties_go_to_the_lower_beam_and_token(V):
    """Constant rows, rows of two values, one beam's row twice: more equal logits than the list holds."""
    x = torch.zeros((6, V))
    check(x, [0.0] * 6, 3, 7)
    x[:, 5:] = 1.0
    check(x, [0.0, 0.0, -1.0] * 2, 3, 7)
    g = torch.Generator().manual_seed(1)
    y = torch.randn((1, V), generator=g).to(BF16)
    check(y.repeat(4, 1), [-1.0, -1.0, -1.0, -1.0], 4, 9)
    z = torch.randint(0, 2, (4, V), generator=g).float()
    check(z, [-1.0, -2.0, -1.0, -3.0], 4, 16, most_left_out=1)


@pytest.mark.parametrize("V", [100, 9000])
def test_masked_vocabularies(V):
    """Most logits -inf, as a grammar leaves them: fewer allowed tokens than picks, and none."""
    g = torch.Generator().manual_seed(2)
    x = torch.full((8, V), float("-inf"))
    for r, n in enumerate((1, 3, 70, 0, 5, V // 2, 2, 0)):
        at = torch.randperm(V, generator=g)[:n]
        x[r, at] = torch.randn(n, generator=g)
    check(x, [-1.0, -2.0, -0.5, -0.1, -3.0, -1.5, -2.5, -9.0], 4, 12)
    check(x, [-1.0, -2.0, -0.5, -0.1, -3.0, -1.5, -2.5, -9.0], 2, 5, lengths=[4, 5, 6, 7, 8, 9, 1, 2], alpha=1.0)


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("V", [100, 9000, 70000])
def test_masks_of_the_lowest_value(V, dtype):
    """Masks of the type's lowest value over all or nearly all of a row, of whole chunks beside others, its largest
    value; and chunks of -inf beside logits far below zero, whose exponentials only their own maximum keeps."""
    g = torch.Generator().manual_seed(7)
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = torch.randn((8, V), generator=g).to(dtype)
    x[0] = low
    x[1, 3:] = low
    x[2, :V // 2] = low
    x[3, V // 2:] = low
    x[4], x[4, V // 3] = low, high / 2
    x[5, V - 4:] = high
    x[6, V // 2:] = -float("inf")
    x[6, :V // 2] -= 20000 if dtype == F16 else 3.0e5
    x[7] = high
    scores = [-1.0, -2.0, -0.5, -0.25, -3.0, -1.5, -2.5, -6.0]
    check(x, scores, 1, 3)
    check(x[:4].contiguous(), scores[:4], 4, 6)
    check(x[6:].contiguous(), scores[6:], 2, 6)


def test_first_step_and_dead_beams():
    """Beams of -inf beside one that lives: their candidates come behind all of its."""
    x = torch.randn((4, 500), generator=torch.Generator().manual_seed(3))
    inf = float("inf")
    check(x, [0.0, -inf, -inf, -inf], 4, 8)
    check(x[:, :3].contiguous(), [-inf, 0.0, -inf, -inf], 4, 8)
    check(x, [-inf] * 4, 4, 8)


def test_finished_groups():
    x = torch.randn((8, 700), generator=torch.Generator().manual_seed(4))
    check(x, [-1.0, -2.0, -3.0, -4.0] * 2, 4, 10, lengths=[3] * 8, finished=[1] * 4 + [1, 0, 0, 1], eos=0)
    check(x, [-1.0, -2.0, -3.0, -4.0] * 2, 4, 4, lengths=[3, 90, 5, 8] * 2, finished=[1, 1, 0, 1] * 2, eos=699, alpha=1.0)


def test_values_that_are_no_numbers():
    nan, inf = float("nan"), float("inf")
    x = torch.randn((6, 2500), generator=torch.Generator().manual_seed(5))
    x[0, 7], x[2, 2100], x[3, 5] = nan, inf, -inf
    check(x, [0.0, -1.0, 0.0, -2.0, nan, inf], 6, 20)
    check(x, [0.0, -1.0, 0.0, -2.0, nan, inf], 3, 3)
    check(x, [nan, -1.0, 0.0, -inf, nan, inf], 3, 9, finished=[1, 0, 0, 1, 1, 1], eos=3)


def test_large_and_small_logits():
    """Logits in the thousands, and rows that differ by their scale alone."""
    g = torch.Generator().manual_seed(6)
    x = torch.randn((4, 5000), generator=g) * torch.tensor([[1000.0], [0.001], [1.0], [60.0]])
    check(x, [-3.0, -1.0, -2.0, 0.0], 4, 16)
    check((x * 30).to(F16), [-3.0, -1.0, -2.0, 0.0], 4, 16)


@pytest.mark.parametrize("dtype,V,stride,off", [(BF16, 1001, 1001, 0), (BF16, 5003, 5120, 1), (F16, 32000, 32064, 3), (F32, 777, 900, 1)])
def test_rows_at_any_stride_and_offset(dtype, V, stride, off):
    """A view of a padded vocabulary: what stands past a row is NaN."""
    wide = torch.full((6, stride + off), float("nan"), dtype=dtype)
    wide[:, off:off + V] = (torch.randn((6, V), generator=torch.Generator().manual_seed(V)) * 2).to(dtype)
    dev = wide.cuda()[:, off:off + V]
    check(wide[:, off:off + V].contiguous(), [-1.0, -2.0, -0.3] * 2, 3, 6, logits=dev)


def test_outputs_in_place_of_new_ones_repeat_bit_for_bit_and_replay():
    g = torch.Generator(device="cuda").manual_seed(7)
    rule = cl.Beams(4, eos=9, alpha=0.5)
    x = torch.randn((32, 70001), device="cuda", generator=g).to(BF16)
    scores = -torch.rand(32, device="cuda", generator=g)
    lengths, finished = i32([5] * 32), i32([0, 0, 1, 0] * 8)
    want = cl.beam_select(rule, x, scores, lengths, finished)
    side = torch.cuda.Stream()
    for _ in range(3):
        got = cl.beam_select(rule, x, scores, lengths, finished, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = tuple(torch.empty_like(t) for t in want)
    ws = cl.workspace(cl.beam_workspace(rule, 8, 70001), "cuda").fill_(255)
    with torch.cuda.stream(side):
        cl.beam_select(rule, x, scores, lengths, finished, out=out, ws=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cl.beam_select(rule, x, scores, lengths, finished, out=out, ws=ws)
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda", generator=g) * (i + 1))
        scores.uniform_(-3, 0, generator=g)
        want = cl.beam_select(rule, x, scores, lengths, finished)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_the_largest_lists():
    """64 beams and picks over 2^19 tokens: a group's candidates and two waves' lists fill the LDS; with ties in every chunk."""
    g = torch.Generator().manual_seed(11)
    x = torch.randn((64, 1 << 19), generator=g).to(F16)
    x[5] = 1.0
    x[9, 100000:] = -float("inf")
    check(x, (-3 * torch.rand(64, generator=g)).tolist(), 64, 64, lengths=[7] * 64, finished=[int(i == 3) for i in range(64)], eos=12345)


def test_more_groups_than_a_grid_of_small_ones():
    """30000 groups of 2 beams: a workgroup each, equal inputs in every thousandth."""
    g = torch.Generator(device="cuda").manual_seed(12)
    x = torch.randn((60000, 70), device="cuda", generator=g)
    x[2000:4000] = x[:2000]
    scores = -torch.rand(60000, device="cuda", generator=g)
    scores[2000:4000] = scores[:2000]
    s, t, p, n, f = cl.beam_select(cl.Beams(2, picks=3), x, scores)
    torch.cuda.synchronize()
    assert n is None and torch.equal(s[:1000], s[1000:2000]) and torch.equal(t[:1000], t[1000:2000])
    assert torch.equal(p[:1000] + 2000, p[1000:2000]) and not f.any()
    total = (scores[:, None].double() + torch.log_softmax(x.double(), 1)).view(30000, 140)
    want = total.sort(dim=1, descending=True).values[:, :3]
    assert (s.double() - want).abs().max() <= 2.0 ** -20
