"""Pins of the fp64 oracle of the operators between a layer's linears, and the
rotary frequencies (host code): properties and hand-worked values that use
none of the oracle's own formulas."""

import math

import numpy as np
import pytest

from oracle import layer
from paper_2605_05819_amd import cl


def test_attend_is_a_convex_combination_and_follows_the_masks():
    g = np.random.default_rng(1)
    q, k, v = g.standard_normal((3, 4, 8)), g.standard_normal((2, 6, 8)), g.standard_normal((2, 6, 8))
    o, lse, _, _ = layer.attend(q, k, v, 0.3)
    # the first of three new tokens sees keys 0..3 only: the others do not matter
    k2, v2 = k.copy(), v.copy()
    k2[:, 4:] = v2[:, 4:] = 1e6
    assert np.array_equal(layer.attend(q, k2, v2, 0.3)[0][0], o[0])
    assert (o.max(axis=-1) <= v.max() + 1e-12).all() and (o.min(axis=-1) >= v.min() - 1e-12).all()
    # equal keys: the mean of the seen values, lse = score + ln(count)
    same = np.repeat(k[:, :1], 6, axis=1)
    o, lse, _, _ = layer.attend(q, same, v, 0.3, window=2)
    assert np.allclose(o[2, 3], v[1, 4:6].mean(axis=0)) and np.allclose(o[0, 0], v[0, 2:4].mean(axis=0))
    assert np.isclose(lse[2, 3], 0.3 * q[2, 3] @ k[1, 0] + math.log(2))
    # shifting every key by a vector orthogonal to q changes nothing
    assert np.allclose(layer.attend(q, k, v, 0.0, causal=False)[0][1, 2], v[1].mean(axis=0))


def test_attend_without_keys_is_zero():
    o, lse, _, _ = layer.attend(np.ones((2, 1, 4)), np.ones((1, 1, 4)), np.ones((1, 1, 4)), 1.0)
    assert (o[0] == 0).all() and lse[0, 0] == -np.inf and np.allclose(o[1], 1.0)


def test_rotate_keeps_lengths_and_depends_on_distance_only():
    g = np.random.default_rng(2)
    x, y = g.standard_normal((1, 16)), g.standard_normal((1, 16))
    f = np.array([1.0, 0.3, 0.05])
    for inter in (False, True):
        a = layer.rotate(x, 1234.0, f, inter)
        assert np.isclose(np.linalg.norm(a), np.linalg.norm(x)) and np.array_equal(a[:, 6:], x[:, 6:])
        near = (layer.rotate(x, 7.0, f, inter) * layer.rotate(y, 4.0, f, inter)).sum()
        far = (layer.rotate(x, 1007.0, f, inter) * layer.rotate(y, 1004.0, f, inter)).sum()
        assert np.isclose(near, far)
    quarter = layer.rotate(np.array([[1.0, 0.0, 5.0, 0.0]]), math.pi / 2, [1.0, 0.0])
    assert np.allclose(quarter, [[-5.0, 0.0, 1.0, 0.0]])
    assert np.allclose(layer.rotate(np.array([[1.0, 5.0]]), math.pi / 2, [1.0], True), [[-5.0, 1.0]])


def test_route_worked_example():
    # two groups of two; sigmoid scores .5 .731 .881 .119; the bias moves the choice, not the weights
    ids, w, _ = layer.route([[0.0, 1.0, 2.0, -2.0]], 2, "sigmoid", renormalize=False)
    assert ids.tolist() == [[2, 1]] and np.allclose(w, [[0.8807970779, 0.7310585786]])
    ids, w, _ = layer.route([[0.0, 1.0, 2.0, -2.0]], 2, "sigmoid", bias=np.array([1.0, 0, 0, 0]))
    assert ids.tolist() == [[0, 2]] and np.allclose(w, [[0.5 / 1.3807970779, 0.8807970779 / 1.3807970779]])
    ids, _, _ = layer.route([[0.0, 1.0, 2.0, -2.0]], 2, "sigmoid", groups=2, top_groups=1, group_best=2)
    assert ids.tolist() == [[1, 0]]                                  # .5 + .731 > .881 + .119
    ids, _, _ = layer.route([[0.0, 1.0, 2.0, -2.0]], 2, "sigmoid", groups=2, top_groups=1)
    assert ids.tolist() == [[2, 3]]
    ids, w, _ = layer.route([[3.0, 3.0, 3.0]], 2)                    # ties to the lower id
    assert ids.tolist() == [[0, 1]] and np.allclose(w, 0.5)


def test_residual_norm_worked_example():
    h, out = layer.residual_norm([[3.0, 4.0]], np.array([2.0, 1.0]), residual=[[1.0, -4.0]], beta=2.0, eps=0.0)
    assert np.allclose(h, [[7.0, 4.0]]) and np.allclose(out, [[14.0 / math.sqrt(32.5), 4.0 / math.sqrt(32.5)]])
    h, out = layer.residual_norm([[[1.0, 0.0], [0.0, 1.0]]], np.ones(2), slot_weights=[[3.0, 4.0]], kind="layer", eps=0.0)
    assert np.allclose(h, [[3.0, 4.0]]) and np.allclose(out, [[-1.0, 1.0]])


def test_rope_frequencies():
    plain, mag = cl.rope_frequencies(8, 10000.0)
    assert mag == 1.0 and np.allclose(plain.numpy(), [1.0, 0.1, 0.01, 0.001], rtol=1e-7)
    lin, _ = cl.rope_frequencies(8, 10000.0, "linear", 4.0)
    assert np.allclose(lin.numpy(), plain.numpy() / 4, rtol=1e-7)
    base, _ = cl.rope_frequencies(8, 10000.0, "base", 4.0)
    assert base[0] == 1.0 and np.isclose(base[3], 0.001 / 4, rtol=1e-6)      # the slowest pair by the factor
    assert (base.numpy() <= plain.numpy()).all()
    # turns over 8192 positions: fast pairs stay, slow ones are divided, the rest lies between
    bands, _ = cl.rope_frequencies(128, 500000.0, "bands", 8.0, 8192, 1.0, 4.0)
    p128 = cl.rope_frequencies(128, 500000.0)[0].numpy().astype(np.float64)
    turns = 8192 * p128 / (2 * math.pi)
    b = bands.numpy()
    assert np.allclose(b[turns > 4.001], p128[turns > 4.001], rtol=1e-6)
    assert np.allclose(b[turns < 0.999], p128[turns < 0.999] / 8, rtol=1e-6)
    mid = (turns > 1.01) & (turns < 3.99)
    assert mid.any() and ((b[mid] < p128[mid]) & (b[mid] > p128[mid] / 8)).all()
    ramp, mag = cl.rope_frequencies(128, 10000.0, "ramp", 16.0, 4096, 1.0, 32.0)
    r, p = ramp.numpy(), cl.rope_frequencies(128, 10000.0)[0].numpy()
    assert np.isclose(mag, 0.1 * math.log(16.0) + 1) and r[0] == p[0] and np.isclose(r[-1], p[-1] / 16, rtol=1e-6)
    ratio = r / p
    assert (np.diff(ratio) <= 1e-6).all()


@pytest.mark.parametrize("kw", [dict(rot_dim=7), dict(rot_dim=2), dict(base=1.0), dict(kind="linear", factor=0.5),
                                dict(kind="bands", factor=2.0, trained_len=0.0),
                                dict(kind="ramp", factor=2.0, trained_len=4096, low=4.0, high=1.0)])
def test_rope_frequencies_refuses(kw):
    with pytest.raises(cl.ClError) as e:
        cl.rope_frequencies(**{"rot_dim": 64, **kw})
    assert e.value.status == cl.CL_EINVAL
