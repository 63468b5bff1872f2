"""The calls over a cache of 8 bits refuse bad arguments before anything is enqueued (CPU: the addresses are never
dereferenced), and the binding refuses tensors that do not fit."""

import ctypes

import pytest
import torch

from paper_2605_05819_amd import cl
from tests.test_layer_refusals import DESCRIPTORS, FAKE, _kv, _raises, _refused


def _kv8(cache=None, batch=None):
    c = dict(k=FAKE, v=FAKE, k_scale=FAKE + 1, v_scale=FAKE + 3, num_pages=10, page_size=16, kv_heads=2, head_dim=128, block=8,
             dtype=cl.CL_FP16)
    c.update(cache or {})
    return cl.KvCache8C(**c), _kv({}, batch)[1]


def _calls(cc, bb):
    lib, c, b = cl.lib(), ctypes.byref(cc), ctypes.byref(bb)
    return [lambda: lib.cl_attention8(c, b, FAKE, 1024, 8, 0.1, 1, 0, FAKE, cl.CL_FP16, None, FAKE, 1 << 30, None),
            lambda: lib.cl_kv_append8(c, b, None, FAKE, 1024, 8, FAKE, 256, FAKE, 256, None, None, 1e-6, None, FAKE, None),
            lambda: lib.cl_kv_read8(c, b, FAKE, FAKE, None)]


@pytest.mark.parametrize("c,b,status,needle", DESCRIPTORS + [
    (dict(k_scale=0), {}, cl.CL_EINVAL, "k_scale"), (dict(v_scale=0), {}, cl.CL_EINVAL, "v_scale"),
    (dict(block=0), {}, cl.CL_EINVAL, "block"), (dict(block=3), {}, cl.CL_EINVAL, "block"),
    (dict(block=32), {}, cl.CL_EINVAL, "block")])
def test_cache_and_batch_descriptors(c, b, status, needle):
    cc, bb = _kv8(c, b)
    for call in _calls(cc, bb):
        _refused(call(), status, needle)
    before = cl.lib().cl_last_error()
    assert cl.lib().cl_attention8_workspace(ctypes.byref(cc), ctypes.byref(bb), 8) == 0 and cl.lib().cl_last_error() == before


def test_null_descriptors():
    lib, (cc, bb) = cl.lib(), _kv8()
    for c, b in ((None, ctypes.byref(bb)), (ctypes.byref(cc), None)):
        _refused(lib.cl_kv_read8(c, b, FAKE, FAKE, None), cl.CL_EINVAL, "descriptor")
        assert lib.cl_attention8_workspace(c, b, 8) == 0


@pytest.mark.parametrize("kw,status,needle", [
    (dict(q=0), cl.CL_EINVAL, "null"), (dict(q=FAKE + 2), cl.CL_EINVAL, "16-byte"), (dict(stride=1016), cl.CL_EINVAL, "shorter"),
    (dict(heads=7), cl.CL_EINVAL, "multiple"), (dict(scale=float("nan")), cl.CL_EINVAL, "scale"),
    (dict(window=-1), cl.CL_EINVAL, "window"), (dict(dt=9), cl.CL_EINVAL, "out_dtype"), (dict(lse=FAKE + 2), cl.CL_EINVAL, "lse")])
def test_attention_arguments(kw, status, needle):
    cc, bb = _kv8()
    a = dict(q=FAKE, stride=1024, heads=8, scale=0.1, window=0, out=FAKE, dt=cl.CL_FP16, lse=None)
    a.update(kw)
    _refused(cl.lib().cl_attention8(ctypes.byref(cc), ctypes.byref(bb), a["q"], a["stride"], a["heads"], a["scale"], 1,
                                    a["window"], a["out"], a["dt"], a["lse"], FAKE, 1 << 30, None), status, needle)


def test_attention_workspace_is_that_of_16_bits():
    for batch in (dict(max_kv_len=1 << 20, table_width=1 << 16), dict(prefix_len=5000, prefix_table=FAKE)):
        cc, bb = _kv8({}, batch)
        c2, b2 = _kv({}, batch)
        need = cl.lib().cl_attention8_workspace(ctypes.byref(cc), ctypes.byref(bb), 8)
        assert need > 0 and need == cl.lib().cl_attention_workspace(ctypes.byref(c2), ctypes.byref(b2), 8)
        _refused(cl.lib().cl_attention8(ctypes.byref(cc), ctypes.byref(bb), FAKE, 1024, 8, 0.1, 1, 0, FAKE, cl.CL_FP16, None, FAKE,
                                        need - 1, None), cl.CL_EWORKSPACE, "workspace")


@pytest.mark.parametrize("kw,needle", [
    (dict(k=0), "null k"), (dict(q=0), "go together"), (dict(q_out=0), "q_out"), (dict(ks=255), "shorter"),
    (dict(pos=FAKE + 2), "positions"), (dict(rope=cl.RopeC(FAKE, 136, 0, 1.0)), "rot_dim")])
def test_append_arguments(kw, needle):
    cc, bb = _kv8()
    a = dict(rope=None, q=FAKE, qs=1024, heads=8, k=FAKE, ks=256, v=FAKE, vs=256, pos=None, q_out=FAKE)
    a.update(kw)
    rope = None if a["rope"] is None else ctypes.byref(a["rope"])
    _refused(cl.lib().cl_kv_append8(ctypes.byref(cc), ctypes.byref(bb), rope, a["q"], a["qs"], a["heads"], a["k"], a["ks"],
                                    a["v"], a["vs"], None, None, 1e-6, a["pos"], a["q_out"], None), cl.CL_EINVAL, needle)


@pytest.mark.parametrize("k,v", [(0, FAKE), (FAKE, 0), (FAKE + 8, FAKE), (FAKE, FAKE + 2)])
def test_read_arguments(k, v):
    cc, bb = _kv8()
    _refused(cl.lib().cl_kv_read8(ctypes.byref(cc), ctypes.byref(bb), k, v, None), cl.CL_EINVAL, "16-byte")
    cc, bb = _kv()
    _refused(cl.lib().cl_kv_read(ctypes.byref(cc), ctypes.byref(bb), k, v, None), cl.CL_EINVAL, "16-byte")


def test_binding_refuses_tensors_that_do_not_fit():
    k = torch.zeros((4, 2, 16, 64), dtype=torch.uint8)
    s = torch.zeros((4, 2, 2), dtype=torch.uint8)
    half = torch.float16
    _raises(lambda: cl.KvCache8(k, k, s, s, torch.float32), "dtype must be")
    _raises(lambda: cl.KvCache8(k.float(), k, s, s, half), "k must have dtype")
    _raises(lambda: cl.KvCache8(k, k[:3], s, s, half), "v must have shape")
    _raises(lambda: cl.KvCache8(k, k, s[:3], s, half), "k_scale must be")
    _raises(lambda: cl.KvCache8(k, k, torch.zeros((4, 2, 3), dtype=torch.uint8), s, half), "k_scale must be")
    _raises(lambda: cl.KvCache8(k, k, s, s[..., :1].contiguous(), half), "v_scale must have shape")
    _raises(lambda: cl.KvCache8(k, k, s, s, half), "on the GPU")
    _raises(lambda: cl.KvCache8.empty(4, 16, 2, 64, block=5, device="cpu"), "divide")
