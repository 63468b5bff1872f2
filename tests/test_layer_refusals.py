"""The entry points between a layer's linears refuse bad arguments before anything is enqueued (CPU: the
addresses are never dereferenced), and the binding refuses tensors that do not fit."""

import ctypes

import pytest
import torch

from paper_2605_05819_amd import cl

FAKE = 0x100000


def _kv(cache=None, batch=None):
    c = dict(k=FAKE, v=FAKE, num_pages=10, page_size=16, kv_heads=2, head_dim=128, dtype=cl.CL_FP16)
    b = dict(q_start=0, kv_len=FAKE, page_table=FAKE, prefix_table=0, num_seqs=3, tokens=3, q_len=1, table_width=4,
             prefix_len=0, max_kv_len=64)
    c.update(cache or {})
    b.update(batch or {})
    return cl.KvCacheC(**c), cl.KvBatchC(**b)


def _refused(status, want, needle):
    assert status == want, cl.lib().cl_last_error()
    assert needle in cl.lib().cl_last_error().decode(), cl.lib().cl_last_error()


DESCRIPTORS = [
    (dict(k=0), {}, cl.CL_EINVAL, "non-null"),
    (dict(v=FAKE + 8), {}, cl.CL_EINVAL, "16-byte"),
    (dict(dtype=cl.CL_FP32), {}, cl.CL_EINVAL, "dtype"),
    (dict(num_pages=0), {}, cl.CL_EINVAL, "positive"),
    (dict(page_size=24), {}, cl.CL_EINVAL, "power of two"),
    (dict(page_size=2048), {}, cl.CL_EINVAL, "power of two"),
    (dict(head_dim=96), {}, cl.CL_EUNSUPPORTED, "head_dim"),
    ({}, dict(num_seqs=0), cl.CL_EINVAL, "positive"),
    ({}, dict(tokens=4), cl.CL_EINVAL, "num_seqs * q_len"),
    ({}, dict(kv_len=0), cl.CL_EINVAL, "kv_len"),
    ({}, dict(kv_len=FAKE + 2), cl.CL_EINVAL, "kv_len"),
    ({}, dict(page_table=0), cl.CL_EINVAL, "page_table"),
    ({}, dict(prefix_len=5), cl.CL_EINVAL, "prefix_table"),
    ({}, dict(max_kv_len=-1), cl.CL_EINVAL, "negative"),
    ({}, dict(q_start=FAKE + 1), cl.CL_EINVAL, "q_start"),
]


@pytest.mark.parametrize("c,b,status,needle", DESCRIPTORS)
def test_cache_and_batch_descriptors(c, b, status, needle):
    cc, bb = _kv(c, b)
    lib = cl.lib()
    _refused(lib.cl_attention(ctypes.byref(cc), ctypes.byref(bb), FAKE, 1024, 8, 0.1, 1, 0, FAKE, cl.CL_FP16, None, FAKE,
                              1 << 30, None), status, needle)
    _refused(lib.cl_kv_append(ctypes.byref(cc), ctypes.byref(bb), None, FAKE, 1024, 8, FAKE, 256, FAKE, 256, None, None,
                              1e-6, None, FAKE, None), status, needle)
    before = lib.cl_last_error()
    assert lib.cl_attention_workspace(ctypes.byref(cc), ctypes.byref(bb), 8) == 0 and lib.cl_last_error() == before


@pytest.mark.parametrize("kw,status,needle", [
    (dict(q=0), cl.CL_EINVAL, "null"), (dict(out=0), cl.CL_EINVAL, "null"), (dict(q=FAKE + 2), cl.CL_EINVAL, "16-byte"),
    (dict(out=FAKE + 8), cl.CL_EINVAL, "16-byte"), (dict(stride=1028), cl.CL_EINVAL, "16-byte"),
    (dict(stride=1016), cl.CL_EINVAL, "shorter"), (dict(heads=7), cl.CL_EINVAL, "multiple"),
    (dict(heads=0), cl.CL_EINVAL, "multiple"), (dict(scale=float("nan")), cl.CL_EINVAL, "scale"),
    (dict(window=-1), cl.CL_EINVAL, "window"), (dict(dt=9), cl.CL_EINVAL, "out_dtype"),
    (dict(lse=FAKE + 2), cl.CL_EINVAL, "lse")])
def test_attention_arguments(kw, status, needle):
    cc, bb = _kv()
    a = dict(q=FAKE, stride=1024, heads=8, scale=0.1, window=0, out=FAKE, dt=cl.CL_FP16, lse=None)
    a.update(kw)
    _refused(cl.lib().cl_attention(ctypes.byref(cc), ctypes.byref(bb), a["q"], a["stride"], a["heads"], a["scale"], 1,
                                   a["window"], a["out"], a["dt"], a["lse"], FAKE, 1 << 30, None), status, needle)


@pytest.mark.parametrize("heads,batch", [
    (8, dict(tokens=1 << 28, num_seqs=1 << 28)),                                                    # rows
    (8, dict(tokens=1 << 20, q_len=1 << 20, num_seqs=1 << 22, q_start=FAKE)),                       # workgroups
    (1 << 12, dict(tokens=1 << 18, q_len=1 << 18, num_seqs=0x7fffffff, q_start=FAKE, max_kv_len=1 << 30))])
def test_attention_beyond_32_bit_numbers(heads, batch):
    cc, bb = _kv({}, batch)
    lib = cl.lib()
    _refused(lib.cl_attention(ctypes.byref(cc), ctypes.byref(bb), FAKE, heads * 128, heads, 0.1, 1, 0, FAKE, cl.CL_FP16, None,
                              FAKE, (1 << 63) - 1, None), cl.CL_EUNSUPPORTED, "2^31")
    before = lib.cl_last_error()
    assert lib.cl_attention_workspace(ctypes.byref(cc), ctypes.byref(bb), heads) == 0 and lib.cl_last_error() == before


@pytest.mark.parametrize("kw,needle", [
    (dict(k=0), "null k"), (dict(v=0), "null k or v"), (dict(q=0), "go together"), (dict(heads=0), "go together"),
    (dict(q_out=0), "q_out"), (dict(q=FAKE + 1), "misaligned"), (dict(ks=255), "shorter"), (dict(vs=0), "shorter"),
    (dict(qs=8 * 128 - 1), "shorter"), (dict(pos=FAKE + 2), "positions"), (dict(qn=FAKE, eps=-1.0), "eps"),
    (dict(rope=cl.RopeC(0, 64, 0, 1.0)), "inv_freq"), (dict(rope=cl.RopeC(FAKE, 20, 0, 1.0)), "rot_dim"),
    (dict(rope=cl.RopeC(FAKE, 136, 0, 1.0)), "rot_dim"), (dict(rope=cl.RopeC(FAKE, 64, 0, float("inf"))), "magnitude")])
def test_append_arguments(kw, needle):
    cc, bb = _kv()
    a = dict(rope=None, q=FAKE, qs=1024, heads=8, k=FAKE, ks=256, v=FAKE, vs=256, qn=None, eps=1e-6, pos=None, q_out=FAKE)
    a.update(kw)
    rope = None if a["rope"] is None else ctypes.byref(a["rope"])
    _refused(cl.lib().cl_kv_append(ctypes.byref(cc), ctypes.byref(bb), rope, a["q"], a["qs"], a["heads"], a["k"], a["ks"],
                                   a["v"], a["vs"], a["qn"], None, a["eps"], a["pos"], a["q_out"], None), cl.CL_EINVAL,
             needle)


@pytest.mark.parametrize("kw,needle", [
    (dict(num_experts=0), "num_experts"), (dict(num_experts=1025), "num_experts"), (dict(k=0), "k must"),
    (dict(k=65, num_experts=128), "k must"), (dict(score=3), "score"), (dict(groups=5), "groups"),
    (dict(groups=0), "groups"), (dict(groups=8, top_groups=9), "top_groups"), (dict(group_best=3), "group_best"),
    (dict(groups=8, top_groups=1, k=9), "fewer"), (dict(scale=float("inf")), "scale"), (dict(bias=FAKE + 1), "misaligned")])
def test_router(kw, needle):
    r = dict(bias=0, num_experts=64, k=8, score=1, groups=1, top_groups=1, group_best=1, renormalize=1, scale=1.0)
    r.update(kw)
    rc = cl.RouterC(**r)
    _refused(cl.lib().cl_moe_route(ctypes.byref(rc), FAKE, cl.CL_FP32, 4, FAKE, FAKE, 0, None, None, 0, None, None),
             cl.CL_EINVAL, needle)


def test_route_arguments():
    lib, rc = cl.lib(), cl.RouterC(0, 64, 8, 1, 1, 1, 1, 1, 1.0)
    two = (ctypes.c_void_p * 2)(FAKE, FAKE)
    lv = (ctypes.c_int32 * 3)(0, 8, 8)
    call = lambda logits=FAKE, dt=cl.CL_FP32, T=4, tables=0, er=None, levels=None, n=0, sr=None: lib.cl_moe_route(  # noqa: E731
        ctypes.byref(rc), logits, dt, T, FAKE, FAKE, tables, er, levels, n, sr, None)
    _refused(call(logits=0), cl.CL_EINVAL, "null")
    _refused(call(logits=FAKE + 2), cl.CL_EINVAL, "misaligned")
    _refused(call(dt=0), cl.CL_EINVAL, "logits_dtype")
    _refused(call(T=0), cl.CL_EINVAL, "T must")
    _refused(call(tables=5), cl.CL_EINVAL, "tables")
    _refused(call(tables=2), cl.CL_EINVAL, "null rank")
    _refused(call(tables=2, er=two, levels=lv, n=0, sr=two), cl.CL_EINVAL, "nlevels")
    _refused(call(tables=2, er=two, levels=lv, n=3, sr=two), cl.CL_EINVAL, "strictly increasing")
    _refused(call(tables=2, er=two, levels=lv, n=2, sr=(ctypes.c_void_p * 2)(FAKE, 0)), cl.CL_EINVAL, "rank table 1")
    assert lib.cl_moe_route(None, FAKE, cl.CL_FP32, 4, FAKE, FAKE, 0, None, None, 0, None, None) == cl.CL_EINVAL


@pytest.mark.parametrize("kw,status,needle", [
    (dict(weight=0), cl.CL_EINVAL, "null"), (dict(y=0), cl.CL_EINVAL, "null"), (dict(out=0), cl.CL_EINVAL, "null"),
    (dict(kind=3), cl.CL_EINVAL, "kind"), (dict(w_dtype=0), cl.CL_EINVAL, "dtypes"), (dict(eps=-1.0), cl.CL_EINVAL, "eps"),
    (dict(alpha=float("nan")), cl.CL_EINVAL, "alpha"), (dict(T=0), cl.CL_EINVAL, "positive"),
    (dict(d=0), cl.CL_EINVAL, "positive"), (dict(d=32769), cl.CL_EUNSUPPORTED, "32768"),
    (dict(slots=2), cl.CL_EINVAL, "go together"), (dict(slots=65, sw=FAKE), cl.CL_EINVAL, "slots"),
    (dict(y=FAKE + 1), cl.CL_EINVAL, "aligned"), (dict(out=FAKE + 2), cl.CL_EINVAL, "aligned")])
def test_residual_norm_arguments(kw, status, needle):
    a = dict(weight=FAKE, w_dtype=cl.CL_FP16, kind=1, eps=1e-6, alpha=1.0, y=FAKE, slots=0, sw=None, out=FAKE, T=2, d=64)
    a.update(kw)
    nc = cl.NormC(a["weight"], 0, 0, 0, a["w_dtype"], a["kind"], 0, a["eps"], a["alpha"], 1.0)
    _refused(cl.lib().cl_residual_norm(ctypes.byref(nc), a["y"], cl.CL_FP16, a["slots"], a["sw"], None, None, cl.CL_FP16,
                                       a["out"], cl.CL_FP32, a["T"], a["d"], None), status, needle)


def _raises(fn, needle):
    with pytest.raises(ValueError) as e:
        fn()
    assert needle in str(e.value), str(e.value)


def test_binding_refuses_tensors_that_do_not_fit():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    k = torch.zeros((4, 2, 16, 64), dtype=torch.float16)
    _raises(lambda: cl.KvCache(k.float(), k.float()), "dtype")
    _raises(lambda: cl.KvCache(k, k.bfloat16()), "v must have dtype")
    _raises(lambda: cl.KvCache(k, k[:3]), "v must have shape")
    _raises(lambda: cl.KvCache(k.transpose(1, 2), k), "contiguous")
    _raises(lambda: cl.KvCache(k, k), "on the GPU")
    _raises(lambda: cl.KvBatch(i(2).long(), i(2, 3), 2), "kv_len must have dtype")
    _raises(lambda: cl.KvBatch(i(2), i(3, 3), 2), "page_table")
    _raises(lambda: cl.KvBatch(i(2), i(2, 3), 3), "num_seqs * q_len")
    _raises(lambda: cl.KvBatch(i(2), i(2, 3), 2, q_start=i(2)), "q_start must have shape")
    _raises(lambda: cl.KvBatch(i(2), i(2, 3), 2, prefix_len=4), "go together")
    _raises(lambda: cl.KvBatch(i(2), i(2, 3), 2), "on the GPU")
    _raises(lambda: cl.Rope(torch.zeros(4, dtype=torch.float64)), "inv_freq must have dtype")
    _raises(lambda: cl.Router(8, 2, "best"), "score must be")
    _raises(lambda: cl.rope_frequencies(64, kind="cubic"), "kind must be")
    r = cl.Router(8, 2)
    x = torch.zeros((3, 8))
    _raises(lambda: cl.moe_route(r, x.double()), "logits must have dtype")
    _raises(lambda: cl.moe_route(r, x), "on the GPU")
    w = torch.zeros(8)
    _raises(lambda: cl.residual_norm(x.long(), w), "y must have dtype")
    _raises(lambda: cl.residual_norm(x, w), "on the GPU")
