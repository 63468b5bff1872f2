"""The calls on pages, rows and beams refuse bad arguments before anything is enqueued (CPU: the addresses are never
dereferenced), and the binding refuses tensors that do not fit."""

import ctypes

import pytest
import torch

from paper_2605_05819_amd import cl
from tests.test_layer_refusals import FAKE, _raises, _refused

BIG = 1 << 40


def _pool(buffers=((FAKE, 64),), listed=True, **kw):
    arr = (cl.PageBufferC * max(1, len(buffers)))(*[cl.PageBufferC(*b) for b in buffers])
    d = dict(refs=FAKE, missing=0, buffers=ctypes.addressof(arr) if listed else 0, num_buffers=len(buffers), num_pages=100, page_size=16)
    d.update(kw)
    p = cl.PagePoolC(**d)
    p.keep = arr
    return p


def _fork(pool=None, **kw):
    a = dict(table=FAKE, kv_len=FAKE, rows=4, width=8, prefix=0, parents=FAKE, new=4, room=1, table2=BIG, len2=BIG, ws=FAKE, bytes=1 << 20)
    a.update(kw)
    return cl.lib().cl_kv_fork(ctypes.byref(pool or _pool()), a["table"], a["kv_len"], a["rows"], a["width"], a["prefix"],
                               a["parents"], a["new"], a["room"], a["table2"], a["len2"], a["ws"], a["bytes"], None)


def _reserve(pool=None, **kw):
    a = dict(table=FAKE, kv_len=FAKE, rows=4, width=8, prefix=0, want=FAKE, ws=FAKE, bytes=1 << 20)
    a.update(kw)
    return cl.lib().cl_kv_reserve(ctypes.byref(pool or _pool()), a["table"], a["kv_len"], a["rows"], a["width"], a["prefix"],
                                  a["want"], a["ws"], a["bytes"], None)


def _free(pool=None, **kw):
    a = dict(table=FAKE, kv_len=FAKE, rows=4, width=8, which=None, n=0)
    a.update(kw)
    return cl.lib().cl_kv_free(ctypes.byref(pool or _pool()), a["table"], a["kv_len"], a["rows"], a["width"], a["which"], a["n"], None)


def _compact(pool=None, tables=(FAKE,), sizes=(32,), n=None, ws=FAKE, bytes=1 << 20):
    t = (ctypes.c_void_p * max(1, len(tables)))(*tables)
    s = (ctypes.c_int64 * max(1, len(sizes)))(*sizes)
    return cl.lib().cl_kv_compact(ctypes.byref(pool or _pool()), len(tables) if n is None else n, t, s, ws, bytes, None)


def _copy(pool=None, src=FAKE, dst=FAKE, n=3):
    return cl.lib().cl_copy_pages(ctypes.byref(pool or _pool()), src, dst, n, None)


@pytest.mark.parametrize("kw,needle", [
    (dict(refs=0), "refs"), (dict(refs=FAKE + 2), "misaligned"), (dict(missing=FAKE + 1), "misaligned"),
    (dict(num_pages=0), "num_pages"), (dict(page_size=0), "page_size"), (dict(page_size=24), "page_size"),
    (dict(page_size=2048), "page_size"), (dict(num_buffers=-1), "num_buffers"), (dict(num_buffers=4097), "num_buffers"),
    (dict(listed=False), "num_buffers"), (dict(buffers=((0, 64),)), "null base"), (dict(buffers=((FAKE, 64), (FAKE, 0))), "buffer 1"),
    (dict(buffers=((FAKE, 1 << 31),)), "page_bytes")])
def test_pools(kw, needle):
    p = _pool(kw.pop("buffers")) if isinstance(kw.get("buffers"), tuple) else _pool(**kw)
    for call in (_fork, _reserve, _free, _compact, _copy):
        _refused(call(p), cl.CL_EINVAL, needle)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(table=0), cl.CL_EINVAL, "table"), (dict(kv_len=FAKE + 2), cl.CL_EINVAL, "kv_len"), (dict(rows=0), cl.CL_EINVAL, "positive"),
    (dict(width=0), cl.CL_EINVAL, "positive"), (dict(rows=(1 << 20) + 1), cl.CL_EUNSUPPORTED, "2^20"),
    (dict(width=(1 << 26) + 1), cl.CL_EUNSUPPORTED, "2^26"), (dict(rows=1 << 10, width=1 << 21), cl.CL_EUNSUPPORTED, "entries"),
    (dict(prefix=-1), cl.CL_EINVAL, "prefix_len"), (dict(ws=0), cl.CL_EWORKSPACE, "workspace"),
    (dict(bytes=100), cl.CL_EWORKSPACE, "workspace"), (dict(ws=FAKE + 16), cl.CL_EINVAL, "256-byte")])
def test_fork_and_reserve(kw, status, needle):
    _refused(_fork(**kw), status, needle)
    _refused(_reserve(**kw), status, needle)


@pytest.mark.parametrize("kw,needle", [
    (dict(parents=0), "parents"), (dict(parents=FAKE + 1), "parents"), (dict(new=0), "positive"), (dict(room=-1), "room"),
    (dict(room=(1 << 30) + 1), "room"), (dict(table2=0), "table"), (dict(len2=0), "table"), (dict(table2=FAKE), "overlap"),
    (dict(table2=FAKE + 124), "overlap"), (dict(table2=FAKE - 4), "overlap"), (dict(len2=FAKE + 12), "overlap")])
def test_fork(kw, needle):
    _refused(_fork(**kw), cl.CL_EINVAL, needle)


def test_reserve_free_compact_copy():
    _refused(_reserve(want=0), cl.CL_EINVAL, "want")
    _refused(_free(table=0), cl.CL_EINVAL, "table")
    _refused(_free(which=FAKE + 2, n=1), cl.CL_EINVAL, "rows")
    _refused(_free(which=FAKE, n=0), cl.CL_EINVAL, "num_rows")
    _refused(_compact(n=17), cl.CL_EINVAL, "num_tables")
    _refused(_compact(n=-1), cl.CL_EINVAL, "num_tables")
    _refused(_compact(tables=(FAKE, 0), sizes=(1, 1)), cl.CL_EINVAL, "table 1")
    _refused(_compact(sizes=(0,)), cl.CL_EINVAL, "table 0")
    _refused(_compact(bytes=10), cl.CL_EWORKSPACE, "workspace")
    _refused(_copy(src=0), cl.CL_EINVAL, "from or to")
    _refused(_copy(n=0), cl.CL_EINVAL, "n must")


def test_workspaces_cover_their_lists():
    for pages, rows in ((1, 1), (100, 5), (1 << 20, 1 << 20), (7, 100000), (1 << 30, 1)):
        need = cl.lib().cl_pages_workspace(ctypes.byref(_pool(num_pages=pages)), rows)
        assert need >= 4 * (4 * rows + pages) and need >= 12 * pages
    assert cl.lib().cl_pages_workspace(ctypes.byref(_pool(num_pages=(1 << 30) + 1)), 1) == 0
    _refused(_compact(_pool(num_pages=(1 << 30) + 1)), cl.CL_EUNSUPPORTED, "2^30")
    assert cl.lib().cl_pages_workspace(None, 1) == 0 and cl.lib().cl_pages_workspace(ctypes.byref(_pool()), 0) == 0


@pytest.mark.parametrize("kw,needle", [
    (dict(n=0), "num_arrays"), (dict(n=4097), "num_arrays"), (dict(src_rows=0), "src_rows"), (dict(rows=0), "src_rows and n"),
    (dict(index=0), "index"), (dict(index=FAKE + 2), "index"), (dict(src=0), "null src"), (dict(bytes=0), "row_bytes"),
    (dict(bytes=1 << 31), "row_bytes"), (dict(dst=FAKE + 79), "overlap")])
def test_gather_rows(kw, needle):
    a = dict(n=1, src=FAKE, dst=BIG, bytes=16, src_rows=5, index=FAKE, rows=3)
    a.update(kw)
    arr = cl.RowArrayC(a["src"], a["dst"], a["bytes"])
    _refused(cl.lib().cl_gather_rows(a["n"], ctypes.byref(arr), a["src_rows"], a["index"], a["rows"], None), cl.CL_EINVAL, needle)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(beams=0), cl.CL_EINVAL, "beams"), (dict(beams=65), cl.CL_EINVAL, "beams"), (dict(picks=0), cl.CL_EINVAL, "picks"),
    (dict(picks=65), cl.CL_EINVAL, "picks"), (dict(alpha=float("nan")), cl.CL_EINVAL, "alpha"), (dict(eos=-2), cl.CL_EINVAL, "eos"),
    (dict(eos=1000), cl.CL_EINVAL, "eos"), (dict(groups=0), cl.CL_EINVAL, "groups"), (dict(vocab=0), cl.CL_EINVAL, "vocab"),
    (dict(vocab=(1 << 19) + 1, stride=1 << 20), cl.CL_EUNSUPPORTED, "2^19"), (dict(vocab=1, picks=5, eos=0), cl.CL_EINVAL, "picks"),
    (dict(groups=1 << 23), cl.CL_EUNSUPPORTED, "2^24"), (dict(dt=7), cl.CL_EINVAL, "logits_dtype"), (dict(logits=0), cl.CL_EINVAL, "null"),
    (dict(logits=FAKE + 1), cl.CL_EINVAL, "aligned"), (dict(scores=FAKE + 2), cl.CL_EINVAL, "aligned"), (dict(stride=999), cl.CL_EINVAL, "stride"),
    (dict(lengths=None), cl.CL_EINVAL, "lengths"), (dict(lengths=None, alpha=0.0), cl.CL_EINVAL, "out_lengths"),
    (dict(finished=FAKE, eos=-1), cl.CL_EINVAL, "eos"), (dict(bytes=64), cl.CL_EWORKSPACE, "workspace"),
    (dict(ws=FAKE + 8), cl.CL_EINVAL, "256-byte")])
def test_beam_select(kw, status, needle):
    a = dict(alpha=0.5, beams=4, picks=4, eos=2, logits=FAKE, dt=cl.CL_BF16, stride=1000, groups=2, vocab=1000, scores=FAKE,
             lengths=FAKE, finished=None, ws=FAKE, bytes=1 << 30)
    a.update(kw)
    r = cl.BeamsC(a["alpha"], a["beams"], a["picks"], a["eos"])
    _refused(cl.lib().cl_beam_select(ctypes.byref(r), a["logits"], a["dt"], a["stride"], a["groups"], a["vocab"], a["scores"],
                                     a["lengths"], a["finished"], FAKE, FAKE, FAKE, FAKE, None, a["ws"], a["bytes"], None), status, needle)


def test_beam_workspace():
    lib = cl.lib()
    for beams, picks, groups, vocab in ((1, 1, 1, 1), (64, 64, 3, 1 << 19), (8, 16, 16, 128000), (4, 4, 1 << 16, 100)):
        r = cl.BeamsC(0.0, beams, picks, -1)
        need = lib.cl_beam_workspace(ctypes.byref(r), groups, vocab)
        assert need >= groups * beams * -(-vocab // 8192) * (8 * picks + 12)
    before = lib.cl_last_error()
    assert lib.cl_beam_workspace(None, 1, 1) == 0 and lib.cl_beam_workspace(ctypes.byref(cl.BeamsC(0.0, 0, 1, -1)), 1, 1) == 0
    assert lib.cl_last_error() == before


def test_binding_refuses_tensors_that_do_not_fit():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    _raises(lambda: cl.PagePool(i(4).long(), 16), "refs must have dtype")
    _raises(lambda: cl.PagePool(i(4, 2), 16), "refs must be")
    _raises(lambda: cl.PagePool(i(4), 16, [1]), "KvCache")
    _raises(lambda: cl.PagePool(i(4), 16), "on the GPU")
    rule = cl.Beams(2)
    x = torch.zeros((4, 10))
    _raises(lambda: cl.beam_select(rule, x.double(), x), "logits must be")
    _raises(lambda: cl.beam_select(rule, x[:3], x), "groups * beams")
    _raises(lambda: cl.beam_select(rule, x.t().contiguous().t(), x), "contiguous")
    _raises(lambda: cl.beam_select(rule, x, x), "on the GPU")
    _raises(lambda: cl.gather_rows([], i(3)), "one array")
    _raises(lambda: cl.gather_rows([x], i(3).long()), "index must have dtype")
