"""The host code of the 8-bit cache, the pages and the beams under clang's undefined-behaviour checks: their refusals and
workspace sizes, and sizes at the ends of the ranges, in a child process that loads the sanitized build."""

import ctypes
import itertools
import os
import subprocess
import sys

from paper_2605_05819_amd import build, cl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000


def test_workspace_sizes_at_the_ends_of_the_ranges():
    lib, most = cl.lib(), 0x7fffffff
    found = 0
    for beams, picks, groups, vocab in itertools.product((1, 64), (1, 64), (1, 1 << 12, 1 << 20, most), (1, 64, 1 << 19, most)):
        need = lib.cl_beam_workspace(ctypes.byref(cl.BeamsC(0.5, beams, picks, -1)), groups, vocab)
        if need:
            found += 1
            assert need >= groups * beams * (8 * picks + 12)
    assert found > 10
    for pages, rows in itertools.product((1, 1 << 30, most), (1, 1 << 20, most)):
        pool = cl.PagePoolC(FAKE, 0, 0, 0, pages, 16)
        need = lib.cl_pages_workspace(ctypes.byref(pool), rows)
        assert need >= 4 * (pages + 4 * rows) if rows <= 1 << 20 and pages <= 1 << 30 else need == 0
    for heads, q_len, seqs, width, prefix, block in itertools.product((1, 8), (1, 1 << 20), (1, most), (0, most), (0, most), (1, 16)):
        cc = cl.KvCache8C(FAKE, FAKE, FAKE, FAKE, most // (heads * 16), 16, heads, 128, block, cl.CL_BF16)
        bb = cl.KvBatchC(FAKE, FAKE, FAKE, FAKE, seqs, q_len, q_len, width, prefix, most)
        c2 = cl.KvCacheC(FAKE, FAKE, most // (heads * 16), 16, heads, 128, cl.CL_BF16)
        assert lib.cl_attention8_workspace(ctypes.byref(cc), ctypes.byref(bb), heads) == \
            lib.cl_attention_workspace(ctypes.byref(c2), ctypes.byref(bb), heads)


def test_abi_tests_pass_on_the_ubsan_build(tmp_path):
    lib = build.build_ubsan(str(tmp_path / "ubsan"))
    env = dict(os.environ, CL_LIBRARY=lib, UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1:report_error_type=1")
    tests = ["tests/test_cache8_refusals.py", "tests/test_pages_refusals.py",
             "tests/test_cache8_ubsan.py::test_workspace_sizes_at_the_ends_of_the_ranges"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-m", "not gpu", "-p", "no:cacheprovider"] + tests,
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = r.stdout + r.stderr
    assert "runtime error" not in out, out[-6000:]
    assert r.returncode == 0, out[-6000:]
