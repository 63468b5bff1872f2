"""The host code of the entry points between a layer's linears under clang's
undefined-behaviour checks: their refusals, workspace sizes and plans
(``tests/test_layer_refusals.py``), the rotary frequencies
(``tests/test_layer_oracle.py``), and sizes at the ends of the descriptors'
ranges, in a child process that loads the sanitized build.  A report ends that
process with a nonzero status and is printed here."""

import ctypes
import itertools
import os
import subprocess
import sys

from paper_2605_05819_amd import build, cl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000


def test_workspace_sizes_at_the_ends_of_the_ranges():
    """Products of the largest sizes neither wrap nor shrink: 0 (refused) or at least the partial results of two
    splits; a larger batch never needs less than none."""
    lib = cl.lib()
    most = 0x7fffffff
    sizes = 0
    for heads, group, q_len, seqs, width, prefix, keys, page, dim in itertools.product(
            (1, 8), (1, 16), (1, 2048, 1 << 24), (1, 4096, most), (0, 1, most), (0, 1 << 20, most), (0, 1, most), (1, 1024),
            (64, 256)):
        cc = cl.KvCacheC(FAKE, FAKE, most // (heads * page), page, heads, dim, cl.CL_FP16)
        tokens = min(q_len, 1 << 20)
        bb = cl.KvBatchC(FAKE, FAKE, FAKE, FAKE, seqs, tokens, q_len, width, prefix, keys)
        need = lib.cl_attention_workspace(ctypes.byref(cc), ctypes.byref(bb), heads * group)
        if need:
            sizes += 1
            assert 2 * tokens * heads * group * (dim + 2) * 4 <= need <= 128 * tokens * heads * group * (dim + 2) * 4 + 512
    assert sizes > 100


def test_layer_abi_tests_pass_on_the_ubsan_build(tmp_path):
    lib = build.build_ubsan(str(tmp_path / "ubsan"))
    env = dict(os.environ, CL_LIBRARY=lib, UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1:report_error_type=1")
    tests = ["tests/test_layer_refusals.py", "tests/test_layer_oracle.py",
             "tests/test_layer_ubsan.py::test_workspace_sizes_at_the_ends_of_the_ranges"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-m", "not gpu", "-p", "no:cacheprovider"] + tests,
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = r.stdout + r.stderr
    assert "runtime error" not in out, out[-6000:]
    assert r.returncode == 0, out[-6000:]
