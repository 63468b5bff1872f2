"""What the waves of an append to an 8-bit cache read of k and v, by the header that the kernel takes its addresses
from, compiled for the host: every element inside the call's tensors, every head read by one wave."""

import os
import subprocess

from paper_2605_05819_amd import build

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "append_units.h"

int main() {
    int bad = 0;
    for (int heads = 1; heads <= 17; ++heads)
        for (int dim : {64, 128, 256})
            for (int gap : {0, 24})
                for (int tokens : {1, 3, 16}) {
                    const long long stride = static_cast<long long>(heads) * dim + gap;
                    const long long size = (tokens - 1) * stride + static_cast<long long>(heads) * dim;
                    std::vector<int> seen[2] = {std::vector<int>(size), std::vector<int>(size)};
                    const int groups = (2 * heads + 3) / 4;             // workgroups of four waves
                    for (int unit = 0; unit < 4 * groups; ++unit) {
                        const cl::KvUnit u = cl::kv_unit(unit, heads);
                        if (u.head < 0 || u.head >= heads) ++bad, std::printf("heads %d wave %d: head %d\n", heads, unit, u.head);
                        for (int t = 0; t < cl::loaded_rows(u, tokens); ++t)
                            for (int i = 0; i < dim; ++i) {
                                const long long at = cl::row_offset(u, stride, dim, t) + i;
                                if (at < 0 || at >= size) {
                                    if (i == 0) std::printf("heads %d dim %d wave %d token %d: element %lld of %lld\n", heads, dim, unit, t, at, size);
                                    ++bad;
                                } else {
                                    ++seen[u.is_v][at];
                                }
                            }
                    }
                    for (const auto& s : seen)
                        for (long long at = 0; at < size; ++at)
                            if (s[at] != (at % stride < static_cast<long long>(heads) * dim)) ++bad;
                }
    return bad != 0;
}
"""


def test_every_read_is_inside_k_and_v(tmp_path):
    src, exe = tmp_path / "reads.cpp", tmp_path / "reads"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout[-3000:]


def test_the_kernel_takes_its_addresses_from_there():
    text = open(os.path.join(build.CSRC, "append8.hip")).read()
    for name in ("kv_unit(", "loaded_rows(", "row_offset("):
        assert text.count(name) == 1, name
