"""Whether strided rows share memory (csrc/overlap.h), built by a host compiler,
against marking every byte."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_10264_amd", "csrc")

PROGRAM = r"""
#include "overlap.h"
#include <cstdio>
#include <cstdlib>
#include <cstring>
using mvk::RowSet;
using mvk::share_memory;

int main() {
    srand(3);
    auto below = [](int n) { return (uint64_t)(rand() % n); };
    static char mark[2000];
    long met = 0, refused = 0;
    for (long it = 0; it < 1000000; ++it) {
        const RowSet a{(void*)(uintptr_t)(1000 + below(60)), below(4), below(40), below(4), below(14), 1 + below(6)};
        const RowSet b{(void*)(uintptr_t)(1000 + below(60)), below(4), below(4) ? a.s0 : below(40), below(4),
                       below(2) ? a.s1 : below(14), 1 + below(6)};
        memset(mark, 0, sizeof mark);
        bool meet = false;
        for (uint64_t i = 0; i < a.n0; ++i)
            for (uint64_t j = 0; j < a.n1; ++j) memset(mark + a.begin() - 1000 + i * a.s0 + j * a.s1, 1, a.len);
        for (uint64_t i = 0; i < b.n0; ++i)
            for (uint64_t j = 0; j < b.n1; ++j)
                for (uint64_t k = 0; k < b.len; ++k) meet |= mark[b.begin() - 1000 + i * b.s0 + j * b.s1 + k];
        const bool got = share_memory(a, b), exact = a.n0 < 2 || b.n0 < 2 || a.s0 == b.s0;
        if (meet ? !got : got && exact) {
            printf("%s: p %lu %lu n0 %lu %lu s0 %lu %lu n1 %lu %lu s1 %lu %lu len %lu %lu\n", meet ? "missed" : "refused",
                   a.begin(), b.begin(), a.n0, b.n0, a.s0, b.s0, a.n1, b.n1, a.s1, b.s1, a.len, b.len);
            return 1;
        }
        met += meet, refused += got && !meet;
    }
    // rows near the ends of what 64 bits hold
    const uint64_t far = 1ull << 61;
    const void *p = (void*)(1ull << 46), *q = (void*)((1ull << 46) + 64);
    if (share_memory({p, 3, far, 2, 128, 64}, {q, 3, far, 2, 128, 64}) || !share_memory({p, 3, far, 2, 128, 65}, {q, 3, far, 2, 128, 64}) ||
        share_memory({p, 2, 256, 1 << 16, 1ull << 45, 64}, {q, 2, 256, 1 << 16, 1ull << 45, 64})) {
        puts("large strides");
        return 1;
    }
    puts(met > 100000 && refused < 10000 ? "ok" : "few");
}
"""


def test_against_every_byte(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("g++ not found")
    src, exe = tmp_path / "overlap.cpp", str(tmp_path / "overlap")
    src.write_text(PROGRAM)
    r = subprocess.run([cxx, "-O2", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", f"-I{CSRC}",
                        "-o", exe, str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr
