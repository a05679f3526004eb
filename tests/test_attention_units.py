"""The work split of attention on the matrix cores (csrc/units.h), built by a host
compiler: units of every tile against a count of what its rows see, and the bound
by which a call is taken against the most that sequences can have."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_10264_amd", "csrc")

PROGRAM = r"""
#define MVK_HD inline
#include "units.h"
#include <algorithm>
#include <cstdio>
#include <cstdlib>
using namespace mvk;

static void fail(const char* what, unsigned long a, unsigned long b, unsigned long c, unsigned long d) {
    printf("%s: %lu %lu %lu %lu\n", what, a, b, c, d);
    exit(1);
}

// tiles one after another, with 64-bit sums
template <uint32_t kRows, uint32_t kUnit, uint32_t kExtra>
static void one(uint32_t c, uint32_t n, uint32_t grp, bool closely) {
    const Tiles<kRows, kUnit, kExtra> t(c, n, grp);
    const uint64_t rows = (uint64_t)c * grp;
    if (t.count != (rows + kRows - 1) / kRows) fail("count", c, n, grp, t.count);
    uint64_t sum = 0;
    for (uint32_t i = 0; i < t.count; ++i) {
        const uint64_t row = std::min<uint64_t>((uint64_t)(i + 1) * kRows, rows) - 1;
        const int64_t sees = std::max<int64_t>((int64_t)n - c + (int64_t)(row / grp) + 1, 0);
        const uint64_t most = std::min<uint64_t>(std::max<int64_t>(n, c) - (int64_t)c + row / grp + 1, std::max(n, 1u));
        const uint64_t u = t.units(i);
        if (u < kExtra + 1 || (u - kExtra) * kUnit < (uint64_t)sees) fail("units too few", c, n, grp, i);
        if ((u - kExtra - 1) * kUnit >= most) fail("units too many", c, n, grp, i);
        if (t.before(i) != sum) fail("before", c, n, grp, i);
        sum += u;
    }
    if (t.all() != sum) fail("all", c, n, grp, sum);
    // one sequence that is all the call has
    if (closely && !units_fit<kRows, kUnit, kExtra>(c, grp, 1, 1, n)) fail("refused", c, n, grp, sum);
    const uint64_t bound = (rows / kRows + 1) * (n / kUnit + 1 + kExtra);
    if (sum > bound) fail("bound", c, n, grp, sum);
}
static void both(uint32_t c, uint32_t n, uint32_t grp, bool closely = true) {
    one<128, 64, 3>(c, n, grp, closely);
    one<32, 128, 0>(c, n, grp, closely);
}

int main() {
    for (uint32_t grp : {1u, 2u, 3u, 7u, 8u, 32u, 40u, 130u})
        for (uint32_t c : {0u, 1u, 2u, 15u, 16u, 17u, 127u, 128u, 129u, 300u, 1000u})
            for (uint32_t n : {0u, 1u, 2u, 31u, 63u, 64u, 65u, 127u, 128u, 129u, 256u, 500u, 999u, 1000u, 1001u, 5000u}) both(c, n, grp);
    srand(1);
    for (int i = 0; i < 3000; ++i) both(rand() % 5000, rand() % 3 ? rand() % 9000 : rand() % 200, 1 + rand() % 70);
    // large ones: a prompt of 2^18, a chunk over 2^30 entries, 2^24 new tokens with few entries
    both(1u << 18, 1u << 18, 8);
    both(513, (1u << 30) + 77, 3);
    both(1u << 24, 8192, 8);
    both(1u << 24, 0, 64);
    both(1000, 0x7fffffffu - 512, 1);

    struct Case { uint64_t tokens, grp, hk, count, cap; bool chunks, single; };
    const Case cases[] = {
        {64 * 8192, 8, 8, 64, 8192, true, true},       // a batch of prompts
        {200000, 8, 8, 1, 200000, true, true},         // one long prompt
        {262144, 1, 32, 1, 262144, true, true},
        {65536, 8, 8, 8, 1 << 20, true, true},         // few prompts in a table for long contexts
        {1 << 22, 8, 8, 512, 8192, true, true},
        {65535, 8, 8, 65535, 32768, true, true},       // single tokens
        {0x7fffffff, 1, 1, 1, 512, true, true},
        {1 << 20, 8, 8, 1, 1 << 20, false, false},     // 2^20 x 2^20 of 64 heads: too many
        {0x7fffffff, 1, 1, 1, 1u << 28, false, false},
        {1, 2, 1, 1, 0x7fffffff, false, false},        // offsets of entries times heads
        {65535, 65535, 65535, 65535, 0x7fffffff, false, false},
        {0x7fffffff, 0x7fffffff, 65535, 65535, 0x7fffffff, false, false},
    };
    for (const Case& c : cases) {
        if (units_fit<128, 64, 3>(c.tokens, c.grp, c.hk, c.count, c.cap) != c.chunks) fail("chunks", c.tokens, c.grp, c.hk, c.cap);
        if (units_fit<32, 128, 0>(c.tokens, c.grp, c.hk, c.count, c.cap) != c.single) fail("tokens", c.tokens, c.grp, c.hk, c.cap);
    }
    // the last size that is taken, and the next: its units stay below 2^32 - 1
    uint64_t lo = 1, hi = 1ull << 31;
    while (hi - lo > 1) ((units_fit<128, 64, 3>((lo + hi) / 2, 1, 32, 1, 1 << 20)) ? lo : hi) = (lo + hi) / 2;
    const uint64_t most = (lo / 128 + 1) * ((1 << 20) / 64 + 4) * 32;
    if (most >= 0xffffffffull || most < 0xfff00000ull) fail("edge", lo, most, 0, 0);
    puts("ok");
}
"""


def test_units(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("g++ not found")
    src, exe = tmp_path / "units.cpp", str(tmp_path / "units")
    src.write_text(PROGRAM)
    r = subprocess.run([cxx, "-O2", "-std=c++17", "-Wall", "-Wno-unknown-pragmas", f"-I{CSRC}", "-o", exe, str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
