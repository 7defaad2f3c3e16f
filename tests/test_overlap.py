"""Whether two strided matrices share a byte (CPU: the rule is plain C++), against marked bytes, and at sizes that no 64-bit product holds."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include <random>
#include "overlap.h"
using namespace dcnn;
int main() {
    std::mt19937 rng(1);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
    static char base[4096], mark[4096];
    int bad = 0, met = 0;
    const int trials = 400000;
    for (int t = 0; t < trials; ++t) {
        Bytes m[2];
        const int common = 1 + upto(60);
        for (Bytes& x : m) {
            x.width = 1 + upto(12);
            x.ld = x.width + upto(30);
            if (upto(3) == 0 && common >= x.width) x.ld = common;      // columns of one buffer
            x.rows = upto(9);
            if (x.rows == 1 && upto(2)) x.ld = upto(3) - 1;             // a single row's is nothing's
            x.p = base + upto(200);
        }
        memset(mark, 0, sizeof(mark));
        bool want = false;
        for (int i = 0; i < m[0].rows; ++i) memset(mark + ((const char*)m[0].p - base) + i * m[0].ld, 1, m[0].width);
        for (int i = 0; i < m[1].rows; ++i)
            for (int c = 0; c < m[1].width; ++c) want |= mark[((const char*)m[1].p - base) + i * m[1].ld + c] != 0;
        if (overlap(m[0], m[1]) != want || overlap(m[1], m[0]) != want) ++bad;
        met += want;
    }
    if (met < trials / 10 || met > trials - trials / 10) ++bad, printf("%d of %d meet\n", met, trials);
    // long matrices: columns of one wide buffer, one byte apart and one byte in
    const int64_t rows = 0x7fffffff, ld = (int64_t)0x7fffffff * 4;
    char* const at = reinterpret_cast<char*>((uintptr_t)1 << 40);
    const Bytes left{"", at, rows, ld, 64}, right{"", at + 64, rows, ld, 64}, in{"", at + 63, rows, ld, 64}, wide{"", at + 64, 1, 1 << 20, 1 << 20};
    if (overlap(left, right) || overlap(right, left) || !overlap(left, in) || !overlap(in, right) || !overlap(right, wide) || overlap(left, wide)) ++bad, printf("columns\n");
    // leading dimensions that differ: they meet after so many rows
    const Bytes a{"", at, 1000000, 1001, 1}, b{"", at + 500, 1000000, 1000, 1}, short_b{"", at + 500, 500, 1000, 1}, next_b{"", at + 500, 501, 1000, 1};
    if (!overlap(a, b) || overlap(a, short_b) || !overlap(a, next_b) || overlap(short_b, a) || !overlap(next_b, a)) ++bad, printf("drift\n");
    const Bytes none{"", nullptr, 4, 4, 4}, empty{"", at, 0, 64, 64};
    if (overlap(none, left) || overlap(left, none) || overlap(empty, left) || overlap(left, empty)) ++bad, printf("empty\n");
    printf("%d wrong\n", bad);
    return bad != 0;
}
"""


def test_overlap_against_marked_bytes(tmp_path):
    src = tmp_path / "overlap.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "overlap"
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2203_03996_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
