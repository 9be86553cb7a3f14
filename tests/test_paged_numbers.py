"""Row starts and lengths as the kernels of the paged cache take them from the device, where they may be any number: the host side
of the same header functions, compiled for the host alone, against whole numbers of any size."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2505_14201_amd", "csrc")

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#include "flashd_paged.h"
int main() {
    for (long long start, next, len, T, most, log2; std::scanf("%lld %lld %lld %lld %lld %lld", &start, &next, &len, &T, &most, &log2) == 6;) {
        const flashd::Seq s = flashd::seq_of((int)start, (int)next, (int)len, (int)T, (int)most);
        const int tokens = flashd::tokens_of(s.row0, (int)next, (int)T);
        std::printf("%d %d %d %d %d\n", s.row0, s.n, s.len, tokens, flashd::columns_beyond(tokens, s.n, (int)log2));
    }
}
"""

INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc to compile the header")
def test_any_start_and_length_stays_inside(tmp_path):
    src, exe = tmp_path / "seq_check.cpp", tmp_path / "seq_check"
    src.write_text(PROGRAM)
    subprocess.run(["hipcc", "-x", "hip", "--cuda-host-only", "-O2", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    edge = (INT_MIN, INT_MIN + 1, -5, -1, 0, 1, 2, 8, 9, 10, 1 << 30, INT_MAX - 1, INT_MAX)
    cases = [(a, b, n, T, most, 4 if most < 100 else 8) for a in edge for b in edge for n in edge for T in (0, 1, 9, 10 ** 7, INT_MAX)
             for most in (16, 48, 10 ** 9 // 256 * 256)]
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, timeout=300)
    got = [tuple(map(int, line.split())) for line in out.stdout.splitlines()]
    assert len(got) == len(cases)
    for (start, nxt, length, T, most, log2), (row0, n, have, tokens, beyond) in zip(cases, got):
        case = (start, nxt, length, T, most)
        assert row0 == max(start, 0) and have == min(max(length, 0), most), case
        assert tokens == max(min(max(nxt, 0), T) - row0, 0) and n == min(tokens, most - have), case
        assert n == 0 or row0 + n <= T, case
        assert beyond == -(-(tokens - n) // (1 << log2)), case
