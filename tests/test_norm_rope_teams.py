"""Which lanes hold which elements of a head's row in norm + rope (csrc/bf1_team.h), over every
size that the operator takes: a team fits the wave that sums it, and every element
belongs to one lane, next to the other half of its pair.  Compiled with the host compiler."""

import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2608_20427_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "bf1_team.h"
template <bool INTER, int P>
bool holds(int d, int half) {
    const int lanes = 1 << bf1::team_shift(d, half, P);
    if (lanes > 64) return false;
    std::vector<int> owner(d, -1), slot(d, -1);
    for (int l = 0; l < lanes; ++l) {
        const bf1::Lane x = bf1::lane_of<INTER, P>(l, d, half);
        if (x.na < 0 || x.nb < 0 || x.na > P || x.nb > P) return false;
        for (int k = 0; k < 2 * P; ++k) {
            if (k % P >= (k < P ? x.na : x.nb)) continue;
            const int at = (k < P ? x.a : x.b) + k % P;
            if (at < 0 || at >= d || owner[at] >= 0 || (at < 2 * half) != x.turn) return false;
            owner[at] = l;
            slot[at] = k;
        }
        for (int i = 0; x.turn && i < P; ++i) {  // pair x.pair + i is elements e0 and e1 of the lane
            if (i >= x.pairs) continue;
            const int p = x.pair + i, a = INTER ? 2 * p : p, b = INTER ? 2 * p + 1 : half + p;
            if (owner[a] != l || owner[b] != l || slot[a] != (INTER ? 2 * i : i) || slot[b] != (INTER ? 2 * i + 1 : P + i))
                return false;
        }
    }
    for (int e = 0; e < d; ++e)
        if (owner[e] < 0) return false;
    return true;
}
int main() {
    long sizes = 0, eights = 0;
    for (int bytes = 2; bytes <= 4; bytes += 2)
        for (int d = 2; d <= 512; d += 2)
            for (int half = 1; 2 * half <= d; ++half, ++sizes) {
                const int P = bf1::pairs_of(bytes, d, half);
                const bool ok = P == 8 ? holds<false, 8>(d, half) && holds<true, 8>(d, half)
                                       : P == 4 && holds<false, 4>(d, half) && holds<true, 4>(d, half);
                // eight elements for float32 rows only where none is read 16 bytes at a time
                const bool apt = bytes == 2 ? P == 8 : P == 4 || (d >= 508 && (half % 4 != 0 || (d - 2 * half) % 4 != 0));
                if (!ok || !apt) std::printf("bytes %d d %d half %d P %d\n", bytes, d, half, P);
                eights += bytes == 4 && P == 8;
            }
    std::printf("%ld sizes, %ld of float32 in eights\n", sizes, eights);
}
"""


def test_every_team_fits_a_wave(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    src, exe = tmp_path / "team.cpp", tmp_path / "team"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-O2", "-std=c++17", "-fsanitize=undefined", "-D_GLIBCXX_ASSERTIONS", "-I", CSRC, str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert out == "65792 sizes, 384 of float32 in eights\n"
