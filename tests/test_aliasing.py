"""Whether arrays share memory (csrc/aliasing.hpp, compiled for the host): every pair of a
few thousand small arrays against the sets of their bytes."""
import os
import random
import subprocess

from helpers import ROOT

MAIN = r"""
#include <cstdio>
#include "aliasing.hpp"
int main() {
    long p, q;
    nsd::Area a{}, b{};
    while (std::scanf("%ld %ld %ld %ld %ld %ld %ld %ld", &p, &a.rows, &a.width, &a.ld, &q, &b.rows,
                      &b.width, &b.ld) == 8) {
        a.p = reinterpret_cast<void *>(p);
        b.p = reinterpret_cast<void *>(q);
        std::printf("%d\n", nsd::areas_meet(a, b));
    }
}
"""


def answers(pairs, tmp_path):
    src, exe = tmp_path / "meet.cpp", tmp_path / "meet"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2303_07030_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True)
    text = "\n".join(" ".join(map(str, (*a, *b))) for a, b in pairs)
    out = subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True).stdout
    return [line == "1" for line in out.split()]


def bytes_of(p, rows, width, ld):
    return {p + i * ld + j for i in range(rows) for j in range(width)}


def test_areas_that_meet(tmp_path):
    rng = random.Random(0)

    def area(ld=None):
        ld = ld or rng.randint(1, 12)
        return rng.randint(100, 160), rng.randint(0, 6), rng.randint(0, ld), ld

    pairs = []
    for i in range(6000):
        a = area()
        pairs.append((a, area(a[3] if i % 2 else None)))
    want = [bool(bytes_of(*a) & bytes_of(*b)) for a, b in pairs]
    assert 1000 < sum(want) < 5000
    assert answers(pairs, tmp_path) == want


def test_areas_of_far_rows(tmp_path):
    """Distances times rows past 64 bits; no array; rows side by side and one apart."""
    far = 2 ** 62
    pairs = [((4096, 9, 8, far), (4096 + 8, 9, 8, far)), ((4096, 9, 8, far), (4096 + 7, 9, 8, far)),
             ((4096, 9, 8, far), (4096 + 100, 1, far - 100, far)),
             ((4096, 9, 8, far), (4096 + 100, 1, far - 99, far)),
             ((0, 9, 8, 8), (0, 9, 8, 8)),
             ((4096, 4, 8, 24), (4104, 4, 16, 24)), ((4096, 4, 8, 24), (4104, 4, 17, 24)),
             ((4096, 4, 8, 24), (4104 + 72, 4, 17, 24)), ((4096, 4, 8, 24), (4104 - 96, 4, 17, 24)),
             ((4096, 4, 8, 24), (4104 - 120, 4, 17, 24))]
    want = [False, True, False, True, False, False, True, False, True, False]
    assert answers(pairs, tmp_path) == want
