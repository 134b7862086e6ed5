"""The paged cache's index arithmetic against its definition and with values that
no caller should give: rows, places and pages stay within their arrays (CPU only)."""
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

from oracle import chunk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_01845_gb300", "csrc")

MIDDLE = r"""
#include "paged_index.h"
#include <cstdio>

int main() {
    float lo, hi;
    while (std::scanf("%f %f", &lo, &hi) == 2) std::printf("%.0f\n", wdc::plan_middle(lo, hi));
}
"""

PROGRAM = r"""
#include "paged_index.h"
#include <cstdio>

int main() {
    int start, end, length, T, room, frame, page, pages;
    while (std::scanf("%d %d %d %d %d %d %d %d", &start, &end, &length, &T, &room, &frame, &page, &pages) == 8) {
        const wdc::PagedSeq s = wdc::paged_seq(start, end, length, T, room);
        std::printf("%d %d %d %d", s.row0, s.n, s.len, wdc::paged_page(page, pages));
        const int rows[4] = {0, s.n / 2, s.n - 1, s.n > 2 ? s.n - 2 : 0};
        for (int i : rows) std::printf(" %d %d", wdc::paged_place(s, i), wdc::paged_limit(s, frame, i));
        std::printf("\n");
    }
}
"""


def compiled(source, d):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = d / "paged.cpp", d / "paged"
    src.write_text(source)
    subprocess.run([cxx, "-std=c++17", "-O1", "-ftrapv", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    return exe


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = compiled(PROGRAM, tmp_path_factory.mktemp("paged"))

    def run(cases):
        r = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True,
                           check=True)
        return [[int(x) for x in line.split()] for line in r.stdout.splitlines()]
    return run


def test_places_and_limits_follow_the_definition(program):
    cases = []
    for n, L, frame in [(1, 1, 1), (1, 7, 1), (5, 5, 1), (5, 12, 0), (5, 12, 4), (7, 20, 20), (3, 20, 1000), (6, 4, 1),
                        (6, 4, 3), (2, 0, 1), (2, 0, 0), (1, 2 ** 30, 2 ** 30), (4, 2 ** 30, 7)]:
        cases.append((10, 10 + n, L, 100, 2 ** 30, frame, 0, 1))
    for c, got in zip(cases, program(cases)):
        n, L, frame = c[1] - c[0], c[2], c[5]
        assert got[:4] == [10, n, L, 0]
        want = chunk.limits(n, L, frame)
        for j, i in enumerate([0, n // 2, n - 1, n - 2 if n > 2 else 0]):
            assert got[4 + 2 * j] == L - n + i
            assert got[5 + 2 * j] == want[i]


def test_bad_values_stay_within_the_arrays(program):
    r = random.Random(3)
    wild = [-2 ** 31, -2 ** 31 + 1, -1, 0, 1, 5, 99, 100, 101, 2 ** 30, 2 ** 31 - 1]
    cases = [(r.choice(wild), r.choice(wild), r.choice(wild), r.choice([0, 1, 100, 2 ** 31 - 1]), r.choice([16, 100, 2 ** 30]),
              r.choice([0, 1, 3, 2 ** 31 - 1]), r.choice(wild), r.choice([1, 7, 2 ** 31 - 1])) for _ in range(4000)]
    for (start, end, length, T, room, frame, page, pages), got in zip(cases, program(cases)):
        row0, n, L, p = got[:4]
        assert 0 <= row0 and 0 <= n and row0 + n <= T and 0 <= L <= room
        assert p == (page if 0 <= page < pages else -1)
        if n:
            for place, lim in np.array(got[4:]).reshape(-1, 2):
                assert place < L and 0 <= lim <= L


def test_middle_of_a_bisection_up_to_the_longest_sequence(tmp_path):
    exe = compiled(MIDDLE, tmp_path)
    top = 2 ** 24                      # steps of 64 keys of 2^30
    cases = [(lo, hi) for hi in (1, 2, 9, 2 ** 23, 2 ** 23 + 2, top - 1, top) for lo in (0, 1, hi - 3, hi - 2, hi - 1, hi) if 0 <= lo <= hi]
    r = subprocess.run([str(exe)], input="\n".join(f"{lo} {hi}" for lo, hi in cases), capture_output=True, text=True, check=True)
    assert [int(x) for x in r.stdout.split()] == [(lo + hi) // 2 for lo, hi in cases]
