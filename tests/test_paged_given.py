"""Which starts and lengths of a paged cache's call are as the interface wants them (CPU only)."""
import random
import subprocess

import pytest

from test_paged_index import compiled

PROGRAM = r"""
#include "paged_index.h"
#include <cstdio>

int main() {
    int start, end, length, T, room, most;
    while (std::scanf("%d %d %d %d %d %d", &start, &end, &length, &T, &room, &most) == 6) {
        const wdc::PagedSeq s = wdc::paged_seq(start, end, length, T, room);
        std::printf("%d %d %d %d\n", wdc::paged_given(start, end, length, T, room, most), s.row0, s.n, s.len);
    }
}
"""


def test_numbers_as_given(tmp_path):
    """In order and within T, the length within the table, no more new tokens than it or than promised; such
    numbers are taken over unchanged."""
    exe = compiled(PROGRAM, tmp_path)
    r = random.Random(7)
    wild = [-2 ** 31, -1, 0, 0, 1, 2, 5, 16, 99, 100, 101, 2 ** 30, 2 ** 31 - 1]
    cases = [[r.choice(wild) for _ in range(3)] + [r.choice([0, 1, 100, 2 ** 31 - 1]), r.choice([16, 100, 2 ** 30]),
                                                   r.choice([0, 1, 5, 100, 2 ** 31 - 1])] for _ in range(20000)]
    run = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True,
                         check=True)
    good = 0
    for (start, end, length, T, room, most), line in zip(cases, run.stdout.splitlines(), strict=True):
        given, row0, n, L = map(int, line.split())
        assert given == (0 <= start <= end <= T and 0 <= length <= room and end - start <= min(length, most))
        if given:
            assert (row0, n, L) == (start, end - start, length)
        good += given
    assert good > 100
