"""Rules of the chunk operators' kernels that a run on a GPU cannot show to be
kept, read from the sources (CPU only): the compiler happens to keep a warp
together, and a race has hardly ever a way to show."""
import os
import re

import pytest

from test_warp_waits import _blocks, _code
from test_warp_waits import test_a_wait_that_gives_up_leaves_no_lane_behind as leaves_no_lane_behind

KERNELS = ["attn_paged.cu", "gemm_fp8.cu", "gemm_fp8_pair.cu"]
# what may part a warp's lanes, and what brings them together again
PARTS = re.compile(r"\bif \([^\n;]*\b(?:lane|valid|row|threadIdx\.x)\b[^\n;]*\)|\bcontinue;")
JOINS = re.compile(r"__syncwarp\(|_sync\(|\bmbar_wait_warp\(|__syncthreads\(|\bepilogue_barrier\(|\bcluster_sync_all\(")
WHOLE = re.compile(r"\btmem_(?:ld|st)\d+\(")


def parted(code, at):
    """The last place before `at` where lanes may part without meeting again."""
    last = None
    for m in PARTS.finditer(code, 0, at):
        if not JOINS.search(m.group()):
            last = m
    return last.group() if last and not JOINS.search(code, last.end(), at) else None


@pytest.mark.parametrize("name", KERNELS)
def test_lanes_are_together_at_tensor_memory(name):
    """tcgen05.ld and tcgen05.st are instructions of the whole warp (.sync.aligned): between them and
    a branch that some lanes take lies a barrier or vote of the warp, around a loop as well."""
    code = _code(name)
    uses = [m.start() for m in WHOLE.finditer(code)]
    assert uses
    for at in uses:
        assert parted(code, at) is None, code[at - 200:at + 40]
    for a, b in _blocks(code, r"\bfor \([^{}]*\) \{"):
        body = code[a:b]
        if "c0 < COLS" in code[code.rindex("for (", 0, a):a]:  # what a loop over pieces does in its last turn only
            for x, y in reversed(list(_blocks(body, r"\bif \(c0 \+ \w+ == COLS\) \{"))):
                body = body[:x] + body[y - 1:]
        for m in WHOLE.finditer(body):
            assert parted(body + body, len(body) + m.start()) is None, body


@pytest.mark.parametrize("name", KERNELS)
def test_a_wait_that_gives_up_leaves_no_lane_behind(name):
    leaves_no_lane_behind(name)


def test_copies_are_awaited_before_the_next_into_the_same_place():
    """Two cp.async into one place are not ordered.  In the pair kernel a tile's bias and gate are fetched
    only by warps that await them: those that do not leave the tile early."""
    code = _code("gemm_fp8_pair.cu")
    tile = next(code[a:b] for a, b in _blocks(code, r"for \(int tile = pair; tile < tiles && ok; tile \+= pairs\) \{")
                if "cp_async16(" in code[a:b])
    first, wait = tile.index("cp_async16("), tile.index("cp_async_wait()")
    assert first < wait and tile.count("cp_async_wait()") == 1
    leaves = re.findall(r"if \((\S+)\) (?:continue|break);", tile[first:wait])
    assert leaves == ["!ok", "!rows"]                          # (!ok ends the loop)
    head = tile[:first].rindex("if (rows && ")                 # the copies' own condition
    assert tile[head:first].count("{") - tile[head:first].count("}") == 1
