"""The rules of the tensor-core kernels' sources (test_chunk_sources, test_warp_waits) for the
fp4 products, and those of their own (CPU only)."""
import re

import pytest

from test_chunk_sources import test_lanes_are_together_at_tensor_memory as together
from test_warp_waits import _blocks, _code
from test_warp_waits import test_a_wait_that_gives_up_leaves_no_lane_behind as leaves_no_lane_behind

KERNELS = ["gemm_fp4.cu", "gemm_fp4_pair.cu"]


@pytest.mark.parametrize("name", KERNELS)
def test_lanes_are_together(name):
    together(name)


@pytest.mark.parametrize("name", KERNELS)
def test_waits(name):
    leaves_no_lane_behind(name)


def test_lanes_meet_after_finishing_tokens():
    """A lane stores its own column's tokens: all meet again before the next load of tensor memory."""
    code = _code("gemm_fp4.cu")
    loops = [code[a:b] for a, b in _blocks(code, r"\bfor \([^{}]*\) \{") if "finish(c0" in code[a:b] and "load16(" in code[a:b]]
    assert loops and all("__syncwarp();" in x[x.index("finish(c0"):] for x in loops)


def test_parts_are_written_before_they_are_counted():
    """A part's sums, a fence of every lane, the lanes' meeting, then the count; and the last one reads
    behind a fence of its own, past L1."""
    code = _code("gemm_fp4_pair.cu")
    a, b = next((a, b) for a, b in _blocks(code, r"if \(t\.tail >= 0 && rows\) \{"))
    body = code[a:b]
    order = [body.index(x) for x in ("__stcg(", "__threadfence();", "__syncwarp();", "atomicAdd(", "__shfl_sync(")]
    assert order == sorted(order)
    last = body[body.index("if (rows) {"):]
    assert last.index("__threadfence();") < last.index("__ldcg(") and "= 0u" in last


@pytest.mark.parametrize("name", KERNELS)
def test_nothing_is_read_before_the_kernel_before_is_done(name):
    """No load of the caller's memory, by TMA or plain, stands before chain_wait()."""
    code = _code(name)
    for a, b in _blocks(code, r"__global__ void __launch_bounds__[^{]*\{"):
        body = code[a:b]
        assert "chain_wait();" in body
        assert not re.search(r"tma_load|ld_chain|__ldcg|cp_async", body[:body.index("chain_wait();")])


def test_every_part_is_counted():
    """An epilogue warp whose wait gave up still counts its part of a split tile, so that no launch finds parts of
    an earlier one: nothing leaves the job before, and the count does not ask whether the waits were answered."""
    code = _code("gemm_fp4_pair.cu")
    epilogue = code[code.index("setmaxnreg_inc<"):]
    a, b = next((a, b) for a, b in _blocks(epilogue, r"for \(int j = 0; j < jobs && ok; \+\+j\) \{"))
    loop = epilogue[a:b]
    before = loop[:loop.index("atomicAdd(")]
    assert not re.search(r"\b(break|return|continue|goto)\b", before)
    assert [x for x in re.findall(r"if \([^{;]*?\)(?= \{| before)", before[before.index("tfull"):])] == ["if (t.tail >= 0 && rows)", "if (lane == 0)"]
    assert re.search(r"bool rows = m0 < g\.M;", before)
