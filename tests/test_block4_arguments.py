"""A block in four bits: what the binding refuses before the library is called, and the
oracle against torch's conversions (CPU only: no context is created)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import block4
from paper_2608_01845_gb300 import wdc
from tests.test_chunk_arguments import BF, F8, I32, cache, ctx, e, test_struct_layout_matches_a_c_compiler as layout  # noqa: F401

F, U8 = torch.float32, torch.uint8


def fp4(M=4, K=64):
    return wdc.Fp4Matrix(e(M, K // 2, dtype=U8), e(-(-M // 128), K // 64, 512, dtype=F8), e(M, dtype=F))


def test_matrix():
    good = (e(4, 32, dtype=U8), e(1, 1, 512, dtype=F8), e(4, dtype=F))
    assert wdc.Fp4Matrix(*good).shape == (4, 64)
    for i, bad in [(0, e(4, 32)), (0, e(4, 16, dtype=U8)), (0, e(4, 0, dtype=U8)), (0, e(32, 4, dtype=U8).t()), (0, e(128, dtype=U8)),
                   (1, e(1, 512, dtype=F8)), (1, e(1, 1, 512, dtype=U8)), (1, e(2, 1, 512, dtype=F8)), (2, e(3, dtype=F)),
                   (2, e(4, 1, dtype=F)), (2, e(4))]:
        with pytest.raises(ValueError):
            wdc.Fp4Matrix(*(bad if i == j else t for j, t in enumerate(good)))
    big = torch.empty(1, 2 ** 31, dtype=U8, device="meta")
    with pytest.raises(ValueError, match="a size of"):
        wdc.Fp4Matrix(big, e(1, 1, 512, dtype=F8), e(1, dtype=F))
    for M, K in [(4, 0), (4, 32), (4, 96), (-1, 64)]:
        with pytest.raises(ValueError):
            wdc.Fp4Matrix.empty(M, K)


def test_quantize_and_products(ctx):
    for x in (e(4, 64, dtype=F), e(4, 128), e(3, 64), e(64, 4).t(), e(4, 128)[:, ::2], e(64)):
        with pytest.raises(ValueError):
            ctx.op_quantize_fp4(x, fp4())
        with pytest.raises(ValueError):
            ctx.op_dequantize_fp4(fp4(), x)
    good = dict(A=fp4(4, 64), W=fp4(8, 64), C=e(4, 8))
    for bad in [dict(A=fp4(4, 128)), dict(W=fp4(16, 64)), dict(C=e(4, 8, dtype=F)), dict(C=e(8, 4).t()), dict(bias=e(8)),
                dict(bias=e(4, dtype=F)), dict(res=e(8, 4)), dict(gate=e(8))]:
        with pytest.raises(ValueError):
            ctx.op_gemm_fp4(**dict(good, **bad))
    good = dict(A=fp4(4, 64), W_gate=fp4(8, 64), W_up=fp4(8, 64), C=e(4, 8))
    for bad in [dict(W_up=fp4(16, 64)), dict(W_up=fp4(8, 128)), dict(W_gate=fp4(16, 64)), dict(C=e(4, 16)),
                dict(gate_bias=e(8)), dict(up_bias=e(16, dtype=F))]:
        with pytest.raises(ValueError):
            ctx.op_gated_fp4(**dict(good, **bad))
    other = fp4()
    other.device = 1
    with pytest.raises(ValueError, match="device"):
        ctx.op_quantize_fp4(e(4, 64), other)


def test_add_norm(ctx):
    good = dict(x=e(4, 64), out=e(4, 64))
    vec = e(64, dtype=F)
    for bad in [dict(x=e(4, 64, dtype=F)), dict(x=e(64)), dict(out=e(4, 128)), dict(out=e(4, 64, dtype=F)), dict(delta=e(3, 64)),
                dict(total=e(4, 64, dtype=F)), dict(weight=e(64)), dict(weight=e(2, 64, dtype=F)), dict(shift=e(32, dtype=F)),
                dict(gate=vec, delta=e(4, 64), rows_per_set=2), dict(weight=e(2, 64, dtype=F), rows_per_set=3, shift=e(3, 64, dtype=F)),
                dict(rows_per_set=-1), dict(rows_per_set=2 ** 32), dict(out=e(4, 64, dtype=F8)),
                dict(out=e(4, 64, dtype=F8), scale=e(4, 1, dtype=F)), dict(scale=e(1, 4, dtype=F)), dict(out=fp4(4, 128)),
                dict(out=fp4(), scale=e(1, 4, dtype=F)), dict(x=e(64, 4).t())]:
        with pytest.raises(ValueError):
            ctx.op_add_norm(**dict(good, **bad))


def test_axes(ctx):
    t = [e(3, 4, 2, dtype=F), e(5, 28, 2, dtype=F)]
    for bad in [([], e(5, 0, dtype=I32)), (t, e(5, 3, dtype=I32)), (t, e(5, 2)), (t, e(2, 5, dtype=I32).t()), (t * 3, e(5, 6, dtype=I32)),
                ([t[0], e(5, 28, dtype=F)], e(5, 2, dtype=I32)), ([t[0], e(5, 28, 2)], e(5, 2, dtype=I32))]:
        with pytest.raises(ValueError):
            wdc.RotAxes(*bad)
    axes = wdc.RotAxes(t, e(5, 2, dtype=I32))
    assert (list(axes.c.rows)[:2], list(axes.c.pairs)[:2], axes.c.axes) == ([3, 5], [4, 28], 2)
    dense = dict(qkv=e(5, 4 * 64), q=e(2, 5, 64), k=e(1, 5, 64), axes=axes)
    app = dict(qkv=e(5, 4 * 64), q=e(5, 2, 64), cache=cache(), q_start=e(2, dtype=I32), axes=axes)
    for bad in [dict(rot=e(5, 32, 2, dtype=F)), dict(positions=e(5, dtype=I32)), dict(axes=wdc.RotAxes(t, e(4, 2, dtype=I32)))]:
        with pytest.raises(ValueError):
            ctx.op_qk_norm_rope(**dict(dense, **bad))
        with pytest.raises(ValueError):
            ctx.op_qk_norm_rope_append(**dict(app, **bad))


@pytest.mark.parametrize("cname,struct", [("wdc_fp4", "Fp4C"), ("wdc_rot_axes", "RotAxesC"), ("wdc_add_norm", "AddNorm")])
def test_struct_layouts(tmp_path, cname, struct):
    layout(tmp_path, cname, struct)


def test_packed_residual_norm():
    """What the binding packs at once lands in the struct's fields."""
    v = list(range(1, 15)) + [0.5, 0.25, 15, 1]
    n = wdc.AddNorm.from_buffer_copy(wdc._ADD_NORM.pack(*v))
    assert wdc._ADD_NORM.size == ctypes.sizeof(n)
    got = [getattr(n, f) if f != "q4" else ctypes.cast(n.q4, ctypes.c_void_p).value for f, _ in n._fields_]
    assert got == v


def test_null_context_is_refused():
    L, N, q = wdc.LIB, None, wdc.Fp4C()
    assert L.wdc_op_quantize_fp4(N, N, 64, q, 1, 64, N) == 1
    assert L.wdc_op_dequantize_fp4(N, q, N, 64, 1, 64, N) == 1
    assert L.wdc_op_gemm_fp4(N, q, q, N, N, 1, 8, 64, 0, N, N, N) == 1
    assert L.wdc_op_gated_fp4(N, q, q, q, N, N, N, 1, 8, 64, 0, N) == 1
    assert L.wdc_op_add_norm(N, wdc.AddNorm(), 1, 64, N) == 1
    n, a, c = wdc.HeadNorm(), wdc.RotAxesC(), wdc.PagedCacheC()
    assert L.wdc_op_qk_norm_rope_axes(N, N, 0, 1, 1, 1, 64, ctypes.byref(n), a, N, N, N, N) == 1
    assert L.wdc_op_qk_norm_rope_append_axes(N, N, 0, 1, 1, ctypes.byref(n), a, c, N, N, N) == 1


def test_oracle_rounds_to_the_format():
    """Every value between two levels goes to the nearer one, a tie to the even code."""
    levels = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    x = np.concatenate([np.linspace(-8, 8, 30001), np.exp2(np.linspace(-20, 4, 999))])
    d = np.abs(np.minimum(np.abs(x), 6)[:, None] - levels)
    got = np.abs(block4.e2m1_round(x))
    assert (np.abs(got - np.minimum(np.abs(x), 6)) <= d.min(1)).all() and np.isin(got, levels).all()
    ties = {0.25: 0, 0.75: 1, 1.25: 1, 1.75: 2, 2.5: 2, 3.5: 4, 5: 4}
    assert [block4.e2m1_round(t) for t in ties] == list(ties.values())
    assert np.float32(1 / 2688) == block4.ROW


def test_oracle_layouts():
    r = np.random.default_rng(0)
    code = r.choice([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -6, -3], (5, 128))
    assert np.array_equal(block4.unpack(block4.pack(code)), code)
    s = r.random((300, 8))
    p = block4.to_pieces(s, 7.0)
    assert p.shape == (3, 2, 512) and np.array_equal(block4.from_pieces(p, 300), s) and (p == 7.0).sum() == (384 - 300) * 8
    assert p[1, 1, 3 * 16 + 2 * 4 + 1] == s[128 + 64 + 3, 5]


def test_oracle_quantizes_a_row():
    """A row by hand: maximum 12 at a scale of 12 / 2688, a block of it exactly 448 steps of 6."""
    x = np.zeros((2, 64), np.float32)
    x[0, :16] = np.arange(16) * 0.8
    x[0, 16:32] = 1e-9
    code, s, row = block4.quantize(x)
    assert row[0] == np.float32(12) * block4.ROW and row[1] == 0 and (s[1] == 0).all()
    assert s[0, 0] == 448 and (s[0, 1:] == 0).all() and code[0, 15] == 6 and (code[0, 16:] == 0).all()
    assert abs(block4.values(code, s, row)[0, 15] - 12) < 1e-5
