"""A block in four bits against fp64: e2m1 rows and back, the product of such matrices
and the gated one, the residual's norm, rotation by several axes, and all of them
together, at the sizes and values where they can go wrong."""
import ctypes
import functools

import numpy as np
import pytest
import torch

from oracle import block4, chunk, dit
from paper_2608_01845_gb300 import synth, wdc
from tests.test_gpu_chunk import DTYPES, HALF, MODEL, Paged, dev, host, norm_bound, rotations, rows_of, starts

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def contexts():
    return {k: wdc.Context(wdc.make_config(dtype=wdc.F32 if k == "f32" else wdc.BF16, **MODEL), 2) for k in DTYPES}


def matrix(code, s, row, fill=np.nan):
    """An Fp4Matrix of these values; `fill`: what rows behind the last hold in the scales."""
    return wdc.Fp4Matrix(torch.from_numpy(block4.pack(code)).cuda(), dev(block4.to_pieces(s, fill), F8), dev(row))


# ---------------------------------------------------------------- rows
def check_rows(q, x):
    """Bit for bit: every intermediate is a single IEEE operation."""
    code, s, row = block4.quantize(x)
    assert np.array_equal(q.row_scale.cpu().numpy(), row, equal_nan=True)
    assert np.array_equal(host(q.scale), block4.to_pieces(s))
    assert np.array_equal(block4.unpack(q.codes.cpu().numpy()), code)
    return block4.values(code, s, row)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 64), (3, 128), (33, 192), (128, 256), (127, 320), (129, 1024), (65, 1088), (130, 2112),
                                 (300, 5120), (2, 16384), (3, 16448), (130, 20544)])
def test_quantize_and_back(contexts, M, K, kind):
    ctx = contexts[kind]
    x = rows_of(11, M, K, kind)
    q = wdc.Fp4Matrix.empty(M, K)
    guard = torch.full((M + 1, K), 3.0, dtype=DTYPES[kind], device="cuda")
    ctx.op_quantize_fp4(dev(x, DTYPES[kind]), q)
    want = check_rows(q, x)
    ctx.op_dequantize_fp4(q, guard[:M])
    # a scale's product and its own are rounded to fp32, the value to its type
    assert (np.abs(host(guard[:M]) - want) <= (HALF[kind] + 2.0 ** -22) * np.abs(want)).all()
    assert bool((guard[M:] == 3.0).all())


def test_quantize_rows_that_lie_apart(contexts):
    x = rows_of(12, 40, 400, "bf16")
    t, q = dev(x, torch.bfloat16), wdc.Fp4Matrix.empty(40, 192)
    contexts["bf16"].op_quantize_fp4(t[:, 80:272], q)
    want = check_rows(q, x[:, 80:272])
    contexts["bf16"].op_dequantize_fp4(q, t[:, 80:272])
    assert (np.abs(host(t[:, 80:272]) - want) <= (2.0 ** -8 + 2.0 ** -22) * np.abs(want)).all()
    assert np.array_equal(host(t[:, :80]), x[:, :80]) and np.array_equal(host(t[:, 272:]), x[:, 272:])


@pytest.mark.parametrize("K", [256, 20544])
def test_quantize_values_of_every_size(contexts, K):
    """Rows from subnormal to the largest, values of every size below them, zeros, infinities and NaN."""
    g = np.random.default_rng(5)
    top = np.exp2(np.concatenate([np.arange(-149, 128), [-100, -100, -101]]).astype(np.float64))
    with np.errstate(over="ignore", under="ignore"):
        x = top[:, None] * (1 + g.random((len(top), K))) * np.exp2(-g.integers(0, 24, (len(top), K))) * g.choice([-1, 1], (len(top), K))
    x = np.clip(x, -3e38, 3e38).astype(np.float32)
    x[3], x[40, 7], x[50, K - 1], x[60, 64:128] = 0, np.inf, np.nan, -np.inf
    x[200, :32] = -0.0
    q, back = wdc.Fp4Matrix.empty(len(x), K), torch.empty(len(x), K, device="cuda")
    contexts["f32"].op_quantize_fp4(dev(x), q)
    check_rows(q, x)
    contexts["f32"].op_dequantize_fp4(q, back)
    b = host(back)
    bad = [40, 50, 60]
    assert np.isnan(b[bad]).all() and np.isfinite(np.delete(b, bad, 0)).all() and (b[3] == 0).all()


# ---------------------------------------------------------------- products
def rows4(seed, M, K, std=1.0):
    return block4.quantize(rows_of(seed, M, K, "bf16") * np.float32(std))


def product_case(seed, M, N, K):
    A, W = rows4(seed, M, K), block4.quantize(synth.bf16_round(synth.normal(seed + 5, (N, K), K ** -0.5)))
    a, w = block4.values(*A), block4.values(*W)
    return A, W, a @ w.T, np.abs(a) @ np.abs(w).T


def product_bound(y, mag, K):
    """An instruction's 64 products and the sums of the instructions lose at most 2^-23
    of the terms' magnitudes an addition (a truncated fp32 sum), split sums a few more;
    two products with the rows' scales, one rounding each."""
    return (64 + K / 64 + 8) * 2.0 ** -23 * mag + 2.0 ** -22 * np.abs(y)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 5, 16, 17, 33, 64, 65, 100, 128, 129, 257, 300])
@pytest.mark.parametrize("N,K", [(8, 64), (136, 192), (256, 1024), (1032, 2112)])
def test_gemm(contexts, M, N, K, kind):
    ctx = contexts[kind]
    A, W, y, mag = product_case(21, M, N, K)
    buf = torch.full((M + 2, N), 7.0, dtype=DTYPES[kind], device="cuda")
    ctx.op_gemm_fp4(matrix(*A), matrix(*W), buf[:M])
    assert ctx.device_errors() == 0
    assert (np.abs(host(buf[:M]) - y) <= product_bound(y, mag, K) + HALF[kind] * np.abs(y)).all()
    assert bool((buf[M:] == 7.0).all())


SHAPES = [(3, 264, 576), (40, 392, 8256), (100, 1544, 4160), (520, 2312, 2112), (1030, 2056, 1088), (2309, 3080, 576),
          (700, 12296, 320), (300, 1032, 16448)]


@functools.lru_cache(1)
def epilogue_case(M, N, K):
    A, W, y, mag = product_case(31, M, N, K)
    return A, W, matrix(*A), matrix(*W), y, mag


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["bias", "gelu", "resid", "resid_gelu", "gateless"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_epilogues(contexts, M, N, K, mode, kind):
    """The epilogue's own error: 1.13 (GELU's steepest slope) of the sum's, 2^-18 of
    GELU's value for its exponential and quotient, the gate's multiple of both."""
    ctx = contexts[kind]
    _, _, da, dw, y, mag = epilogue_case(M, N, K)
    b, g = synth.normal(3, (N,), 0.5), synth.normal(5, (N,))
    r = synth.bf16_round(synth.normal(4, (M, N)))
    err = product_bound(y, mag, K)
    y = y + b
    err = err + 2.0 ** -22 * np.abs(y)
    kw = dict(bias=dev(b))
    if "gelu" in mode:
        y, err, kw["gelu"] = dit.gelu_tanh(y), 1.13 * err + 2.0 ** -18 * np.abs(y) + 1e-6, True
    C = torch.empty(M, N, dtype=DTYPES[kind], device="cuda")
    if mode not in ("bias", "gelu"):
        C.copy_(dev(r))
        kw["res"] = C                                      # in place
        if mode != "gateless":
            y, err, kw["gate"] = g * y, np.abs(g) * err + 2.0 ** -22 * np.abs(g * y), dev(g)
        y = r + y
    ctx.op_gemm_fp4(da, dw, C, **kw)
    assert ctx.device_errors() == 0
    assert (np.abs(host(C) - y) <= err + HALF[kind] * np.abs(y) + 2.0 ** -22 * np.abs(y)).all()


GATED = [(1, 8, 64), (5, 136, 192), (17, 256, 4160), (64, 1032, 1024), (100, 264, 2112), (129, 520, 576)] + SHAPES


@functools.lru_cache(1)
def gated_case(M, N, K):
    A, W, da, dw, g, gmag = epilogue_case(M, N, K)
    U = block4.quantize(synth.bf16_round(synth.normal(77, (N, K), K ** -0.5)))
    a, u = block4.values(*A), block4.values(*U)
    return da, dw, matrix(*U), g, gmag, a @ u.T, np.abs(a) @ np.abs(u).T


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,N,K", GATED)
def test_gated(contexts, M, N, K, gelu, bias, kind):
    """f's slope is at most 1.13, its own error 2^-18 of its value; the product adds each factor's."""
    ctx = contexts[kind]
    da, dw, du, g, gmag, u, umag = gated_case(M, N, K)
    ge, ue = product_bound(g, gmag, K), product_bound(u, umag, K)
    kw = dict(gelu=gelu)
    if bias:
        bg, bu = synth.normal(3, (N,), 0.5), synth.normal(5, (N,), 0.5)
        g, u, kw = g + bg, u + bu, dict(kw, gate_bias=dev(bg), up_bias=dev(bu))
        ge, ue = ge + 2.0 ** -22 * np.abs(g), ue + 2.0 ** -22 * np.abs(u)
    f = dit.gelu_tanh(g) if gelu else block4.silu(g)
    fe = 1.13 * ge + 2.0 ** -18 * np.abs(f) + 1e-6
    want = f * u
    buf = torch.full((M + 1, N), 7.0, dtype=DTYPES[kind], device="cuda")
    ctx.op_gated_fp4(da, dw, du, buf[:M], **kw)
    assert ctx.device_errors() == 0
    err = fe * np.abs(u) + np.abs(f) * ue + fe * ue + 2.0 ** -22 * np.abs(want) + HALF[kind] * np.abs(want)
    assert (np.abs(host(buf[:M]) - want) <= err).all()
    assert bool((buf[M:] == 7.0).all())


def activation_arguments(n):
    """From far below where the exponentials end to far above, closer around 0 and at the borders."""
    x = np.concatenate([np.linspace(-60, 12, n - 2048), -np.geomspace(1e-6, 1e30, 1024), np.geomspace(1e-6, 1e30, 992), [0.0, -0.0],
                        np.linspace(-7.1, -6.9, 15), np.linspace(-42, -41, 15)])
    return x.astype(np.float32)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("op", ["gemm_fp8", "gemm_fp4", "gated_gelu", "gated_silu"])
@pytest.mark.parametrize("M", [2, 2048])                   # (few rows, CTA pairs)
def test_activations_over_their_whole_range(contexts, M, op, kind):
    """The bias alone is the argument x, f(x) = x / (1 + 2^u).  u is off by 2^-21 of itself for GELU (three
    roundings of its cubic term, the sum's, the constants' three and the product's: 8 of 2^-24) and by 2^-23 for
    SiLU, so 2^u by |u| ln 2 times that, with |u| at most 60 before f is below 2^-54: 2^-15.6 and 2^-17.6; above
    -5/2 |u| is below 7.4: 2^-18.6.  The exponential's 2^-22, the sum, quotient and products add 2^-20.5.
    (The kernel for few rows has an exponential of 2 + 1.17 |x| ulp for SiLU: 2^-17.4 at -41.)"""
    ctx, N = contexts[kind], 8192
    x = activation_arguments(N)
    zero = lambda rows, k: torch.zeros(rows, k, dtype=torch.uint8, device="cuda")
    C = torch.full((M, N), 7.0, dtype=DTYPES[kind], device="cuda")
    if op == "gemm_fp8":
        one = torch.ones
        ctx.op_gemm_fp8(zero(M, 128).view(F8), one(1, M, device="cuda"), zero(N, 128).view(F8), one(N // 128, 1, device="cuda"), C,
                        bias=dev(x), gelu=True)
    else:
        m = lambda rows: wdc.Fp4Matrix(zero(rows, 32), zero(-(-rows // 128), 512).view(-1, 1, 512).view(F8), torch.ones(rows, device="cuda"))
        if op == "gemm_fp4":
            ctx.op_gemm_fp4(m(M), m(N), C, bias=dev(x), gelu=True)
        else:
            ctx.op_gated_fp4(m(M), m(N), m(N), C, gate_bias=dev(x), up_bias=dev(np.ones(N)), gelu=op == "gated_gelu")
    xd = x.astype(np.float64)
    with np.errstate(over="ignore"):
        f = xd / (1 + np.exp(-xd if op == "gated_silu" else -2 * np.sqrt(2 / np.pi) * (xd + 0.044715 * xd ** 3)))
    bound = np.where(xd > -2.5, 2.0 ** -18, 2.0 ** -17 if op == "gated_silu" else 2.0 ** -15) + HALF[kind]
    bound = np.where(np.abs(f) < 2.0 ** -54, 1.01, bound)
    got = host(C)
    assert (got == got[:1]).all() and (np.abs(got[0] - f) <= bound * np.abs(f)).all() and ctx.device_errors() == 0


@pytest.mark.parametrize("M,N,K", [(9, 264, 1088), (150, 520, 320), (900, 4104, 576)])
def test_products_of_any_scales(contexts, M, N, K):
    """Scales are any e4m3 numbers, the rows' any fp32 ones of either sign; codes are all sixteen."""
    g = np.random.default_rng(7)
    levels = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    e4m3 = np.concatenate([np.arange(8) / 512.0] + [(8 + np.arange(8)) * 2.0 ** (e - 9) for e in range(14)] +
                          [(8 + np.arange(7)) * 32.0])             # (there is no 15 * 32: that code is NaN)
    code = lambda n: g.choice(np.concatenate([levels, -levels]), (n, K))
    A = (code(M), g.choice(e4m3, (M, K // 16)), (g.standard_normal(M) * np.exp2(g.integers(-20, 20, M))).astype(np.float32))
    W = (code(N), g.choice(e4m3, (N, K // 16)), g.standard_normal(N).astype(np.float32))
    a, w = block4.values(*A), block4.values(*W)
    C = torch.empty(M, N, device="cuda")
    contexts["f32"].op_gemm_fp4(matrix(*A), matrix(*W), C)
    y, mag = a @ w.T, np.abs(a) @ np.abs(w).T
    assert (np.abs(host(C) - y) <= product_bound(y, mag, K) + 2.0 ** -24 * np.abs(y)).all()


@pytest.mark.parametrize("M", [40, 300])
def test_nonfinite_rows_stay_in_their_rows(contexts, M):
    """A NaN scale, a NaN or infinite row scale: its row of A or its column, nothing else."""
    A, W, y, _ = product_case(43, M, 136, 256)
    a = [np.array(t, copy=True) for t in A]
    w = [np.array(t, copy=True) for t in W]
    a[1][5, 3], a[2][9], a[2][11], w[2][20], w[1][33, 2] = np.nan, np.inf, np.nan, np.nan, np.nan
    C = torch.empty(M, 136, device="cuda")
    contexts["f32"].op_gemm_fp4(matrix(*a), matrix(*w), C)
    got = host(C)
    assert np.isnan(got[[5, 11]]).all() and np.isnan(got[:, [20, 33]]).all() and not np.isfinite(got[9]).any()
    rest = np.delete(np.delete(got, [5, 9, 11], 0), [20, 33], 1)
    assert np.isfinite(rest).all() and np.allclose(rest, np.delete(np.delete(y, [5, 9, 11], 0), [20, 33], 1), rtol=1e-4, atol=1e-4)


# (16, 32, 64 and 128 tokens a tile, alone and with K over 2, 4 and 8 CTAs, one of which ends short)
FEW = [(1, 8, 4160), (3, 2056, 4160), (2, 8200, 8256), (17, 8, 64), (17, 8200, 8256), (20, 2056, 4160), (33, 8, 4160), (50, 2056, 4160),
       (60, 8200, 8256), (65, 8, 4160), (90, 2056, 8256), (65, 8200, 16448), (130, 264, 4160),
       (65, 8, 8256)]


@functools.lru_cache(1)
def few_case(M, N, K):
    A, W, y, mag = product_case(61, M, N, K)
    return matrix(*A), matrix(*W), y, mag


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", FEW)                     # (the slowest of the three to vary)
def test_every_way_for_few_rows(contexts, M, N, K, gated, kind):
    ctx = contexts[kind]
    a, w, y, mag = few_case(M, N, K)
    e = product_bound(y, mag, K)
    buf = torch.full((M + 1, N), 7.0, dtype=DTYPES[kind], device="cuda")
    if gated:
        ctx.op_gated_fp4(a, w, w, buf[:M])
        f = block4.silu(y)
        y, e = f * y, (1.13 * e + 2.0 ** -18 * np.abs(f) + 1e-6) * np.abs(y) + np.abs(f) * e + 3 * e * e + 2.0 ** -22 * np.abs(f * y)
    else:
        r = synth.bf16_round(synth.normal(4, (M, N)))
        buf[:M] = dev(r)
        ctx.op_gemm_fp4(a, w, buf[:M], res=buf[:M])
        y, e = r + y, e + 2.0 ** -22 * np.abs(r)
    assert ctx.device_errors() == 0
    assert (np.abs(host(buf[:M]) - y) <= e + HALF[kind] * np.abs(y)).all()
    assert bool((buf[M:] == 7.0).all())


SPLIT = (1300, 3592, 8256)      # 90 tiles of 256 x 256 on 76 pairs: 14 are split over K


@functools.lru_cache(1)
def split_case():
    return product_case(51, *SPLIT)


def test_split_sums_repeat_themselves(contexts):
    """Parts of K are added in their order whichever comes last: the same bits every time, on any stream."""
    A, W, y, mag = split_case()
    a, w, outs = matrix(*A), matrix(*W), []
    for i in range(6):
        C = torch.empty(*SPLIT[:2], device="cuda")
        contexts["f32"].op_gemm_fp4(a, w, C)
        outs.append(C)
    assert (np.abs(host(outs[0]) - y) <= product_bound(y, mag, SPLIT[2]) + 2.0 ** -24 * np.abs(y)).all()
    assert all(torch.equal(outs[0], c) for c in outs[1:]) and contexts["f32"].device_errors() == 0


def planned(ctx, want, M, N, K, gated=False):
    """A test for a kernel's path has reached it (the choices are those for 152 SMs)."""
    if torch.cuda.get_device_properties(0).multi_processor_count == 152:
        got = ctx.fp4_plan(M, N, K, gated)
        assert all(w is None or w == g for w, g in zip(want, got)), got


class Drawn:
    """Rows drawn from 48 different ones, each with a scale of its own: long products that fp64 is quick to give."""

    def __init__(self, seed, rows, K, std=1.0):
        r = np.random.default_rng(seed)
        code, s, row = block4.quantize(synth.bf16_round(synth.normal(seed, (48, K), std)))
        self.pick = r.integers(0, 48, rows)
        self.row = (row[self.pick] * (0.5 + r.random(rows))).astype(np.float32)
        self.base = code * np.asarray(s, np.float64).repeat(16, 1)
        self.m = wdc.Fp4Matrix(torch.from_numpy(block4.pack(code)).cuda()[torch.from_numpy(self.pick).cuda()].contiguous(),
                               dev(block4.to_pieces(s[self.pick], np.nan), F8), dev(self.row))

    def product(self, w):
        """(A W^T, of the magnitudes)"""
        scales = self.row[:, None].astype(np.float64) * w.row[None]
        return [(f(self.base) @ f(w.base).T)[self.pick][:, w.pick] * scales for f in (np.asarray, np.abs)]


@functools.lru_cache(3)
def drawn_case(M, N, K, gated):
    A, W = Drawn(31, M, K), Drawn(32, N, K, K ** -0.5)
    U = Drawn(33, N, K, K ** -0.5) if gated else None
    return A, W, U, A.product(W), A.product(U) if gated else None


# (a round of 76 tiles and some behind it that are split over K in so many parts; M, N and K ragged)
SPLITS = [(1300, 3592, 8256, 14, 3), (1250, 3976, 8256, 4, 3), (1282, 4616, 16448, 38, 2)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["store", "bias", "gelu", "resid", "resid_gelu", "gateless"])
@pytest.mark.parametrize("M,N,K,tail,parts", SPLITS)
def test_split_epilogues(contexts, M, N, K, tail, parts, mode, kind):
    """test_gemm_epilogues where the last tiles' sums are joined from parts, the residual in place fetched behind that."""
    ctx = contexts[kind]
    planned(ctx, (256, 0, tail, parts), M, N, K)
    A, W, _, (y, mag), _ = drawn_case(M, N, K, False)
    b, g = synth.normal(3, (N,), 0.5), synth.normal(5, (N,))
    r = synth.bf16_round(synth.normal(4, (M, N)))
    err, kw = product_bound(y, mag, K), {}
    if mode != "store":
        y, kw = y + b, dict(bias=dev(b))
        err = err + 2.0 ** -22 * np.abs(y)
    if "gelu" in mode:
        y, err, kw["gelu"] = dit.gelu_tanh(y), 1.13 * err + 2.0 ** -18 * np.abs(y) + 1e-6, True
    buf = torch.full((M + 1, N), 7.0, dtype=DTYPES[kind], device="cuda")
    C = buf[:M]
    if mode in ("resid", "resid_gelu", "gateless"):
        C.copy_(dev(r))
        kw["res"] = C
        if mode != "gateless":
            y, err, kw["gate"] = g * y, np.abs(g) * err + 2.0 ** -22 * np.abs(g * y), dev(g)
        y = r + y
    ctx.op_gemm_fp4(A.m, W.m, C, **kw)
    assert (np.abs(host(C) - y) <= err + HALF[kind] * np.abs(y) + 2.0 ** -22 * np.abs(y)).all()
    assert bool((buf[M:] == 7.0).all()) and ctx.device_errors() == 0


GATED_SPLITS = [(1100, 2184, 8256, 14, 3), (1282, 2312, 16448, 38, 2), (1250, 1992, 16448, 4, 8)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,N,K,tail,parts", GATED_SPLITS)
def test_split_gated(contexts, M, N, K, tail, parts, bias, gelu, kind):
    """test_gated where both sums of the last tiles are joined from parts."""
    ctx = contexts[kind]
    planned(ctx, (256, 0, tail, parts), M, N, K, True)
    A, W, U, (g, gmag), (u, umag) = drawn_case(M, N, K, True)
    ge, ue, kw = product_bound(g, gmag, K), product_bound(u, umag, K), dict(gelu=gelu)
    if bias:
        bg, bu = synth.normal(3, (N,), 0.5), synth.normal(5, (N,), 0.5)
        g, u, kw = g + bg, u + bu, dict(kw, gate_bias=dev(bg), up_bias=dev(bu))
        ge, ue = ge + 2.0 ** -22 * np.abs(g), ue + 2.0 ** -22 * np.abs(u)
    want, f = block4.gated(g, u, gelu), block4.gated(g, 1.0, gelu)
    fe = 1.13 * ge + 2.0 ** -18 * np.abs(f) + 1e-6
    buf = torch.full((M + 1, N), 7.0, dtype=DTYPES[kind], device="cuda")
    ctx.op_gated_fp4(A.m, W.m, U.m, buf[:M], **kw)
    err = fe * np.abs(u) + np.abs(f) * ue + fe * ue + 2.0 ** -22 * np.abs(want) + HALF[kind] * np.abs(want)
    assert (np.abs(host(buf[:M]) - want) <= err).all()
    assert bool((buf[M:] == 7.0).all()) and ctx.device_errors() == 0


@pytest.mark.parametrize("M,N,K,gated,want", [
    (3, 264, 576, False, (16, 1)), (3, 2056, 4160, False, (16, 4)), (2, 8200, 8256, False, (16, 2)), (1, 8, 4160, False, (32, 8)),
    (17, 8, 64, False, (32, 1)), (17, 8200, 8256, False, (32, 2)), (20, 2056, 4160, False, (32, 4)), (33, 8, 4160, False, (64, 8)),
    (50, 2056, 4160, False, (64, 4)), (60, 8200, 8256, False, (64, 2)), (100, 1544, 4160, False, (128, 1)),
    (65, 8200, 16448, False, (128, 2)), (90, 2056, 8256, False, (128, 4)), (65, 8, 8256, False, (128, 8)),
    (40, 392, 8256, True, (64, 8)), (100, 1544, 4160, True, (128, 8)), (300, 1032, 16448, True, (128, 4)), (17, 8, 64, True, (32, 1)),
    (1030, 2056, 1088, False, (256, 0, 0, 0)), (2309, 3080, 576, True, (256, 0, 0, 0)), (*SPLIT, False, (256, 0, 14, 3))])
def test_the_shapes_above_take_every_way(contexts, M, N, K, gated, want):
    """Tokens a tile and CTAs a tile's K, the pairs and their split tiles: what the tests of the products reach."""
    for ctx in contexts.values():
        planned(ctx, want, M, N, K, gated)


def test_plans_of_no_products(contexts):
    for bad in [(0, 8, 64), (4, 0, 64), (4, 8, 0), (4, 4, 64), (4, 8, 32), (4, 8, 2 ** 31 - 64), (-1, 8, 64)]:
        with pytest.raises((wdc.WdcError, ValueError)):
            contexts["bf16"].fp4_plan(*bad)


# ---------------------------------------------------------------- residual and norm
def norm_case(M, D, kind, add, per, seed=91):
    sets = -(-M // per) if per else 1
    f = lambda a: synth.bf16_round(a) if kind == "bf16" else a.astype(np.float32)
    x = f(rows_of(seed, M, D, kind) + (np.arange(M) % 3 - 1)[:, None].astype(np.float32))
    kw = dict(weight=synth.normal(92, (sets, D), 0.3), shift=synth.normal(93, (sets, D), 0.3))
    if add:
        kw.update(delta=f(synth.normal(94, (M, D), 2.0)), gate=synth.normal(95, (sets, D)))
    return x, kw


def norm_errors(x, kw, offset, center, eps, per):
    """(r, y, error of y): a thread sums at most 32 terms and 9 steps join them, so the mean of
    squares is off by 41 2^-24 of itself and its root by half that; with the root's and
    the products' own 2^-21, 2^-19 of the normalised value.  A layer norm's mean is off by
    (41 + 2) 2^-24 of the mean magnitude, the sum r by 2^-24 of its terms, both multiplied by
    1 / std and the weight."""
    r, y = block4.add_norm(x, kw.get("delta"), kw.get("gate"), kw.get("weight"), offset, kw.get("shift"), center, eps, per)
    pick = lambda v: np.asarray(v, np.float64)[np.arange(len(x)) // per if per else np.zeros(len(x), int)]
    terms = np.abs(x).astype(np.float64)
    if "delta" in kw:
        terms = terms + np.abs((pick(kw["gate"]) if "gate" in kw else 1.0) * kw["delta"])
    c = r - r.mean(1, keepdims=True) if center else r
    inv = 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    w = np.abs(pick(kw["weight"]) + offset) if "weight" in kw else 1.0
    slip = 2.0 ** -23 * terms + (2.0 ** -23 * np.abs(r) + 45 * 2.0 ** -24 * terms.mean(1, keepdims=True) if center else 0)
    # an error of the values moves the mean of squares too, by at most twice its relative size
    err = w * inv * (slip + np.abs(c) * 2 * np.sqrt((slip ** 2).mean(1, keepdims=True)) * inv) + 2.0 ** -19 * w * np.abs(c) * inv
    return r, terms, y, err + 2.0 ** -22 * (np.abs(y) + (np.abs(pick(kw["shift"])) if "shift" in kw else 0))


def to_device(kw, dt):
    return {k: dev(v, dt if k == "delta" else torch.float32) for k, v in kw.items()}


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("D", [16, 64, 80, 256, 272, 1024, 1040, 2064, 5120, 8208, 16384])
@pytest.mark.parametrize("M,add,per", [(1, True, 0), (7, False, 3), (130, True, 50)])
def test_add_norm(contexts, M, D, add, per, center, kind):
    ctx, dt = contexts[kind], DTYPES[kind]
    x, kw = norm_case(M, D, kind, add, per)
    r, terms, y, err = norm_errors(x, kw, 1.0, center, 1e-5, per)
    wide = torch.full((M + 1, D + 8), 3.0, dtype=dt, device="cuda")
    total = torch.full((M + 1, D + 16), 4.0, dtype=dt, device="cuda")
    xw = torch.full((M, D + 24), 9.0, dtype=dt, device="cuda")                 # rows lie apart
    xw[:, :D] = dev(x, dt)
    args = dict(to_device(kw, dt), weight_offset=1.0, center=center, eps=1e-5, rows_per_set=per)
    ctx.op_add_norm(xw[:, :D], wide[:M, :D], total=total[:M, :D], **args)
    assert (np.abs(host(wide[:M, :D]) - y) <= err + HALF[kind] * np.abs(y)).all()
    assert (np.abs(host(total[:M, :D]) - r) <= 2.0 ** -23 * terms + HALF[kind] * np.abs(r)).all()
    assert bool((wide[M:] == 3.0).all()) and bool((wide[:, D:] == 3.0).all())
    assert bool((total[M:] == 4.0).all()) and bool((total[:, D:] == 4.0).all())

    kb = -(-D // 128)
    q, s = torch.full((M + 1, D), 3.0, device="cuda").to(F8), torch.full((kb * M + 4,), 7.0, device="cuda")
    ctx.op_add_norm(xw[:, :D], q[:M], scale=s[:kb * M].view(kb, M), **args)
    top = np.stack([np.abs(y[:, 128 * j:128 * j + 128]).max(1) for j in range(kb)])
    most = np.stack([err[:, 128 * j:128 * j + 128].max(1) for j in range(kb)])
    got = host(s[:kb * M].view(kb, M))
    assert (np.abs(got * 448 - top) <= most + 2.0 ** -22 * top).all()
    step = got.T.repeat(128, 1)[:, :D]
    # half a step of e4m3: 2^-4 of the value, 2^-10 of the scale below its normal numbers
    assert (np.abs(host(q[:M]) * step - y) <= err + 2.0 ** -20 * np.abs(y) + np.maximum(2.0 ** -4 * (np.abs(y) + err), 2.0 ** -10 * step)).all()
    assert bool((q[M:].float() == 3.0).all()) and bool((s[kb * M:] == 7.0).all())

    if D % 64 == 0:
        m = wdc.Fp4Matrix.empty(M, D)
        m.scale.fill_(1.0)
        ctx.op_add_norm(xw[:, :D], m, **args)
        row, sc = host(m.row_scale), block4.from_pieces(host(m.scale), M)
        assert (np.abs(row * 2688 - np.abs(y).max(1)) <= err.max(1) + 2.0 ** -21 * np.abs(y).max(1)).all()
        pieces = host(m.scale)
        pieces[block4.places(M, D // 16)] = 0
        assert (pieces == 0).all()                                             # the rows behind M
        b = np.abs(y).reshape(M, -1, 16)
        be = err.reshape(M, -1, 16).max(2)
        t = b.max(2) / np.maximum(6 * row, 1e-300)[:, None]
        assert (np.abs(sc - np.minimum(t, 448)) <= np.maximum(2.0 ** -4 * t, 2.0 ** -10) + (be / np.maximum(6 * row, 1e-300)[:, None]) + 2.0 ** -20 * t).all()
        v = block4.values(block4.unpack(m.codes.cpu().numpy()), sc, row)
        step = (sc * row[:, None]).repeat(16, 1)
        # half a step of e2m1: a quarter of the value from the smallest step on; a scale that is 0 drops its block
        assert (np.abs(v - y) <= err + 0.25 * np.maximum(np.abs(y) + err, step) * (1 + 2.0 ** -20) + np.where(step == 0, 6 * row[:, None] * 2.0 ** -10, 0)).all()


def test_add_norm_forms(contexts):
    """Without vectors, without a gate, one set given flat, in place, and by an e4m3 result that op_gemm_fp8 takes."""
    ctx = contexts["f32"]
    x, kw = norm_case(9, 144, "f32", True, 0)
    for drop in [("weight", "shift", "gate"), ("gate",), ("shift",), ("weight",), ()]:
        k = {n: v for n, v in kw.items() if n not in drop}
        r, terms, y, err = norm_errors(x, k, 0.0, False, 1e-6, 0)
        xd = dev(x)
        d = {n: (v if n == "delta" else v[0]) for n, v in to_device(k, torch.float32).items()}
        d["delta"] = d["delta"].clone()
        ctx.op_add_norm(xd, d["delta"], total=xd, **d)                         # both outputs over their inputs
        assert (np.abs(host(xd) - r) <= 2.0 ** -22 * terms).all()
        assert (np.abs(host(d["delta"]) - y) <= err + 2.0 ** -24 * np.abs(y)).all()
    q, s = torch.empty(9, 144, dtype=F8, device="cuda"), torch.empty(2, 9, device="cuda")
    ctx.op_add_norm(dev(x), q, scale=s, **to_device(kw, torch.float32))
    wq, ws = chunk.quantize(synth.bf16_round(synth.normal(6, (24, 144))), 128)
    C = torch.empty(9, 24, device="cuda")
    ctx.op_gemm_fp8(q, s, dev(wq, F8), dev(ws), C)
    a, w = chunk.dequantize(host(q), s.cpu().numpy(), 1), chunk.dequantize(wq, ws, 128)
    assert np.allclose(host(C), a @ w.T, rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_addresses_that_are_multiples_of_16_bytes_only(contexts, kind):
    """Rows and vectors that do not start on 32 bytes: the same bits as those that do."""
    ctx, dt, D = contexts[kind], DTYPES[kind], 1088
    x, kw = norm_case(9, D, kind, True, 4)
    def moved(t, skip):
        b = torch.full((t.shape[0] * (t.shape[1] + 16 * (t.dtype == dt)) + 64,), 3.0, dtype=t.dtype, device="cuda")
        v = b[skip:].as_strided(t.shape, (t.shape[1] + 16 * (t.dtype == dt and t.shape[0] == 9), 1))
        v.copy_(t)
        assert v.data_ptr() % 32 == 16
        return v
    got = []
    for shift in (False, True):
        put = (lambda t: moved(t, 4 if t.dtype == torch.float32 else 8)) if shift else (lambda t: t)
        d = {n: put(v) for n, v in to_device(kw, dt).items()}
        xd, out, total, q = put(dev(x, dt)), put(dev(np.zeros((9, D)), dt)), put(dev(np.zeros((9, D)), dt)), wdc.Fp4Matrix.empty(9, D)
        ctx.op_add_norm(xd, out, total=total, rows_per_set=4, center=True, **d)
        ctx.op_quantize_fp4(xd, q)
        got.append([out.clone(), total.clone(), q.codes, q.scale.view(torch.uint8), q.row_scale])
        ctx.op_dequantize_fp4(q, out)
        got[-1].append(out.clone())
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_add_norm_of_zeros_and_nonfinite_rows(contexts):
    ctx = contexts["f32"]
    x = np.ones((5, 256), np.float32)
    x[0], x[1, 7], x[2, 9], x[3] = 0, np.nan, np.inf, 5e-20
    for center in (False, True):
        out, m = torch.empty(5, 256, device="cuda"), wdc.Fp4Matrix.empty(5, 256)
        q, s = torch.empty(5, 256, dtype=F8, device="cuda"), torch.empty(2, 5, device="cuda")
        ctx.op_add_norm(dev(x), out, center=center, weight=dev(np.ones(256)))
        ctx.op_add_norm(dev(x), q, scale=s, center=center, weight=dev(np.ones(256)))
        ctx.op_add_norm(dev(x), m, center=center, weight=dev(np.ones(256)))
        o = host(out)
        assert (o[0] == 0).all() and np.isnan(o[1]).all() and np.isnan(o[2]).any() and np.isfinite(o[[3, 4]]).all()
        assert (host(q)[0] == 0).all() and (host(s)[:, 0] == 0).all() and np.isnan(host(s)[:, 1]).all()
        r = host(m.row_scale)
        assert r[0] == 0 and np.isnan(r[[1, 2]]).all() and np.isfinite(r[[3, 4]]).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 256, 1024, 4096, 16384])
def test_layer_norm_of_equal_values(contexts, D, kind):
    """100.5 summed over a power of two of columns is exact, and so is the mean: the row less it is 0, whatever
    1 / sqrt(eps) is, and the result is the shift."""
    ctx, dt = contexts[kind], DTYPES[kind]
    x = np.full((3, D), 100.5, np.float32)
    x[1], x[2] = -0.75, 3.0
    shift = synth.bf16_round(synth.normal(93, (1, D), 0.3))
    for eps in (1e-6, 1e-5, 3e-7):
        out, q, s = torch.empty(3, D, dtype=dt, device="cuda"), torch.empty(3, D, dtype=F8, device="cuda"), torch.empty(-(-D // 128), 3, device="cuda")
        ctx.op_add_norm(dev(x, dt), out, center=True, eps=eps, weight=dev(np.full((1, D), 3.0)), shift=dev(shift))
        assert np.array_equal(host(out), np.repeat(shift, 3, 0))
        ctx.op_add_norm(dev(x, dt), q, scale=s, center=True, eps=eps)
        assert bool((s == 0).all()) and bool((q.float() == 0).all())


# ---------------------------------------------------------------- several axes
def axes_case(seed, T, pairs, rows):
    r = np.random.default_rng(seed)
    tables = [rotations(n, 2 * p) for n, p in zip(rows, pairs)]
    coords = np.stack([r.integers(0, n, T) for n in rows], 1).astype(np.int32).reshape(T, len(rows))
    return tables, coords, wdc.RotAxes([dev(t) for t in tables], dev(coords, torch.int32))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,kv,pairs", [(64, 4, 4, (12, 10, 10)), (64, 6, 1, (5, 3)), (128, 3, 3, (22, 21, 21)), (128, 8, 2, (1, 0, 54, 1)),
                                          (128, 2, 1, (64,)), (64, 2, 1, (0, 0))])
@pytest.mark.parametrize("T", [1, 9, 130])
@pytest.mark.parametrize("interleaved", [True, False])
def test_axes_dense(contexts, T, d, H, kv, pairs, interleaved, kind):
    ctx, dt = contexts[kind], DTYPES[kind]
    tables, coords, axes = axes_case(T, T, pairs, (7, 30, 45, 3)[:len(pairs)])
    x = synth.normal(51, (T, (H + 2 * kv) * d), 1.5)
    x = synth.bf16_round(x) if kind == "bf16" else x.astype(np.float32)
    wq, wk = 1 + synth.normal(52, (d,), 0.2), 1 + synth.normal(53, (d,), 0.2)
    ldv = -(-T // 8) * 8 if kind == "bf16" else T
    q, k = torch.empty(H, T, d, dtype=dt, device="cuda"), torch.empty(kv, T, d, dtype=dt, device="cuda")
    vt = torch.full((kv, d, ldv), 5.0, dtype=torch.half if kind == "bf16" else dt, device="cuda")
    kw = dict(q_weight=dev(wq), k_weight=dev(wk), eps=1e-5, interleaved=interleaved)
    ctx.op_qk_norm_rope(dev(x, dt), q, k, vt=vt, axes=axes, **kw)
    assert ctx.device_errors() == 0
    h = x.reshape(T, H + 2 * kv, d)
    cs = block4.axes_table(tables, coords)
    for got, part, w in ((q, h[:, :H], wq), (k, h[:, H:H + kv], wk)):
        want = chunk.norm_rotate(part, w, 1e-5, cs, np.arange(T), interleaved).transpose(1, 0, 2)
        assert (np.abs(host(got) - want) <= norm_bound(part, w, want, kind)).all()
    assert np.abs(host(vt[:, :, :T]) - h[:, H + kv:].transpose(1, 2, 0)).max() <= (2.0 ** -25 if kind == "bf16" else 0)
    q2, k2 = torch.empty_like(q), torch.empty_like(k)
    if sum(pairs):                                         # the same angles in one table: the same bits
        ctx.op_qk_norm_rope(dev(x, dt), q2, k2, rot=dev(cs), **kw)
        assert torch.equal(q, q2) and torch.equal(k, k2)


@pytest.mark.parametrize("d,H,kv,page,pairs", [(64, 6, 2, 16, (12, 10, 10)), (128, 5, 1, 32, (22, 21, 21)), (128, 4, 2, 256, (7, 1))])
@pytest.mark.parametrize("interleaved", [True, False])
def test_axes_append(contexts, d, H, kv, page, pairs, interleaved):
    """As with a table of the same angles by position in the sequence: the same bits in q and in the cache."""
    ctx = contexts["bf16"]
    new, past = [1, 5, 0, 70, 33], [0, 15, 9, 3, 40]
    T, extra = sum(new), 3
    tables, coords, axes = axes_case(8, T + extra, pairs, (7, 30, 45)[:len(pairs)])
    x = dev(synth.normal(62, (T + extra, (H + 2 * kv) * d), 1.5), torch.bfloat16)
    kw = dict(q_weight=dev(1 + synth.normal(63, (d,), 0.2)), interleaved=interleaved)
    got = []
    for form in (dict(axes=axes), dict(rot=dev(block4.axes_table(tables, coords)), positions=dev(np.arange(T + extra), torch.int32))):
        P = Paged(61, [n + p for n, p in zip(new, past)], page, kv, d)
        q = torch.full((T + extra, H, d), 5.0, dtype=torch.bfloat16, device="cuda")
        ctx.op_qk_norm_rope_append(x, q, P.cache, dev(starts(new), torch.int32), **kw, **form)
        assert ctx.device_errors() == 0 and bool((q[T:] == 5.0).all())
        got.append([t.view(torch.int16) for t in (q, P.dk, P.dv)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,kv,d", [(9605, 24, 24, 64), (5003, 48, 48, 64), (4801, 48, 8, 128), (9431, 10, 3, 128)])
@pytest.mark.parametrize("form", ["rot", "rot_halves", "axes"])
def test_a_long_clip_is_its_pieces(contexts, T, H, kv, d, form, kind):
    """Long clips take runs of heads and V^T tiles of more tokens (a whole token's heads a run, or two runs of
    equal or unequal length): the same bits as calls of 700 tokens at a time, which take neither."""
    ctx, dt = contexts[kind], DTYPES[kind]
    r = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(T, (H + 2 * kv) * d, device="cuda", generator=r).to(dt)
    w, tables = dev(1 + synth.normal(52, (d,), 0.2)), [dev(rotations(40, d // 2)), dev(rotations(9, d // 2))]
    angles, place = dev(rotations(300, d)), torch.randint(0, 300, (T,), device="cuda", generator=r, dtype=torch.int32)
    coords = torch.stack([place % 40, place % 9], 1).contiguous()

    def run(t0, t1):
        n = t1 - t0
        q, k = torch.empty(H, n, d, dtype=dt, device="cuda"), torch.empty(kv, n, d, dtype=dt, device="cuda")
        vt = torch.full((kv, d, -(-n // 8) * 8 if kind == "bf16" else n), 5.0, dtype=torch.half if kind == "bf16" else dt, device="cuda")
        how = dict(axes=wdc.RotAxes(tables, coords[t0:t1])) if form == "axes" else dict(rot=angles, positions=place[t0:t1])
        ctx.op_qk_norm_rope(x[t0:t1], q, k, vt=vt, q_weight=w, k_weight=w, interleaved=form != "rot_halves", **how)
        assert bool((vt[:, :, n:] == 5.0).all())
        return q, k, vt[:, :, :n].transpose(1, 2)
    whole, parts = run(0, T), [run(t, min(t + 700, T)) for t in range(0, T, 700)]
    assert all(torch.equal(a, torch.cat([p[i] for p in parts], 1)) for i, a in enumerate(whole)) and ctx.device_errors() == 0


@pytest.mark.parametrize("T,H,kv,d", [(9431, 24, 4, 64), (4801, 48, 8, 128), (3301, 24, 24, 128)])
@pytest.mark.parametrize("interleaved", [True, False])
def test_a_long_chunk_is_its_pieces(contexts, T, H, kv, d, interleaved):
    """The same for tokens appended to a cache: one sequence's all at once, and 700 at a time."""
    ctx, got = contexts["bf16"], []
    x = dev(synth.normal(62, (T, (H + 2 * kv) * d), 1.5), torch.bfloat16)
    w, angles = dev(1 + synth.normal(63, (d,), 0.2)), dev(rotations(T, d))
    for step in (T, 700):
        page, pages = 64, -(-T // 64)
        k, v = torch.zeros(pages, kv, page, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(pages, kv, page, d, dtype=torch.half, device="cuda")
        table, length = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0).view(1, -1).contiguous(), torch.zeros(1, dtype=torch.int32, device="cuda")
        cache, q = wdc.PagedCache(k, v, table, length), torch.empty(T, H, d, dtype=torch.bfloat16, device="cuda")
        for t in range(0, T, step):
            n = min(step, T - t)
            length.fill_(t + n)
            ctx.op_qk_norm_rope_append(x[t:t + n], q[t:t + n], cache, dev(starts([n]), torch.int32), q_weight=w, k_weight=w, rot=angles,
                                       interleaved=interleaved)
        assert ctx.device_errors() == 0
        got.append([a.view(torch.int16) for a in (q, k, v)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_coordinates_outside_their_table_are_reported(contexts):
    ctx = contexts["f32"]
    x = synth.normal(3, (3, 3 * 64))
    tables = [rotations(4, 32), rotations(6, 32)]
    q, k = torch.empty(1, 3, 64, device="cuda"), torch.empty(1, 3, 64, device="cuda")
    coords = np.array([[-5, 2], [3, 6], [0, 5]], np.int32)
    ctx.op_qk_norm_rope(dev(x), q, k, axes=wdc.RotAxes([dev(t) for t in tables], dev(coords, torch.int32)))
    assert ctx.device_errors() == 2
    cs = block4.axes_table(tables, [[0, 2], [3, 5], [0, 5]])
    want = chunk.norm_rotate(x.reshape(3, 3, 64)[:, :1], None, 1e-6, cs, [0, 1, 2], True).transpose(1, 0, 2)
    assert np.abs(host(q) - want).max() <= 2.0 ** -19 * 8


# ---------------------------------------------------------------- together
class Block:
    """A block of a chunk in four bits: norm, QKV, heads, attention over a paged cache, projection, norm, gated MLP."""
    D, H, kv, d, F, frame = 256, 4, 2, 64, 448, 24

    def __init__(self, ctx, T, seed=5):
        self.ctx, self.T = ctx, T
        r = np.random.default_rng(seed)
        w = lambda n, k: block4.quantize(synth.bf16_round((r.standard_normal((n, k)) * k ** -0.5).astype(np.float32)))
        self.host_w = dict(qkv=w((self.H + 2 * self.kv) * self.d, self.D), o=w(self.D, self.D), g=w(self.F, self.D), u=w(self.F, self.D),
                           down=w(self.D, self.F))
        self.w = {k: matrix(*v) for k, v in self.host_w.items()}
        e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
        self.x = dev(synth.normal(1, (T, self.D)), torch.bfloat16)
        self.mod = {n: dev(r.standard_normal((1, self.D)) * 0.3) for n in ("w1", "s1", "w2", "s2", "g1", "g2")}
        self.tables = [rotations(4, 24), rotations(6, 20), rotations(4, 20)]
        self.paged = Paged(7, [T + 37], 16, self.kv, self.d)
        at = np.arange(37, 37 + T)
        self.coords = np.stack([at // 24 % 4, at % 24 // 4, at % 4], 1).astype(np.int32)
        self.axes = wdc.RotAxes([dev(t) for t in self.tables], dev(self.coords, torch.int32))
        self.start = dev(starts([T]), torch.int32)
        self.h = wdc.Fp4Matrix.empty(T, self.D)
        self.qkv, self.q, self.att = e(T, (self.H + 2 * self.kv) * self.d), e(T, self.H, self.d), e(T, self.D)
        self.a4, self.branch, self.x1, self.h2 = wdc.Fp4Matrix.empty(T, self.D), e(T, self.D), e(T, self.D), wdc.Fp4Matrix.empty(T, self.D)
        self.mid, self.m4, self.out = e(T, self.F), wdc.Fp4Matrix.empty(T, self.F), e(T, self.D)

    def run(self, stream=None):
        c, m, s = self.ctx, self.mod, dict(stream=stream)
        c.op_add_norm(self.x, self.h, weight=m["w1"], weight_offset=1.0, shift=m["s1"], center=True, **s)
        c.op_gemm_fp4(self.h, self.w["qkv"], self.qkv, **s)
        c.op_qk_norm_rope_append(self.qkv, self.q, self.paged.cache, self.start, axes=self.axes, **s)
        c.op_attention_paged(self.q, self.paged.cache, self.start, self.att, self.T, frame=self.frame, **s)
        c.op_quantize_fp4(self.att, self.a4, **s)
        c.op_gemm_fp4(self.a4, self.w["o"], self.branch, **s)
        c.op_add_norm(self.x, self.h2, delta=self.branch, gate=m["g1"], total=self.x1, weight=m["w2"], weight_offset=1.0,
                      shift=m["s2"], center=True, **s)
        c.op_gated_fp4(self.h2, self.w["g"], self.w["u"], self.mid, **s)
        c.op_quantize_fp4(self.mid, self.m4, **s)
        c.op_gemm_fp4(self.m4, self.w["down"], self.out, res=self.x1, gate=m["g2"][0], **s)

    def results(self):
        return [t.clone() for t in (self.h.codes, self.h.scale.view(torch.uint8), self.qkv, self.q, self.att, self.branch, self.x1,
                                    self.h2.codes, self.mid, self.m4.codes, self.out)]

    def check(self):
        """Each step against fp64 on what the step before it gave."""
        val = lambda m: block4.values(block4.unpack(m.codes.cpu().numpy()), block4.from_pieces(host(m.scale), m.shape[0]), host(m.row_scale))
        mul = lambda m, w: (val(m) @ block4.values(*self.host_w[w]).T, np.abs(val(m)) @ np.abs(block4.values(*self.host_w[w])).T)
        near = lambda got, want, err: (np.abs(host(got) - want) <= err + 2.0 ** -8 * np.abs(want)).all()
        y, mag = mul(self.h, "qkv")
        assert near(self.qkv, y, product_bound(y, mag, self.D))
        h = host(self.qkv).reshape(self.T, -1, self.d)[:, :self.H]
        want = chunk.norm_rotate(h, None, 1e-6, block4.axes_table(self.tables, self.coords), np.arange(self.T), True)
        assert (np.abs(host(self.q) - want) <= norm_bound(h, None, want, "bf16")).all()
        check_rows(self.a4, host(self.att).astype(np.float32))
        y, mag = mul(self.a4, "o")
        assert near(self.branch, y, product_bound(y, mag, self.D))
        r = host(self.x) + host(self.mod["g1"]) * host(self.branch)
        assert near(self.x1, r, 2.0 ** -22 * (np.abs(host(self.x)) + np.abs(r)))
        (g, gm), (u, um) = mul(self.h2, "g"), mul(self.h2, "u")
        f = block4.silu(g)
        ge, ue = 1.13 * product_bound(g, gm, self.D) + 2.0 ** -18 * np.abs(f) + 1e-6, product_bound(u, um, self.D)
        assert near(self.mid, f * u, ge * np.abs(u) + np.abs(f) * ue + ge * ue)
        check_rows(self.m4, host(self.mid).astype(np.float32))
        y, mag = mul(self.m4, "down")
        gate = host(self.mod["g2"])
        assert near(self.out, host(self.x1) + gate * y, np.abs(gate) * product_bound(y, mag, self.F) + 2.0 ** -22 * np.abs(host(self.x1)))
        assert self.ctx.device_errors() == 0


@pytest.mark.parametrize("T", [1, 5, 24, 150])
def test_a_block_in_four_bits(contexts, T):
    b = Block(contexts["bf16"], T)
    b.run()
    b.check()


def test_captured_on_another_stream_and_replayed(contexts):
    b = Block(contexts["bf16"], 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run()
    side.synchronize()
    first = b.results()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run()
    for seed in (9, 1):                                    # other inputs, then the first again
        b.x.copy_(dev(synth.normal(seed, (40, b.D)), torch.bfloat16))
        b.out.zero_()
        g.replay()
        torch.cuda.synchronize()
        b.check()
    assert all(torch.equal(x, y) for x, y in zip(first, b.results()))


def test_two_contexts_at_once(contexts):
    """Split products of two contexts on two streams, each with its own workspace."""
    A, W, _, _ = split_case()
    a, w = matrix(*A), matrix(*W)
    both = [contexts["bf16"], wdc.Context(wdc.make_config(dtype=wdc.BF16, **MODEL), 2)]
    outs = [[torch.empty(*SPLIT[:2], dtype=torch.bfloat16, device="cuda") for _ in range(4)] for _ in both]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for i in range(4):
        for c, o, st in zip(both, outs, streams):
            c.op_gemm_fp4(a, w, o[i], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0][0], t) for o in outs for t in o)
    assert all(c.device_errors() == 0 for c in both)


def test_after_a_wait_that_gave_up(contexts):
    """The context is as before: a split product's counters too."""
    ctx = contexts["f32"]
    A, W, y, mag = split_case()
    ctx.selftest_wait_timeout(1000)
    assert ctx.device_errors() == 1
    C = torch.empty(*SPLIT[:2], device="cuda")
    ctx.op_gemm_fp4(matrix(*A), matrix(*W), C)
    assert (np.abs(host(C) - y) <= product_bound(y, mag, SPLIT[2]) + 2.0 ** -24 * np.abs(y)).all() and ctx.device_errors() == 0


def test_two_streams_of_one_context(contexts):
    """Split products of one context on streams by turns, none waiting on the host: one after the other on
    the device, through the one workspace; and beside a stream that was left."""
    A, W, _, _ = split_case()
    a, w, ctx = matrix(*A), matrix(*W), contexts["bf16"]
    new = lambda: torch.empty(*SPLIT[:2], dtype=torch.bfloat16, device="cuda")
    want = new()
    ctx.op_gemm_fp4(a, w, want)
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [(st, new()) for _ in range(4) for st in streams]
    torch.cuda.synchronize()
    for st, o in outs:
        ctx.op_gemm_fp4(a, w, o, stream=st)
    ctx.op_gemm_fp4(a, w, outs[0][1])
    torch.cuda.synchronize()
    assert all(torch.equal(want, o) for _, o in outs) and ctx.device_errors() == 0


def test_split_products_beside_a_capture(contexts):
    """A capture takes up no wait for products outside it, and those go on; replays give the same bits."""
    A, W, _, _ = split_case()
    a, w, ctx = matrix(*A), matrix(*W), contexts["bf16"]
    new = lambda: torch.zeros(*SPLIT[:2], dtype=torch.bfloat16, device="cuda")
    want, before, inside, after = new(), new(), new(), new()
    ctx.op_gemm_fp4(a, w, want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ctx.op_gemm_fp4(a, w, before, stream=side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.op_gemm_fp4(a, w, inside)
    torch.cuda.synchronize()
    for _ in range(2):
        inside.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, inside)
    ctx.op_gemm_fp4(a, w, after, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(want, before) and torch.equal(want, after) and ctx.device_errors() == 0


def test_device_errors_makes_the_counters_zero(contexts):
    """Whatever counts calls at the same time have left, with no error bit set."""
    ctx = contexts["f32"]
    A, W, y, mag = split_case()
    C = torch.empty(*SPLIT[:2], device="cuda")
    ctx.selftest_fp4_counters()
    assert ctx.device_errors() == 0
    ctx.op_gemm_fp4(matrix(*A), matrix(*W), C)
    assert (np.abs(host(C) - y) <= product_bound(y, mag, SPLIT[2]) + 2.0 ** -24 * np.abs(y)).all() and ctx.device_errors() == 0


# ---------------------------------------------------------------- offsets past 32 bits
def ends(t, n=3):
    return torch.cat([t[:n], t[-n:]])


def test_rows_past_32_bits(contexts):
    """More than 2^31 elements: the first and the last rows of a matrix of codes and back."""
    ctx, M, K = contexts["bf16"], 66000, 32832
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    rows = rows_of(5, 6, K, "bf16")
    x[:3], x[-3:] = dev(rows[:3], torch.bfloat16), dev(rows[3:], torch.bfloat16)
    q = wdc.Fp4Matrix.empty(M, K)
    ctx.op_quantize_fp4(x, q)
    x.fill_(7.0)
    ctx.op_dequantize_fp4(q, x)
    want = block4.values(*block4.quantize(rows))
    assert (np.abs(host(ends(x)) - want) <= (2.0 ** -8 + 2.0 ** -22) * np.abs(want)).all()
    assert np.array_equal(block4.unpack(ends(q.codes).cpu().numpy()), block4.quantize(rows)[0])
    assert bool((x[3:-3] == 0).all())


@pytest.mark.parametrize("gated", [False, True])
def test_results_past_32_bits(contexts, gated):
    ctx, M, N, K = contexts["bf16"], 66000, 32832, 64
    A, W = block4.quantize(rows_of(6, 6, K, "bf16")), block4.quantize(rows_of(7, 4, K, "bf16"))
    a = wdc.Fp4Matrix(*(torch.zeros_like(t) for t in (lambda m: (m.codes, m.scale, m.row_scale))(wdc.Fp4Matrix.empty(M, K))))
    w = wdc.Fp4Matrix(*(torch.zeros_like(t) for t in (lambda m: (m.codes, m.scale, m.row_scale))(wdc.Fp4Matrix.empty(N, K))))
    for m, v, n in ((a, A, M), (w, W, N)):
        k = len(v[2]) // 2
        at = np.concatenate([np.arange(k), np.arange(n - k, n)])
        m.codes[at], m.row_scale[at] = torch.from_numpy(block4.pack(v[0])).cuda(), dev(v[2])
        r, j = at[:, None], np.arange(K // 16)[None]
        m.scale.view(torch.uint8)[r // 128, j // 4, r % 32 * 16 + r // 32 % 4 * 4 + j % 4] = dev(v[1], F8).view(torch.uint8)
    C = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    if gated:
        ctx.op_gated_fp4(a, w, w, C)
    else:
        ctx.op_gemm_fp4(a, w, C)
    y = block4.values(*A) @ block4.values(*W).T
    mag = np.abs(block4.values(*A)) @ np.abs(block4.values(*W)).T
    e = product_bound(y, mag, K)
    if gated:
        f = block4.silu(y)
        y, e = f * y, (1.13 * e + 2.0 ** -18 * np.abs(f) + 1e-6) * np.abs(y) + np.abs(f) * e + 3 * e * e
    got = host(ends(ends(C).t().contiguous(), 2).t())
    assert (np.abs(got - y) <= e + 2.0 ** -8 * np.abs(y)).all()
    assert bool((C[3:-3] == 0).all()) and bool((C[:, 2:-2] == 0).all()) and ctx.device_errors() == 0


def test_norm_past_32_bits(contexts):
    ctx, M, D = contexts["bf16"], 140000, 16384
    x = torch.ones(M, D, dtype=torch.bfloat16, device="cuda")
    rows = synth.bf16_round(synth.normal(8, (6, D)))
    x[:3], x[-3:] = dev(rows[:3], torch.bfloat16), dev(rows[3:], torch.bfloat16)
    q, s = torch.empty(M, D, dtype=F8, device="cuda"), torch.empty(D // 128, M, device="cuda")
    ctx.op_add_norm(x, q, scale=s)
    ctx.op_add_norm(x, x)                                          # in place
    _, _, y, err = norm_errors(rows, {}, 0.0, False, 1e-6, 0)
    assert (np.abs(host(ends(x)) - y) <= err + 2.0 ** -8 * np.abs(y)).all()
    step = host(ends(s.t().contiguous())).repeat(128, 1)
    assert (np.abs(host(ends(q)) * step - y) <= err + 2.0 ** -20 * np.abs(y) + np.maximum(2.0 ** -4 * (np.abs(y) + err), 2.0 ** -10 * step)).all()
    assert bool((x[3:-3] == 1).all())


# ---------------------------------------------------------------- refusals
def test_refusals_of_the_library(contexts):
    ctx = contexts["bf16"]
    x, m, out = dev(np.ones((4, 64)), torch.bfloat16), wdc.Fp4Matrix.empty(4, 64), torch.empty(4, 8, dtype=torch.bfloat16, device="cuda")
    w, L, s, p = wdc.Fp4Matrix.empty(8, 64), wdc.LIB, torch.cuda.current_stream().cuda_stream, x.data_ptr()
    off = wdc.Fp4C(m.codes.data_ptr() + 4, m.c.scale, m.c.row_scale)
    none = wdc.Fp4C(m.c.codes, None, m.c.row_scale)
    before = ctx.launches
    for want, got in [(1, L.wdc_op_quantize_fp4(ctx._h, p, 64, m.c, -1, 64, s)), (1, L.wdc_op_quantize_fp4(ctx._h, p, 32, m.c, 4, 64, s)),
                      (3, L.wdc_op_quantize_fp4(ctx._h, p, 96, m.c, 4, 96, s)), (3, L.wdc_op_quantize_fp4(ctx._h, p, 68, m.c, 4, 64, s)),
                      (1, L.wdc_op_quantize_fp4(ctx._h, p + 2, 64, m.c, 4, 64, s)), (1, L.wdc_op_quantize_fp4(ctx._h, p, 64, off, 4, 64, s)),
                      (1, L.wdc_op_quantize_fp4(ctx._h, p, 64, none, 4, 64, s)), (1, L.wdc_op_quantize_fp4(ctx._h, None, 64, m.c, 4, 64, s)),
                      (1, L.wdc_op_quantize_fp4(ctx._h, p, 64, None, 4, 64, s)), (0, L.wdc_op_quantize_fp4(ctx._h, None, 64, m.c, 0, 64, s)),
                      (3, L.wdc_op_quantize_fp4(ctx._h, p, 64, m.c, 2 ** 31 - 1, 64, s)),
                      (3, L.wdc_op_quantize_fp4(ctx._h, p, 2 ** 31, m.c, 4, 2 ** 31 - 64, s)),
                      (1, L.wdc_op_dequantize_fp4(ctx._h, m.c, None, 64, 4, 64, s)), (1, L.wdc_op_dequantize_fp4(ctx._h, none, p, 64, 4, 64, s)),
                      (3, L.wdc_op_dequantize_fp4(ctx._h, m.c, p, 96, 4, 96, s)), (0, L.wdc_op_dequantize_fp4(ctx._h, m.c, p, 64, 0, 64, s)),
                      (3, L.wdc_op_gemm_fp4(ctx._h, m.c, w.c, None, p, 4, 4, 64, 0, None, None, s)),
                      (3, L.wdc_op_gemm_fp4(ctx._h, m.c, w.c, None, p, 4, 8, 32, 0, None, None, s)),
                      (1, L.wdc_op_gemm_fp4(ctx._h, m.c, w.c, None, None, 4, 8, 64, 0, None, None, s)),
                      (1, L.wdc_op_gemm_fp4(ctx._h, m.c, w.c, p + 4, p, 4, 8, 64, 0, None, None, s)),
                      (1, L.wdc_op_gemm_fp4(ctx._h, none, w.c, None, p, 4, 8, 64, 0, None, None, s)),
                      (1, L.wdc_op_gemm_fp4(ctx._h, m.c, None, None, p, 4, 8, 64, 0, None, None, s)),
                      (1, L.wdc_op_gemm_fp4(ctx._h, m.c, w.c, None, p, -4, 8, 64, 0, None, None, s)),
                      (0, L.wdc_op_gemm_fp4(ctx._h, m.c, w.c, None, p, 0, 8, 64, 0, None, None, s)),
                      (1, L.wdc_op_gated_fp4(ctx._h, m.c, w.c, None, None, None, p, 4, 8, 64, 0, s)),
                      (1, L.wdc_op_gated_fp4(ctx._h, m.c, w.c, off, None, None, p, 4, 8, 64, 0, s)),
                      (1, L.wdc_op_gated_fp4(ctx._h, m.c, w.c, w.c, None, p + 8, p, 4, 8, 64, 0, s)),
                      (0, L.wdc_op_gated_fp4(ctx._h, m.c, w.c, w.c, None, None, p, 0, 8, 64, 0, s))]:
        assert got == want
    good = dict(x=p, ldx=64, out=p, ldo=64, eps=1e-6)
    q4 = ctypes.pointer(m.c)
    for want, M, D, kw in [(1, -1, 64, {}), (1, 4, 0, {}), (3, 4, 72, dict(ldx=72, ldo=72)), (3, 1, 16400, dict(ldx=16400, ldo=16400)), (1, 4, 64, dict(eps=-1.0)),
                           (1, 4, 64, dict(eps=float("nan"))), (1, 4, 64, dict(rows_per_set=-1)), (1, 4, 64, dict(out=None)),
                           (1, 4, 64, dict(q8=p, scale=p)), (1, 4, 64, dict(out=None, q8=p)), (1, 4, 64, dict(gate=p)), (1, 4, 64, dict(ldx=56)),
                           (3, 4, 64, dict(ldo=68)), (1, 4, 64, dict(delta=p, ldd=32)), (1, 4, 64, dict(total=p + 512)), (1, 4, 64, dict(x=p + 4)),
                           (1, 4, 64, dict(x=None)), (3, 4, 80, dict(ldx=80, out=None, q4=q4)), (1, 4, 64, dict(out=None, q4=ctypes.pointer(off))),
                           (1, 4, 64, dict(weight=p + 4)), (1, 4, 64, dict(total=p, ldt=64)), (0, 0, 64, {})]:
        assert L.wdc_op_add_norm(ctx._h, wdc.AddNorm(**dict(good, **kw)), M, D, s) == want, (M, D, kw)
    assert L.wdc_op_add_norm(ctx._h, None, 4, 64, s) == 1

    def axes(**kw):
        a = wdc.RotAxesC(kw.get("axes", 2), coords=kw.get("coords", p))
        for i in range(2):
            a.table[i], a.rows[i], a.pairs[i] = kw.get("table", p), kw.get("rows", 4), kw.get("pairs", (4, 12))[i]
        return a
    norm = wdc.HeadNorm(None, None, 1e-6, None, 0, 0, 1, None)
    with_table = wdc.HeadNorm(None, None, 1e-6, p, 4, 16, 1, None)
    for want, n, a in [(1, norm, axes(axes=0)), (1, norm, axes(axes=5)), (1, norm, axes(pairs=(-8, 16))), (1, norm, axes(pairs=(24, 16))),
                       (1, norm, axes(pairs=(4, 8))), (1, norm, axes(rows=0)), (1, norm, axes(table=None)), (1, norm, axes(table=p + 4)),
                       (1, norm, axes(coords=None)), (1, norm, axes(coords=p + 2)), (1, with_table, axes()), (1, norm, None), (1, None, axes())]:
        assert L.wdc_op_qk_norm_rope_axes(ctx._h, p, 192, 1, 1, 1, 64, n, a, p, p, None, s) == want
    assert ctx.launches == before and ctx.device_errors() == 0


def test_axes_look_at_nothing_else(contexts):
    """With axes the norm's rot_positions, rot_dim and positions are not looked at, nor is what belongs to an axis
    without pairs: whatever they hold, the call is taken and turns the heads as without them."""
    ctx, L = contexts["bf16"], wdc.LIB
    s = torch.cuda.current_stream().cuda_stream
    x = dev(synth.normal(3, (5, 3 * 64)), torch.bfloat16)
    tables, coords, axes = axes_case(3, 5, (4, 12), (7, 30))
    outs = []
    for positions, size, dim, skip in [(None, 0, 0, False), (x.data_ptr() + 2, -1, 7, False), (x.data_ptr() + 1, 3, 16, True)]:
        a = wdc.RotAxesC(2, coords=axes.c.coords)
        for i in range(2):
            a.table[i], a.rows[i], a.pairs[i] = axes.c.table[i], axes.c.rows[i], axes.c.pairs[i]
        q, k = torch.zeros(1, 5, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 5, 64, dtype=torch.bfloat16, device="cuda")
        if skip:                                           # no axis has pairs: no coordinates either
            a.coords = x.data_ptr() + 2
            for i in range(2):
                a.table[i], a.rows[i], a.pairs[i] = x.data_ptr() + 1, -5, 0
        n = wdc.HeadNorm(None, None, 1e-6, None, size, dim, 1, positions)
        assert L.wdc_op_qk_norm_rope_axes(ctx._h, x.data_ptr(), 192, 5, 1, 1, 64, n, a, q.data_ptr(), k.data_ptr(), None, s) == 0
        outs.append((q, k))
    plain = [torch.zeros(1, 5, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx.op_qk_norm_rope(x, *plain)
    assert all(torch.equal(u, v) for u, v in zip(outs[0], outs[1])) and all(torch.equal(u, v) for u, v in zip(outs[2], plain))
    assert not torch.equal(outs[0][0], plain[0]) and ctx.device_errors() == 0


def test_refusals_of_places(contexts):
    """A row is read by one block while another writes its own: an output lies on an input row for row or not at
    all, and a result in few bits on neither the inputs nor the sum."""
    ctx, L = contexts["bf16"], wdc.LIB
    s = torch.cuda.current_stream().cuda_stream
    x, y, t = (torch.ones(4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    p, d, o = (v.data_ptr() for v in (x, y, t))
    m = wdc.Fp4Matrix.empty(4, 64)
    q4 = lambda **kw: dict(out=None, q4=ctypes.pointer(wdc.Fp4C(*(kw.get(n, getattr(m.c, n)) for n in ("codes", "scale", "row_scale")))))
    good = dict(x=p, ldx=128, delta=d, ldd=128, out=o, ldo=64, eps=1e-6)
    before = ctx.launches
    for kw in [dict(out=p, ldo=64), dict(out=d, ldo=64), dict(total=p, ldt=64), dict(total=d, ldt=72), dict(out=p, ldo=128, ldx=64),
               dict(total=o, ldt=64), dict(out=None, q8=p, scale=o), dict(out=None, q8=d, scale=o), dict(out=None, q8=o, scale=p),
               dict(out=None, q8=o, scale=d), dict(out=None, q8=o, scale=p + 512, total=o, ldt=64),
               dict(out=None, q8=o, scale=p + 512, total=p + 512, ldt=64)]:
        assert L.wdc_op_add_norm(ctx._h, wdc.AddNorm(**dict(good, **kw)), 4, 64, s) == 1, kw
    for field in ("codes", "scale", "row_scale"):
        for at in (p, d):
            assert L.wdc_op_add_norm(ctx._h, wdc.AddNorm(**dict(good, **q4(**{field: at}))), 4, 64, s) == 1
        assert L.wdc_op_add_norm(ctx._h, wdc.AddNorm(**dict(good, total=o, ldt=64, **q4(**{field: o}))), 4, 64, s) == 1
    assert ctx.launches == before
    for M, kw in [(1, dict(out=p, ldo=64)), (4, dict(out=p, ldo=128)), (4, dict(total=d, ldt=128))]:
        assert L.wdc_op_add_norm(ctx._h, wdc.AddNorm(**dict(good, **kw)), M, 64, s) == 0, kw
    assert ctx.launches == before + 3 and ctx.device_errors() == 0


def test_nothing_to_do(contexts):
    ctx, e = contexts["bf16"], lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
    before, m = ctx.launches, wdc.Fp4Matrix.empty(0, 64)
    ctx.op_add_norm(e(0, 64), e(0, 64))
    ctx.op_add_norm(e(0, 64), m)
    ctx.op_quantize_fp4(e(0, 64), m)
    ctx.op_dequantize_fp4(m, e(0, 64))
    ctx.op_gemm_fp4(m, wdc.Fp4Matrix.empty(8, 64), e(0, 8))
    ctx.op_gated_fp4(m, wdc.Fp4Matrix.empty(8, 64), wdc.Fp4Matrix.empty(8, 64), e(0, 8))
    t = [torch.empty(3, 16, 2, device="cuda")]
    ctx.op_qk_norm_rope(e(0, 192), e(1, 0, 64), e(1, 0, 64), axes=wdc.RotAxes(t, torch.empty(0, 1, dtype=torch.int32, device="cuda")))
    assert ctx.launches == before
