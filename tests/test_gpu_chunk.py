"""The chunk operators against fp64: e4m3 blocks, their product, head norms with
rotation (dense and into a paged cache) and attention over that cache, at the
sizes, masks and page ends where they can go wrong, and all of them together."""
import numpy as np
import pytest
import torch

from oracle import chunk, dit
from paper_2608_01845_gb300 import synth, wdc

pytestmark = pytest.mark.gpu

MODEL = dict(layers=1, hidden=256, heads=4, head_dim=64, mlp=256, temb_dim=256, freq_dim=256, in_ch=16, frames=1,
             height=16, width=16, patch=2, cond_tokens=16, cond_dim=64)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# a result's one rounding: half a step, relative
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def contexts():
    return {k: wdc.Context(wdc.make_config(dtype=wdc.F32 if k == "f32" else wdc.BF16, **MODEL), 2) for k in DTYPES}


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def host(t):
    return t.double().cpu().numpy()


def rows_of(seed, M, K, kind):
    """Activations with wide and narrow channels; some rows (and so whole blocks) zero."""
    x = synth.normal(seed, (M, K)) * np.exp(synth.normal(seed + 1, (K,)))
    x[::7] *= 1e-6
    if M > 2:
        x[2] = 0
    return synth.bf16_round(x) if kind == "bf16" else x.astype(np.float32)


# ---------------------------------------------------------------- e4m3 blocks
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 16), (1, 128), (3, 144), (8, 1024), (9, 1040), (127, 256), (129, 272), (300, 2064)])
def test_quantize(contexts, M, K, rows, kind):
    """Bit for bit: scale and quotient are single IEEE operations."""
    ctx = contexts[kind]
    x = rows_of(11, M, K, kind)
    want, ws = chunk.quantize(x, rows)
    buf = torch.full((M + 1, K), 3.0, device="cuda").to(torch.float8_e4m3fn)
    scale = torch.full((ws.size + 4,), 7.0, device="cuda")
    s = scale[:ws.size].view(ws.shape)
    ctx.op_quantize_fp8(dev(x, DTYPES[kind]), buf[:M], s, block_rows=rows)
    assert np.array_equal(s.cpu().numpy(), ws)
    assert np.array_equal(host(buf[:M]), want)
    assert bool((buf[M:].float() == 3.0).all()) and bool((scale[ws.size:] == 7.0).all())


@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_quotients_are_ieee(contexts, rows):
    """Scales of every size, from subnormal to the largest, and values of every size below them: bit for bit."""
    g = np.random.default_rng(5)
    M, K = 256 * rows // (2 if rows > 1 else 1), 256
    top = np.exp2(g.integers(-149, 127, (M // rows, K // 128))).repeat(rows, 0).repeat(128, 1)
    with np.errstate(over="ignore", under="ignore"):
        x = (top * (1 + g.random((M, K))) * np.exp2(-g.integers(0, 20, (M, K))) * g.choice([-1, 1], (M, K))).astype(np.float32)
    x = np.clip(x, -3e38, 3e38)
    want, ws = chunk.quantize(x, rows)
    q, s = torch.empty(M, K, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(ws.shape, device="cuda")
    contexts["f32"].op_quantize_fp8(dev(x), q, s, block_rows=rows)
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(host(q), want)


def test_quantize_rows_that_lie_apart(contexts):
    x = rows_of(12, 20, 400, "bf16")
    t = dev(x, torch.bfloat16)
    q, s = torch.empty(20, 160, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(2, 20, device="cuda")
    contexts["bf16"].op_quantize_fp8(t[:, 80:240], q, s)
    want, ws = chunk.quantize(x[:, 80:240])
    assert np.array_equal(host(q), want) and np.array_equal(s.cpu().numpy(), ws)


def test_quantize_nonfinite_and_tiny(contexts):
    x = np.ones((5, 256), np.float32)
    x[0, 3], x[1, 130], x[2, 5] = np.inf, np.nan, -np.inf
    x[3] = 1e-45
    t = dev(x)
    q, s = torch.empty(5, 256, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(2, 5, device="cuda")
    contexts["f32"].op_quantize_fp8(t, q, s)
    q, s = host(q), s.cpu().numpy()
    assert np.isinf(s[0, 0]) and np.isnan(s[1, 1]) and np.isinf(s[0, 2]) and np.isfinite(s[1, [0, 2, 4]]).all()
    assert np.isnan(q[0, 3]) and np.isnan(q[1, 128:]).all() and np.isnan(q[2, 5])
    assert (np.delete(q[0, :128], 3) == 0).all() and (q[1, :128] == 448).all() and (q[4] == 448).all()
    assert (s[:, 3] == 0).all() and (q[3] == 0).all()          # a scale that underflows: the block is zero


# ---------------------------------------------------------------- product
def gemm_case(seed, M, N, K, kind):
    A, sa = chunk.quantize(rows_of(seed, M, K, "bf16"))
    W, sw = chunk.quantize(synth.bf16_round(synth.normal(seed + 5, (N, K), K ** -0.5)), 128)
    return A, sa, W, sw


def run_gemm(ctx, A, sa, W, sw, C, **kw):
    f8 = torch.float8_e4m3fn
    ctx.op_gemm_fp8(dev(A, f8), dev(sa), dev(W, f8), dev(sw), C, **kw)


def gemm_bound(A, sa, W, sw, want, kind):
    """A block's products are summed with at most 2^-23 lost an addition (a
    truncated fp32 sum), the blocks and the epilogue's few terms in fp32: in all at
    most (128 + blocks + 4) 2^-23 of the terms' magnitudes, and one rounding."""
    mag = np.abs(chunk.dequantize(A, sa, 1)) @ np.abs(chunk.dequantize(W, sw, 128)).T
    return HALF[kind] * np.abs(want) + (132 + sa.shape[0]) * 2.0 ** -23 * mag


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 5, 16, 17, 33, 64, 100, 129, 300])
@pytest.mark.parametrize("N,K", [(8, 16), (136, 144), (256, 1024), (1032, 2064)])
def test_gemm(contexts, M, N, K, kind):
    ctx = contexts[kind]
    A, sa, W, sw = gemm_case(21, M, N, K, kind)
    want = chunk.dequantize(A, sa, 1) @ chunk.dequantize(W, sw, 128).T
    buf = torch.full((M + 2, N), 7.0, dtype=DTYPES[kind], device="cuda")
    run_gemm(ctx, A, sa, W, sw, buf[:M])
    assert ctx.device_errors() == 0
    assert (np.abs(host(buf[:M]) - want) <= gemm_bound(A, sa, W, sw, want, kind)).all()
    assert bool((buf[M:] == 7.0).all())


@pytest.mark.parametrize("kind", ["bf16", "f32"])
# (in this order: one narrow tile; several, K over a cluster; the pair kernel's tiles
# of 128 and of 256 columns, several a pair in the last)
@pytest.mark.parametrize("M,N,K", [(3, 264, 528), (40, 392, 8208), (520, 2312, 2064), (1030, 2056, 1040), (2309, 3080, 528)])
@pytest.mark.parametrize("mode", ["bias", "gelu", "resid", "resid_gelu", "gateless"])
def test_gemm_epilogues(contexts, M, N, K, mode, kind):
    """The epilogue's own error: 1.13 (GELU's steepest slope) of the sum's, 2^-18 of
    GELU's value for its exponential and quotient, the gate's multiple of both."""
    ctx = contexts[kind]
    A, sa, W, sw = gemm_case(31, M, N, K, kind)
    b, g = synth.normal(3, (N,), 0.5), synth.normal(5, (N,))
    r = synth.bf16_round(synth.normal(4, (M, N)))
    y = chunk.dequantize(A, sa, 1) @ chunk.dequantize(W, sw, 128).T + b
    err = gemm_bound(A, sa, W, sw, 0 * y, kind) + 2.0 ** -22 * np.abs(y)
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
    run_gemm(ctx, A, sa, W, sw, C, **kw)
    assert (np.abs(host(C) - y) <= err + HALF[kind] * np.abs(y) + 2.0 ** -22 * np.abs(y)).all()


def test_gemm_any_scales(contexts):
    """Scales are fp32 values of any size and sign, not only quantize's."""
    A, sa, W, sw = gemm_case(41, 70, 264, 1040, "f32")
    sa = (sa * np.exp(4 * synth.normal(1, sa.shape))).astype(np.float32)
    sw = (sw * synth.normal(2, sw.shape)).astype(np.float32)
    C = torch.empty(70, 264, device="cuda")
    run_gemm(contexts["f32"], A, sa, W, sw, C)
    want = chunk.dequantize(A, sa, 1) @ chunk.dequantize(W, sw, 128).T
    assert (np.abs(host(C) - want) <= gemm_bound(A, sa, W, sw, want, "f32") + 2.0 ** -22 * np.abs(want)).all()


def test_gemm_nonfinite_rows_stay_in_their_rows(contexts):
    A, sa, W, sw = gemm_case(43, 40, 136, 256, "f32")
    want = chunk.dequantize(A, sa, 1) @ chunk.dequantize(W, sw, 128).T
    A[5, 3], sa[1, 9] = np.nan, np.inf
    C = torch.empty(40, 136, device="cuda")
    run_gemm(contexts["f32"], A, sa, W, sw, C)
    got = host(C)
    assert np.isnan(got[5]).all() and not np.isfinite(got[9]).any()
    rest = [i for i in range(40) if i not in (5, 9)]
    assert np.isfinite(got[rest]).all() and np.allclose(got[rest], want[rest], rtol=1e-4, atol=1e-4)


# ---------------------------------------------------------------- norm and rotation
def rotations(n, rot):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def norm_bound(x, w, want, kind):
    """fp32: a mean of at most 128 squares, a root, a quotient, two products and the
    rotation's two, each off by a few 2^-24: below 2^-19 of the pair's magnitudes
    (of which |y| <= sqrt(d) max |w| is the most); and one rounding."""
    top = np.sqrt(x.shape[-1]) * (1 if w is None else np.abs(w).max())
    return HALF[kind] * np.abs(want) + 2.0 ** -19 * top


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,kv", [(64, 4, 4), (64, 6, 1), (128, 3, 3), (128, 8, 2)])
@pytest.mark.parametrize("T", [1, 7, 8, 65, 130])
@pytest.mark.parametrize("interleaved", [True, False])
def test_norm_rope_dense(contexts, T, d, H, kv, interleaved, kind):
    ctx, dt = contexts[kind], DTYPES[kind]
    rot = {1: 0, 7: 16, 8: d, 65: d - 16, 130: d}[T]
    x = synth.normal(51, (T, (H + 2 * kv) * d), 1.5)
    x = synth.bf16_round(x) if kind == "bf16" else x.astype(np.float32)
    wq, wk = 1 + synth.normal(52, (d,), 0.2), None if T == 8 else 1 + synth.normal(53, (d,), 0.2)
    pos = None if T < 65 else np.random.default_rng(1).integers(0, 300, T).astype(np.int32)
    cs = rotations(300, rot) if rot else None
    wide = torch.full((T, x.shape[1] + 16), 9.0, dtype=dt, device="cuda")      # rows lie apart
    wide[:, :x.shape[1]] = dev(x, dt)
    ldv = -(-T // 8) * 8 if kind == "bf16" else T
    q, k = torch.empty(H, T, d, dtype=dt, device="cuda"), torch.empty(kv, T, d, dtype=dt, device="cuda")
    vt = torch.full((kv, d, ldv), 5.0, dtype=torch.half if kind == "bf16" else dt, device="cuda")
    ctx.op_qk_norm_rope(wide[:, :x.shape[1]], q, k, vt=vt, q_weight=dev(wq), k_weight=None if wk is None else dev(wk),
                        eps=1e-5, rot=None if cs is None else dev(cs), positions=None if pos is None else dev(pos, torch.int32),
                        interleaved=interleaved)
    assert ctx.device_errors() == 0
    h = x.reshape(T, H + 2 * kv, d)
    at = np.arange(T) if pos is None else pos
    for got, part, w in ((q, h[:, :H], wq), (k, h[:, H:H + kv], wk)):
        want = chunk.norm_rotate(part, w, 1e-5, cs, at, interleaved).transpose(1, 0, 2)
        assert (np.abs(host(got) - want) <= norm_bound(part, w, want, kind)).all()
    v = h[:, H + kv:].transpose(1, 2, 0)
    assert np.abs(host(vt[:, :, :T]) - v).max() <= (2.0 ** -25 if kind == "bf16" else 0)
    assert bool((vt[:, :, T:] == 5.0).all())


def test_norm_of_zeros_and_without_eps(contexts):
    x = np.zeros((2, 3 * 64), np.float32)
    x[1] = 2.0
    q, k = torch.empty(1, 2, 64, device="cuda"), torch.empty(1, 2, 64, device="cuda")
    contexts["f32"].op_qk_norm_rope(dev(x), q, k, eps=1e-6)
    assert bool((q[0, 0] == 0).all()) and np.allclose(host(q[0, 1]), 1.0, atol=1e-6)
    contexts["f32"].op_qk_norm_rope(dev(x), q, k, eps=0.0)
    assert bool(q[0, 0].isnan().all()) and np.allclose(host(k[0, 1]), 1.0, atol=1e-6)


def test_rot_dim_without_angles_is_not_looked_at(contexts):
    x = synth.normal(4, (5, 3 * 64)).astype(np.float32)
    q, k = torch.empty(1, 5, 64, device="cuda"), torch.empty(1, 5, 64, device="cuda")
    ctx, dx = contexts["f32"], dev(x)
    for pairs in (0, 1):
        n = wdc.HeadNorm(None, None, 1e-5, None, 0, 1 << 20, pairs, None)
        q.fill_(9)
        assert wdc.LIB.wdc_op_qk_norm_rope(ctx._h, dx.data_ptr(), 3 * 64, 5, 1, 1, 64, n, q.data_ptr(), k.data_ptr(), None,
                                           torch.cuda.current_stream().cuda_stream) == 0
        h = x.reshape(5, 3, 64)
        want = chunk.norm_rotate(h[:, :1], None, 1e-5, None, np.arange(5), bool(pairs)).transpose(1, 0, 2)
        assert (np.abs(host(q) - want) <= norm_bound(h, None, want, "f32")).all()


def test_positions_outside_the_table_are_reported(contexts):
    ctx = contexts["f32"]
    x, cs = synth.normal(3, (3, 3 * 64)), rotations(4, 64)
    q, k = torch.empty(1, 3, 64, device="cuda"), torch.empty(1, 3, 64, device="cuda")
    ctx.op_qk_norm_rope(dev(x), q, k, rot=dev(cs), positions=torch.tensor([-5, 2, 4], dtype=torch.int32, device="cuda"))
    assert ctx.device_errors() == 2
    want = chunk.norm_rotate(x.reshape(3, 3, 64)[:, :1], None, 1e-6, cs, [0, 2, 3], True).transpose(1, 0, 2)
    assert np.abs(host(q) - want).max() <= 2.0 ** -19 * 8


# ---------------------------------------------------------------- paged cache
class Paged:
    """Sequences' pages in a random order in a pool that is full of NaN and infinities."""

    def __init__(self, seed, lens, page, kv, d, spare=2, fill=True):
        r = np.random.default_rng(seed)
        self.page, self.kv, self.d, self.lens = page, kv, d, list(lens)
        width = max([-(-n // page) for n in lens] + [0]) + spare
        self.pages = len(lens) * width + 3
        self.table = r.permutation(self.pages)[:len(lens) * width].reshape(len(lens), width).astype(np.int32)
        bad = np.where(r.random((self.pages, kv, page, d)) < 0.5, np.nan, np.inf)
        self.k, self.v = bad.astype(np.float32), (-bad).astype(np.float32)
        for b, n in enumerate(lens if fill else []):
            i = np.arange(n)
            p = self.table[b, i // page]
            self.k[p, :, i % page] = synth.bf16_round(r.standard_normal((n, kv, d)).astype(np.float32))
            self.v[p, :, i % page] = r.standard_normal((n, kv, d)).astype(np.float16)
        self.dk, self.dv = dev(self.k, torch.bfloat16), dev(self.v, torch.half)
        self.dtable, self.dlen = dev(self.table, torch.int32), torch.tensor(list(lens), dtype=torch.int32, device="cuda")
        self.cache = wdc.PagedCache(self.dk, self.dv, self.dtable, self.dlen)

    def take(self, b):
        """Sequence b's keys and values on the device, in order."""
        n = self.lens[b]
        ps = self.table[b, :-(-n // self.page)]
        k, v = host(self.dk), host(self.dv)
        j = lambda a: np.concatenate([a[p] for p in ps], 1)[:, :n] if n else np.zeros((self.kv, 0, self.d))
        return j(k), j(v)


def starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


@pytest.mark.parametrize("d,H,kv,page", [(64, 4, 4, 16), (64, 6, 2, 64), (128, 5, 1, 32), (128, 4, 2, 256)])
@pytest.mark.parametrize("interleaved", [True, False])
def test_append(contexts, d, H, kv, page, interleaved):
    ctx = contexts["bf16"]
    new, past = [1, 5, 0, 70, 33], [0, 15, 9, 3, 40]
    lens = [n + p for n, p in zip(new, past)]
    P = Paged(61, lens, page, kv, d)
    T, extra = sum(new), 3
    x = synth.bf16_round(synth.normal(62, (T + extra, (H + 2 * kv) * d), 1.5))
    wq, wk, cs = 1 + synth.normal(63, (d,), 0.2), 1 + synth.normal(64, (d,), 0.2), rotations(200, d)
    q = torch.full((T + extra, H, d), 5.0, dtype=torch.bfloat16, device="cuda")
    before_k, before_v = P.dk.clone(), P.dv.clone()
    ctx.op_qk_norm_rope_append(dev(x, torch.bfloat16), q, P.cache, dev(starts(new), torch.int32), q_weight=dev(wq),
                               k_weight=dev(wk), rot=dev(cs), interleaved=interleaved)
    assert ctx.device_errors() == 0
    pos = np.concatenate([np.arange(p, p + n) for n, p in zip(new, past)])
    h = x[:T].reshape(T, H + 2 * kv, d)
    want = chunk.norm_rotate(h[:, :H], wq, 1e-6, cs, pos, interleaved)
    assert (np.abs(host(q[:T]) - want) <= norm_bound(h, wq, want, "bf16")).all()
    assert bool((q[T:] == 5.0).all())                              # rows behind the last sequence
    want_k = chunk.norm_rotate(h[:, H:H + kv], wk, 1e-6, cs, pos, interleaved)
    touched = torch.zeros(P.pages, page, dtype=torch.bool)
    t = 0
    for b, (n, p) in enumerate(zip(new, past)):
        for i in range(p, p + n):
            pg, slot = P.table[b, i // page], i % page
            touched[pg, slot] = True
            gk, gv = host(P.dk[pg, :, slot]), host(P.dv[pg, :, slot])
            assert (np.abs(gk - want_k[t]) <= norm_bound(h, wk, want_k[t], "bf16")).all()
            assert np.abs(gv - h[t, H + kv:]).max() <= 2.0 ** -25
            t += 1
    keep = ~touched.cuda()[:, None, :, None].expand_as(P.dk)       # everything else as it was, bit for bit
    assert torch.equal(P.dk.view(torch.int16)[keep], before_k.view(torch.int16)[keep])
    assert torch.equal(P.dv.view(torch.int16)[keep], before_v.view(torch.int16)[keep])


def test_append_saturates_values_beyond_fp16(contexts):
    ctx = contexts["bf16"]
    P = Paged(65, [2], 16, 1, 64)
    x = np.ones((2, 3 * 64), np.float32)
    x[0, 128], x[1, 130] = 1e6, -np.inf
    q = torch.empty(2, 1, 64, dtype=torch.bfloat16, device="cuda")
    ctx.op_qk_norm_rope_append(dev(x, torch.bfloat16), q, P.cache, dev(starts([2]), torch.int32))
    assert ctx.device_errors() == 8
    v = P.take(0)[1]
    assert v[0, 0, 0] == 65504 and v[0, 1, 2] == -65504 and v[0, 1, 3] == 1


def attend(ctx, q, P, new, frame, max_new=None, extra=0):
    T = q.shape[0]
    o = torch.full((T + extra, q.shape[1] * q.shape[2]), 5.0, dtype=torch.bfloat16, device="cuda")
    qd = torch.cat([dev(q, torch.bfloat16), torch.full((extra, *q.shape[1:]), float("nan"), dtype=torch.bfloat16, device="cuda")])
    ctx.op_attention_paged(qd, P.cache, dev(starts(new), torch.int32), o, max(new) if max_new is None else max_new, frame=frame)
    return o


def attention_bound(want, mag, keys):
    """Each probability is off by: its exponent rounded to fp16, at most 2^-9 where
    it is below 8 in size, and the fp16 exponential, 2^-9.9 (larger ones stand for
    probabilities below 2^-8, off by twice that): together below 2^-8 of it, the
    same in numerator and row sum.  What underflows is below 2^-24 a key.  One
    rounding of the result."""
    return 2.0 ** -8 * (mag + np.abs(want)) + keys * 2.0 ** -24 * 5 + HALF["bf16"] * np.abs(want) + 1e-6


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,kv", [(2, 2), (4, 1), (6, 2), (3, 1)])
@pytest.mark.parametrize("page,frame", [(16, 1), (16, 0), (32, 5), (64, 1), (128, 40), (256, 1)])
@pytest.mark.parametrize("new,past", [([1], [0]), ([1, 1, 1], [0, 63, 300]), ([3, 0, 140, 1], [5, 9, 0, 127]),
                                      ([260, 17], [250, 0])])
def test_attention_paged(contexts, d, H, kv, page, frame, new, past):
    ctx = contexts["bf16"]
    lens = [n + p for n, p in zip(new, past)]
    P = Paged(71, lens, page, kv, d)
    q = synth.bf16_round(synth.normal(72, (sum(new), H, d), 2.0))
    o = attend(ctx, q, P, new, frame, extra=2)
    assert ctx.device_errors() == 0
    want, mag = chunk.attention_paged(q, P.k, P.v, P.table, lens, starts(new), frame)
    got = host(o[:-2]).reshape(want.shape)
    assert (np.abs(got - want) <= attention_bound(want, mag, max(lens))).all()
    assert bool((o[-2:] == 5.0).all())


def test_attention_long_and_split(contexts):
    """One token over thousands of keys (many CTAs a sequence), scores that grow along the sequence."""
    ctx = contexts["bf16"]
    for d, H, kv, lens in ((128, 8, 2, [5000]), (64, 3, 3, [4097, 1, 0, 777]), (128, 48, 1, [3333])):
        P = Paged(73, lens, 64, kv, d)
        for b, n in enumerate(lens):
            for i in range(n):
                P.k[P.table[b, i // 64], :, i % 64] = synth.bf16_round(P.k[P.table[b, i // 64], :, i % 64] * np.float32(0.2 + 2.0 * i / n))
        P.dk.copy_(dev(P.k, torch.bfloat16))
        new = [min(1, n) for n in lens]
        q = synth.bf16_round(synth.normal(74, (sum(new), H, d)))
        o = attend(ctx, q, P, new, 1)
        want, mag = chunk.attention_paged(q, P.k, P.v, P.table, lens, starts(new), 1)
        assert (np.abs(host(o).reshape(want.shape) - want) <= attention_bound(want, mag, max(lens))).all()


@pytest.mark.parametrize("d,H,kv,new,past,frame", [(128, 2, 2, [60], [3000], 1), (64, 4, 1, [30, 7, 0], [2500, 40, 9], 16),     # one tile
                                                   (128, 24, 1, [5], [4000], 1), (64, 8, 4, [1, 16], [1900, 2100], 0),
                                                   (128, 3, 1, [200], [2600], 1), (64, 2, 2, [400, 90, 300], [1500, 700, 0], 50),
                                                   (128, 2, 2, [700], [0], 1), (64, 3, 3, [515, 257], [0, 300], 0)])
def test_attention_chunks_split_and_in_order(contexts, d, H, kv, new, past, frame):
    """Chunks whose keys are split, rows of one tile and of several blocks, some of them short; the longest
    blocks first, or head by head; equal calls give equal bits."""
    ctx = contexts["bf16"]
    lens = [n + p for n, p in zip(new, past)]
    P = Paged(95, lens, 32, kv, d)
    q = synth.bf16_round(synth.normal(96, (sum(new), H, d), 1.5))
    o = attend(ctx, q, P, new, frame, extra=3)
    again = attend(ctx, q, P, new, frame, extra=3)
    assert ctx.device_errors() == 0
    assert torch.equal(o.view(torch.int16), again.view(torch.int16))
    want, mag = chunk.attention_paged(q, P.k, P.v, P.table, lens, starts(new), frame)
    assert (np.abs(host(o[:-3]).reshape(want.shape) - want) <= attention_bound(want, mag, max(lens))).all()
    assert bool((o[-3:] == 5.0).all())


@pytest.mark.parametrize("lens,kv,d", [([2500] + [1 + 61 * i % 2400 for i in range(39)], 8, 128),     # longest first
                                       ([1 + 7 * i % 130 for i in range(70)], 2, 64),                 # too many to plan for
                                       ([3] * 32 + [4000] + [5, 0, 6], 1, 64),                        # one to split, past lane 31
                                       ([0] * 3 + [1] * 61, 8, 128)])
def test_attention_many_sequences(contexts, lens, kv, d):
    ctx = contexts["bf16"]
    P = Paged(89, lens, 16, kv, d, spare=0)
    new = [min(1, n) for n in lens]
    q = synth.bf16_round(synth.normal(90, (sum(new), 2 * kv, d)))
    o = attend(ctx, q, P, new, 1)
    assert ctx.device_errors() == 0
    want, mag = chunk.attention_paged(q, P.k, P.v, P.table, lens, starts(new), 1)
    assert (np.abs(host(o).reshape(want.shape) - want) <= attention_bound(want, mag, max(lens))).all()


def test_attention_rows_that_see_nothing_are_zero(contexts):
    """More new tokens than the sequence is long: those before its start see nothing (bit 2); an empty sequence too."""
    ctx = contexts["bf16"]
    for lens, new in (([3, 40], [9, 40]), ([0], [4]), ([150], [400])):
        P = Paged(75, lens, 16, 1, 64)
        q = synth.bf16_round(synth.normal(76, (sum(new), 2, 64)))
        o = attend(ctx, q, P, new, 1)
        assert ctx.device_errors() == 2
        want, mag = chunk.attention_paged(q, P.k, P.v, P.table, lens, starts(new), 1)
        got = host(o).reshape(want.shape)
        assert (got[:new[0] - lens[0]] == 0).all()
        assert (np.abs(got - want) <= attention_bound(want, mag, max(lens))).all()


def test_attention_bad_pages_and_lengths_are_reported(contexts):
    """Page numbers outside the pool read as zeros, a length beyond the table as the table's."""
    ctx = contexts["bf16"]
    P = Paged(77, [40, 20], 16, 1, 64, spare=0)
    q = synth.bf16_round(synth.normal(78, (2, 1, 64)))
    P.dtable[0, 1] = P.pages
    P.dtable[1, 0] = -1
    o = attend(ctx, q, P, [1, 1], 1)
    assert ctx.device_errors() == 2
    k, v = P.k.copy(), P.v.copy()
    k[P.table[0, 1]] = v[P.table[0, 1]] = k[P.table[1, 0]] = v[P.table[1, 0]] = 0
    want, mag = chunk.attention_paged(q, k, v, P.table, [40, 20], starts([1, 1]), 1)
    assert (np.abs(host(o).reshape(want.shape) - want) <= attention_bound(want, mag, 48)).all()
    P = Paged(79, [48], 16, 1, 64, spare=0)
    P.dlen.fill_(2 ** 31 - 1)
    o = attend(ctx, q[:1], P, [1], 1)
    assert ctx.device_errors() == 2
    want, mag = chunk.attention_paged(q[:1], P.k, P.v, P.table, [48], starts([1]), 1)
    assert (np.abs(host(o).reshape(want.shape) - want) <= attention_bound(want, mag, 48)).all()


def test_append_bad_pages_are_reported_and_skipped(contexts):
    ctx = contexts["bf16"]
    P = Paged(80, [20], 16, 1, 64, spare=0)
    before = P.dk.clone()
    P.dtable[0, 1] = P.pages + 5
    x = synth.bf16_round(synth.normal(81, (20, 3 * 64)))
    q = torch.empty(20, 1, 64, dtype=torch.bfloat16, device="cuda")
    ctx.op_qk_norm_rope_append(dev(x, torch.bfloat16), q, P.cache, dev(starts([20]), torch.int32))
    assert ctx.device_errors() == 2
    same = [p for p in range(P.pages) if p != P.table[0, 0]]
    assert torch.equal(P.dk[same].view(torch.int16), before[same].view(torch.int16))
    assert not torch.equal(P.dk[P.table[0, 0]].view(torch.int16), before[P.table[0, 0]].view(torch.int16))


def test_attention_more_new_rows_than_promised(contexts):
    ctx = contexts["bf16"]
    P = Paged(82, [700], 16, 1, 64)
    q = synth.bf16_round(synth.normal(83, (700, 1, 64)))
    o = attend(ctx, q, P, [700], 1, max_new=256)
    assert ctx.device_errors() == 2
    want, mag = chunk.attention_paged(q, P.k, P.v, P.table, [700], starts([700]), 1)
    assert (np.abs(host(o).reshape(want.shape) - want) <= attention_bound(want, mag, 700))[:256].all()
    assert bool((o[256:] == 5.0).all())


def test_attention_shared_pages(contexts):
    """Two sequences with the same first pages, and a page that a sequence's table names twice."""
    ctx = contexts["bf16"]
    P = Paged(84, [150, 170], 32, 2, 64)
    P.table[1, :3] = P.table[0, :3]
    P.table[1, 4] = P.table[1, 3]
    P.k[P.table[1, 3]], P.v[P.table[1, 3]] = 0.25, 0.5             # (both its places are filled)
    P.dtable.copy_(dev(P.table, torch.int32))
    P.dk.copy_(dev(P.k, torch.bfloat16))
    P.dv.copy_(dev(P.v, torch.half))
    q = synth.bf16_round(synth.normal(85, (12, 4, 64)))
    o = attend(ctx, q, P, [5, 7], 1)
    want, mag = chunk.attention_paged(q, P.k, P.v, P.table, [150, 170], starts([5, 7]), 1)
    assert (np.abs(host(o).reshape(want.shape) - want) <= attention_bound(want, mag, 170)).all()


def test_attention_scores_of_minus_infinity(contexts):
    """Keys whose scores are -infinity (visible ones) have no weight, however many come first; a row of nothing else is zero."""
    ctx = contexts["bf16"]
    for d, H in ((64, 2), (128, 1)):
        P = Paged(86, [300], 16, 1, d)
        for i in range(256):
            P.k[P.table[0, i // 16], 0, i % 16, 0] = -np.inf
        P.dk.copy_(dev(P.k, torch.bfloat16))
        q = synth.bf16_round(synth.normal(87, (300, H, d)))
        q[:, :, 0] = np.abs(q[:, :, 0]) + 0.5
        q[:, :, 1:] *= 8                                           # finite scores far below 0 among them
        o = attend(ctx, q, P, [300], 1)
        with np.errstate(invalid="ignore"):
            want, mag = chunk.attention_paged(q, P.k, P.v, P.table, [300], starts([300]), 1)
        got = host(o).reshape(want.shape)
        assert (got[:256] == 0).all()
        assert (np.abs(got - want) <= attention_bound(want, mag, 300)).all()


def test_two_contexts_at_once_on_streams_of_their_own(contexts):
    """Calls of two contexts overlap on two streams (given and current); each gives what it gives alone."""
    other = wdc.Context(wdc.make_config(dtype=wdc.BF16, **MODEL), 2)
    jobs = []
    for i, (ctx, lens, H) in enumerate(((contexts["bf16"], [3000, 1, 77], 8), (other, [900, 2500], 6))):
        P = Paged(88 + i, lens, 64, 2, 128)
        new = [1] * len(lens)
        q = dev(synth.normal(90 + i, (len(lens), H, 128)), torch.bfloat16)
        o = torch.zeros(len(lens), H * 128, device="cuda", dtype=torch.bfloat16)
        jobs.append((ctx, q, P, dev(starts(new), torch.int32), o))
    want = []
    for ctx, q, P, s, o in jobs:
        ctx.op_attention_paged(q, P.cache, s, o, 1)
        want.append(o.clone())
        o.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        jobs[0][0].op_attention_paged(*jobs[0][1:2], jobs[0][2].cache, jobs[0][3], jobs[0][4], 1, stream=streams[0])
        with torch.cuda.stream(streams[1]):
            jobs[1][0].op_attention_paged(*jobs[1][1:2], jobs[1][2].cache, jobs[1][3], jobs[1][4], 1)
    torch.cuda.synchronize()
    for w, j in zip(want, jobs):
        assert torch.equal(w, j[4])


# ---------------------------------------------------------------- together
def chunk_path(ctx, t, P, start, new, frame):
    """A block's attention half on a chunk: fp8 QKV projection, norms and rotation into the cache, attention, fp8 output
    projection with the gated residual."""
    f8 = torch.float8_e4m3fn
    x, T, D, H, kv, d = t["x"], t["x"].shape[0], t["x"].shape[1], t["H"], P.kv, P.d
    q8, s8 = torch.empty(T, D, device="cuda", dtype=f8), torch.empty(-(-D // 128), T, device="cuda")
    qkv = torch.empty(T, (H + 2 * kv) * d, device="cuda", dtype=torch.bfloat16)
    q, o = torch.empty(T, H, d, device="cuda", dtype=torch.bfloat16), torch.empty(T, H * d, device="cuda", dtype=torch.bfloat16)
    o8, so = torch.empty(T, H * d, device="cuda", dtype=f8), torch.empty(-(-H * d // 128), T, device="cuda")
    y = torch.empty_like(x)
    ctx.op_quantize_fp8(x, q8, s8)
    ctx.op_gemm_fp8(q8, s8, t["w"], t["sw"], qkv, bias=t["b"])
    ctx.op_qk_norm_rope_append(qkv, q, P.cache, start, q_weight=t["wq"], k_weight=t["wk"], rot=t["rot"])
    ctx.op_attention_paged(q, P.cache, start, o, max(new), frame=frame)
    ctx.op_quantize_fp8(o, o8, so)
    ctx.op_gemm_fp8(o8, so, t["wo"], t["swo"], y, res=x, gate=t["g"])
    return qkv, q, o, y


def chunk_operands(ctx, T, D, H, kv, d):
    f8 = torch.float8_e4m3fn
    N = (H + 2 * kv) * d
    t = dict(H=H, x=dev(synth.normal(91, (T, D)), torch.bfloat16), b=dev(synth.normal(92, (N,), 0.1)),
             wq=dev(1 + synth.normal(93, (d,), 0.1)), wk=dev(1 + synth.normal(94, (d,), 0.1)), rot=dev(rotations(400, d)),
             g=dev(synth.normal(95, (D,))))
    for name, rows, cols in (("w", N, D), ("wo", D, H * d)):
        w = dev(synth.normal(96, (rows, cols), cols ** -0.5), torch.bfloat16)
        t[name] = torch.empty(rows, cols, device="cuda", dtype=f8)
        t["s" + name] = torch.empty(-(-rows // 128), -(-cols // 128), device="cuda")
        ctx.op_quantize_fp8(w, t[name], t["s" + name], block_rows=128)
    return t


def test_chunks_in_turn_agree_with_one_long_one(contexts):
    """A rollout of three chunks over a growing cache against the whole sequence at once, frame by frame causal:
    each step of both from the same operands; and each step against fp64."""
    ctx = contexts["bf16"]
    D, H, kv, d, frame, sizes = 256, 4, 2, 64, 24, [48, 24, 72]
    T = sum(sizes)
    t = chunk_operands(ctx, T, D, H, kv, d)
    one = Paged(97, [T], 16, kv, d, fill=False)
    qkv, q, o, y = chunk_path(ctx, t, one, torch.tensor([0, T], dtype=torch.int32, device="cuda"), [T], frame)
    grow = Paged(98, [T], 16, kv, d, fill=False)
    got, end = [], 0
    for n in sizes:
        end += n
        grow.dlen.fill_(end)
        part = dict(t, x=t["x"][end - n:end].contiguous())
        got.append(chunk_path(ctx, part, grow, torch.tensor([0, n], dtype=torch.int32, device="cuda"), [n], frame))
    assert ctx.device_errors() == 0
    for a, b in zip((qkv, q), zip(*[g[:2] for g in got])):
        assert torch.equal(a, torch.cat(b))                # rows are independent of their neighbours
    assert torch.equal(one.dk[one.dtable[0, :9].long()], grow.dk[grow.dtable[0, :9].long()])
    # attention of the whole against fp64, and of the chunks: the same bound
    k, v = host(one.dk), host(one.dv)
    want, mag = chunk.attention_paged(host(q), k, v, one.table, [T], [0, T], frame)
    for a in (o, torch.cat([g[2] for g in got])):
        assert (np.abs(host(a).reshape(want.shape) - want) <= attention_bound(want, mag, T)).all()
    # the projection's own step against fp64 of its quantised operands
    A, sa = chunk.quantize(host(o).astype(np.float32))
    wo, swo = host(t["wo"]), t["swo"].cpu().numpy()
    proj = chunk.dequantize(A, sa, 1) @ chunk.dequantize(wo, swo, 128).T
    g64, x64 = host(t["g"]), host(t["x"])
    bound = np.abs(g64) * gemm_bound(A, sa, wo, swo, 0 * proj, "bf16") + (HALF["bf16"] + 2.0 ** -21) * np.abs(x64 + g64 * proj)
    assert (np.abs(host(y) - (x64 + g64 * proj)) <= bound + 2.0 ** -21 * np.abs(g64 * proj)).all()


def test_captured_and_replayed_on_another_stream(contexts):
    """The path captured into a graph gives the same bits as eager calls, again on new inputs in the same buffers."""
    ctx = contexts["bf16"]
    D, H, kv, d, new = 256, 6, 2, 64, [5, 1, 40]
    lens = [105, 1, 340]
    t = chunk_operands(ctx, sum(new), D, H, kv, d)
    P = Paged(99, lens, 32, kv, d)
    start = dev(starts(new), torch.int32)
    want = [a.clone() for a in chunk_path(ctx, t, P, start, new, 1)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        chunk_path(ctx, t, P, start, new, 1)
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(g, stream=s):
        got = chunk_path(ctx, t, P, start, new, 1)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    t["x"].mul_(-0.5)
    lens2 = [77, 1, 300]
    P.dlen.copy_(torch.tensor(lens2, dtype=torch.int32))
    want = [a.clone() for a in chunk_path(ctx, t, P, start, new, 1)]
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert ctx.device_errors() == 0


def test_calls_without_rows_do_nothing(contexts):
    ctx = contexts["bf16"]
    n0 = ctx.launches
    e = lambda *s, dtype=torch.bfloat16: torch.empty(*s, device="cuda", dtype=dtype)
    f8 = torch.float8_e4m3fn
    ctx.op_quantize_fp8(e(0, 64), e(0, 64, dtype=f8), e(1, 0, dtype=torch.float32))
    ctx.op_gemm_fp8(e(0, 64, dtype=f8), e(1, 0, dtype=torch.float32), e(8, 64, dtype=f8), e(1, 1, dtype=torch.float32), e(0, 8))
    ctx.op_qk_norm_rope(e(0, 3 * 64), e(1, 0, 64), e(1, 0, 64))
    P = Paged(1, [4], 16, 1, 64)
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    ctx.op_qk_norm_rope_append(e(0, 3 * 64), e(0, 1, 64), P.cache, z)
    ctx.op_attention_paged(e(0, 1, 64), P.cache, z, e(0, 64), 4)
    ctx.op_attention_paged(e(3, 1, 64), P.cache, z, e(3, 64), 0)
    assert ctx.launches == n0


def test_refusals(contexts):
    """Behind the C ABI: sizes and alignments that the operators do not take."""
    ctx, f32 = contexts["bf16"], contexts["f32"]
    f8 = torch.float8_e4m3fn
    e = lambda *s, dtype=torch.bfloat16: torch.empty(*s, device="cuda", dtype=dtype)
    one = lambda n: e(n, dtype=torch.float32)
    P = Paged(1, [4], 16, 1, 64)
    z = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    small = wdc.Context(wdc.make_config(width=64), 2)
    small_cfg_f32 = e(4, 64, dtype=torch.float32)

    def refused(status, f, *a, **k):
        with pytest.raises(wdc.WdcError) as r:
            f(*a, **k)
        assert r.value.status == status

    refused(3, ctx.op_quantize_fp8, e(4, 72), e(4, 72, dtype=f8), one(4).view(1, 4))
    refused(1, ctx.op_quantize_fp8, e(4, 80)[:, 4:68], e(4, 64, dtype=f8), one(4).view(1, 4))
    refused(1, ctx.op_quantize_fp8, e(4, 64), e(4, 64, dtype=f8), one(5)[1:].view(1, 4))
    refused(3, ctx.op_gemm_fp8, e(4, 64, dtype=f8), one(4).view(1, 4), e(12, 64, dtype=f8), one(1).view(1, 1), e(4, 12))
    refused(3, ctx.op_gemm_fp8, e(4, 72, dtype=f8), one(4).view(1, 4), e(16, 72, dtype=f8), one(1).view(1, 1), e(4, 16))
    refused(3, small.op_quantize_fp8, small_cfg_f32, e(4, 64, dtype=f8), one(4).view(1, 4))
    refused(3, ctx.op_qk_norm_rope, e(2, 3 * 32), e(1, 2, 32), e(1, 2, 32))
    refused(1, ctx.op_qk_norm_rope, e(2, 3 * 64), e(1, 2, 64), e(1, 2, 64), eps=-1.0)
    refused(1, ctx.op_qk_norm_rope, e(2, 3 * 64), e(1, 2, 64), e(1, 2, 64), rot=e(4, 4, 2, dtype=torch.float32))
    refused(1, ctx.op_qk_norm_rope, e(2, 3 * 64), e(1, 2, 64), e(1, 2, 64), rot=e(4, 40, 2, dtype=torch.float32))
    bad = wdc.PagedCache(e(3, 1, 24, 64), e(3, 1, 24, 64, dtype=torch.half), P.dtable, P.dlen)
    refused(3, ctx.op_attention_paged, e(1, 1, 64), bad, z, e(1, 64), 1)
    refused(1, ctx.op_attention_paged, e(1, 1, 64), P.cache, z, e(1, 64), -1)
    refused(1, ctx.op_attention_paged, e(1, 1, 64), P.cache, z, e(1, 64), 1, frame=-1)
    two = wdc.PagedCache(e(3, 2, 16, 64), e(3, 2, 16, 64, dtype=torch.half), P.dtable, P.dlen)
    refused(1, ctx.op_attention_paged, e(1, 3, 64), two, z, e(1, 192), 1)
    refused(3, ctx.op_attention_paged, e(1, 129, 64), P.cache, z, e(1, 129 * 64), 1)
    refused(3, f32.op_attention_paged, e(1, 1, 64, dtype=torch.float32), P.cache, z, e(1, 64, dtype=torch.float32), 1)
    with pytest.raises(ValueError):
        ctx.op_attention_paged(e(1, 1, 64, dtype=torch.float32), P.cache, z, e(1, 64), 1)
    assert ctx.device_errors() == 0
