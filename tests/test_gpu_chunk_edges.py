"""The chunk operators where their numbers come to an edge: scores of -infinity
before finite ones far below 0, sums far outside a GELU's range, tiles without
rows among tiles with some, starts and lengths that no caller should give, sizes
next to the C ABI's largest."""
import numpy as np
import pytest
import torch

from oracle import chunk
from paper_2608_01845_gb300 import synth, wdc
from test_gpu_chunk import (DTYPES, HALF, Paged, attend, attention_bound, contexts, dev, gemm_bound, gemm_case,  # noqa: F401
                            host, run_gemm, starts)

pytestmark = pytest.mark.gpu


# (one tile, whole and split; two tiles, whole and split; a group; several sequences)
@pytest.mark.parametrize("H,kv,new,past,frame", [(2, 2, [40], [260], 1), (4, 1, [1], [3100], 1), (2, 1, [300], [0], 1),
                                                 (3, 3, [300], [2900], 0), (6, 2, [1, 20, 5], [900, 2000, 0], 7),
                                                 (1, 1, [260, 140], [1100, 800], 50)])
@pytest.mark.parametrize("d", [64, 128])
def test_finite_scores_far_below_0_after_minus_infinity(contexts, d, H, kv, new, past, frame):
    """Scores of -infinity, however many steps of them, and then one near -160: the finite ones
    alone have weight.  (Taken over from a base of 0, the first sum would be 0 * 2^231.)

    The bound: a score is a sum of d products of which one is 160 sqrt(d), so each addition is off
    by at most 2^-23 of that, and the score by d 160 2^-23 < 2^-8 after its division by sqrt(d);
    a probability by as much, relatively, beside what attention_bound counts."""
    ctx = contexts["bf16"]
    lens = [n + p for n, p in zip(new, past)]
    P = Paged(101, lens, 32, kv, d)
    for b, n in enumerate(lens):
        i = np.arange(n)
        at = P.table[b, i // 32], slice(None), i % 32
        k = P.k[at]
        k[:, :, 0] = np.where(i % 197 == 150, 0, -np.inf)[:, None]
        k[:, :, 1] = synth.bf16_round(np.float32(-10.0 * np.sqrt(d)))
        P.k[at] = k
    P.dk.copy_(dev(P.k, torch.bfloat16))
    q = synth.bf16_round(synth.normal(102, (sum(new), H, d)))
    q[:, :, 0], q[:, :, 1] = 1.0, 16.0
    o = attend(ctx, q, P, new, frame)
    assert ctx.device_errors() == 0
    want, mag = chunk.attention_paged(q, P.k, P.v, P.table, lens, starts(new), frame)
    assert np.isfinite(want).all()
    got = host(o).reshape(want.shape)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= attention_bound(want, mag, max(lens)) + 2.0 ** -8 * (mag + np.abs(want))).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("resid", [False, True])
def test_warps_without_rows_among_tiles_with_some(contexts, resid, kind):
    """One block of K, several tiles a pair, and in the last row block most warps without a row: each tile
    gets its own columns' bias and gate."""
    ctx, (M, N, K) = contexts[kind], (4 * 256 + 5, 8200, 128)
    A, sa, W, sw = gemm_case(51, M, N, K, kind)
    n = np.arange(N, dtype=np.float32)
    b, g = 1000 + n, 2.0 - n / 4096                                # (a neighbour's would be far off)
    y = chunk.dequantize(A, sa, 1) @ chunk.dequantize(W, sw, 128).T + b
    err = gemm_bound(A, sa, W, sw, 0 * y, kind) + 2.0 ** -22 * np.abs(y)
    C, kw = torch.zeros(M, N, dtype=DTYPES[kind], device="cuda"), dict(bias=dev(b))
    if resid:
        kw.update(res=C, gate=dev(g))
        y, err = g * y, np.abs(g) * err + 2.0 ** -22 * np.abs(g * y)
    run_gemm(ctx, A, sa, W, sw, C, **kw)
    assert ctx.device_errors() == 0
    assert (np.abs(host(C) - y) <= err + HALF[kind] * np.abs(y) + 2.0 ** -22 * np.abs(y)).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("resid", [False, True])
@pytest.mark.parametrize("M,N", [(12, 264), (1029, 8200)])             # narrow kernel, pair kernel
def test_gelu_far_from_0(contexts, M, N, resid, kind):
    """GELU(x) is x, or 0, from 8 on: below -8 it is smaller than 8 * 2^-60 (tanh form: 2^-70 x), above 8
    nearer to x than 2^-18.  Sums up to 1e20 in size, whichever kernel the number of rows brings."""
    sizes = np.float32([8, 30, 1e3, 1e6, 1e10, 1e20])
    x = sizes[np.arange(M) % len(sizes)]
    A, W = np.ones((M, 128)), np.ones((N, 128)) * np.where(np.arange(N) % 3 == 0, 1, -1)[:, None]
    C, kw = torch.zeros(M, N, dtype=DTYPES[kind], device="cuda"), {}
    if resid:
        kw["res"] = C
    run_gemm(contexts[kind], A, (x / 128)[None], W, np.ones((-(-N // 128), 1)), C, gelu=True, **kw)
    got, up = host(C), np.arange(N) % 3 == 0
    assert (np.abs(got[:, ~up]) <= 2.0 ** -57).all()
    assert (np.abs(got[:, up] - x[:, None]) <= (2.0 ** -18 + HALF[kind]) * x[:, None]).all()


@pytest.mark.parametrize("start,lens,ok", [([0, 2, 3], [40, 20], True), ([1, 1, 3], [40, 20], True), ([0, 0, 0], [0, 0], True),
                                           ([-1, 2, 3], [40, 20], False), ([0, 2, 4], [40, 20], False), ([2, 1, 3], [40, 20], False),
                                           ([0, 5, 3], [40, 20], False), ([2 ** 31 - 1] * 3, [40, 20], False),
                                           ([0, 3, 2 ** 31 - 1], [40, 20], False), ([-2 ** 31, 0, 3], [40, 20], False),
                                           ([0, 3, 3], [40, -1], False), ([0, 0, 3], [10 ** 6, 20], False), ([0, 0, 3], [40, 2], False)])
def test_starts_and_lengths_out_of_range_are_reported(contexts, start, lens, ok):
    """Those of a sequence without new tokens too; what lies behind the T rows stays as it is."""
    ctx, T = contexts["bf16"], 3
    P = Paged(103, [48, 48], 16, 2, 64, spare=0)
    P.dlen.copy_(torch.tensor(lens, dtype=torch.int32))
    s = torch.tensor(start, dtype=torch.int64).to(torch.int32).cuda()
    q = dev(synth.normal(104, (T, 4, 64)), torch.bfloat16)
    o = torch.full((T + 4, 4 * 64), 5.0, dtype=torch.bfloat16, device="cuda")
    ctx.op_attention_paged(q, P.cache, s, o[:T], T, frame=1)
    assert ctx.device_errors() == (0 if ok else 2)
    assert bool((o[T:] == 5.0).all())
    x = dev(synth.normal(105, (T, 8 * 64)), torch.bfloat16)
    out = torch.full((T + 4, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    ctx.op_qk_norm_rope_append(x, out[:T], P.cache, s)
    assert ctx.device_errors() == (0 if ok else 2)
    assert bool((out[T:] == 5.0).all())
    spare = [p for p in range(P.pages) if p not in set(P.table.reshape(-1).tolist())]
    assert torch.equal(P.dk[spare].view(torch.int16), dev(P.k, torch.bfloat16)[spare].view(torch.int16))


def test_every_sequence_is_looked_at(contexts):
    """One bad length among many sequences, most without new tokens, wherever it is."""
    ctx, B = contexts["bf16"], 75
    P = Paged(106, [16] * B, 16, 1, 64, spare=0)
    q, x = dev(synth.normal(107, (1, 1, 64)), torch.bfloat16), dev(synth.normal(108, (1, 3 * 64)), torch.bfloat16)
    o, s = torch.empty(1, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(B + 1, dtype=torch.int32, device="cuda")
    s[0] = 0
    for b in (None, 0, 1, 31, 32, 63, 64, 74):
        P.dlen.fill_(16)
        if b is not None:
            P.dlen[b] = 17
        ctx.op_attention_paged(q, P.cache, s, o, 1)
        assert ctx.device_errors() == (0 if b is None else 2)
        ctx.op_qk_norm_rope_append(x, q.clone(), P.cache, s)
        assert ctx.device_errors() == (0 if b is None else 2)


def test_widths_that_tiles_would_take_past_an_int(contexts):
    """Refused before anything is launched: rounded up to whole blocks they are negative."""
    ctx, f8 = contexts["bf16"], torch.float8_e4m3fn
    x, q, s = (torch.empty(1, 256, device="cuda", dtype=t) for t in (torch.bfloat16, f8, torch.float32))
    at, n0 = [t.data_ptr() for t in (x, q, s)], ctx.launches
    stream = torch.cuda.current_stream().cuda_stream
    for big in (2 ** 31 - 496, 2 ** 31 - 16):
        for rows in (1, 128):
            assert wdc.LIB.wdc_op_quantize_fp8(ctx._h, at[0], big, at[1], at[2], 1, big, rows, stream) == 3
        for N, K in ((8, big), (big, 16), (big, big)):
            assert wdc.LIB.wdc_op_gemm_fp8(ctx._h, at[1], at[2], at[1], at[2], None, at[0], 1, N, K, 0, None, None, stream) == 3
    assert ctx.launches == n0


@pytest.mark.parametrize("new,past", [([1], [1500]), ([200], [30]), ([300], [1700])])
@pytest.mark.parametrize("d,key", [(64, 2.0 ** 16.5), (128, 2.0 ** 17)])
def test_scores_near_the_largest(contexts, d, key, new, past):
    """Two kinds of keys with scores of about 2^26.5 and minus that: the mean over the first kind's values,
    of equal probabilities, so that an error of theirs drops out."""
    ctx = contexts["bf16"]
    lens = [n + p for n, p in zip(new, past)]
    P = Paged(109, lens, 32, 2, d)
    for b, n in enumerate(lens):
        i = np.arange(n)
        k = np.zeros((n, 2, d), np.float32)
        k[:, :, 1] = synth.bf16_round(np.where(i % 3 == 0, key, -key).astype(np.float32))[:, None]
        P.k[P.table[b, i // 32], :, i % 32] = k
    P.dk.copy_(dev(P.k, torch.bfloat16))
    q = np.zeros((sum(new), 4, d), np.float32)
    q[:, :, 1] = 2.0 ** 13
    o = attend(ctx, q, P, new, 1)
    want, mag = chunk.attention_paged(q, P.k, P.v, P.table, lens, starts(new), 1)
    assert (np.abs(host(o).reshape(want.shape) - want) <= attention_bound(want, mag, max(lens))).all()
