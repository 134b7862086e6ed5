"""What the binding of the chunk operators refuses before the library is called:
types, shapes, strides and devices (CPU only: no context is created)."""
import numpy as np
import pytest
import torch

from oracle import chunk
from paper_2608_01845_gb300 import wdc

F8, BF, I32 = torch.float8_e4m3fn, torch.bfloat16, torch.int32


@pytest.fixture
def ctx(monkeypatch):
    c = wdc.Context.__new__(wdc.Context)
    c.cfg, c.device, c._h = wdc.make_config(layers=1, dtype=wdc.BF16), 0, None
    monkeypatch.setattr(c, "_operand_types", lambda: (BF, -1, F8, torch.float32, I32))
    return c


def e(*shape, dtype=BF):
    return torch.empty(*shape, dtype=dtype)


def cache(page=16, kv=1, d=64, B=1):
    return wdc.PagedCache(e(3, kv, page, d), e(3, kv, page, d, dtype=torch.half), e(B, 2, dtype=I32), e(B, dtype=I32))


def test_quantize_and_gemm(ctx):
    f = torch.float32
    for x, q, s, rows in [(e(4, 64, dtype=f), e(4, 64, dtype=F8), e(1, 4, dtype=f), 1),
                          (e(4, 64), e(4, 64, dtype=torch.uint8), e(1, 4, dtype=f), 1),
                          (e(4, 64), e(4, 64, dtype=F8), e(4, 1, dtype=f), 1),
                          (e(4, 64), e(4, 64, dtype=F8), e(1, 4, dtype=f), 128),
                          (e(64, 4).t(), e(4, 64, dtype=F8), e(1, 4, dtype=f), 1),
                          (e(4, 64), e(8, 64, dtype=F8)[::2], e(1, 4, dtype=f), 1), (e(4), e(4, dtype=F8), e(1, 4, dtype=f), 1)]:
        with pytest.raises(ValueError):
            ctx.op_quantize_fp8(x, q, s, block_rows=rows)
    good = dict(A=e(4, 64, dtype=F8), a_scale=e(1, 4, dtype=f), W=e(8, 64, dtype=F8), w_scale=e(1, 1, dtype=f), C=e(4, 8))
    for bad in [dict(A=e(4, 64)), dict(W=e(8, 80, dtype=F8)), dict(a_scale=e(4, 1, dtype=f)), dict(w_scale=e(1, 2, dtype=f)),
                dict(C=e(4, 8, dtype=f)), dict(bias=e(4, dtype=f)), dict(res=e(8, 4)), dict(gate=e(8)),
                dict(C=e(8, 4).t())]:
        with pytest.raises(ValueError):
            ctx.op_gemm_fp8(**dict(good, **bad))


def test_norm_and_attention(ctx):
    f = torch.float32
    good = dict(qkv=e(5, 4 * 64), q=e(2, 5, 64), k=e(1, 5, 64))
    for bad in [dict(qkv=e(5, 5 * 64)), dict(k=e(1, 4, 64)), dict(vt=e(1, 64, 8)), dict(vt=e(1, 64, 5, dtype=torch.half)),
                dict(q_weight=e(64)), dict(k_weight=e(32, dtype=f)), dict(rot=e(5, 32, dtype=f)), dict(rot=e(5, 32, 2)),
                dict(positions=e(5, dtype=torch.int64)), dict(positions=e(4, dtype=I32)), dict(q=e(5, 64))]:
        with pytest.raises(ValueError):
            ctx.op_qk_norm_rope(**dict(good, **bad))
    good = dict(qkv=e(5, 4 * 64), q=e(5, 2, 64), cache=cache(), q_start=e(2, dtype=I32))
    for bad in [dict(cache=cache(d=128)), dict(cache=cache(kv=2)), dict(q_start=e(3, dtype=I32)), dict(q=e(4, 2, 64)),
                dict(q_start=e(2, dtype=torch.int64))]:
        with pytest.raises(ValueError):
            ctx.op_qk_norm_rope_append(**dict(good, **bad))
    good = dict(q=e(5, 2, 64), cache=cache(), q_start=e(2, dtype=I32), o=e(5, 128), max_new=5)
    for bad in [dict(o=e(5, 64)), dict(q=e(5, 2, 64, dtype=f)), dict(cache=cache(d=128)), dict(q_start=e(1, dtype=I32))]:
        with pytest.raises(ValueError):
            ctx.op_attention_paged(**dict(good, **bad))


def test_cache_tensors():
    k, v, t, n = e(3, 1, 16, 64), e(3, 1, 16, 64, dtype=torch.half), e(2, 4, dtype=I32), e(2, dtype=I32)
    for a in [(k.float(), v, t, n), (k, v.float(), t, n), (k, v[:2], t, n), (k, v, t.long(), n), (k, v, t, n[:1]),
              (k, v, t[:, ::2], n), (k[0], v, t, n), (k.transpose(1, 2), v, t, n)]:
        with pytest.raises(ValueError):
            wdc.PagedCache(*a)
    c = wdc.PagedCache(k, v, t, n).c
    assert (c.pages, c.page, c.kv_heads, c.head_dim, c.sequences, c.table_width) == (3, 16, 1, 64, 2, 4)


def test_null_context_is_refused():
    n, c = wdc.HeadNorm(), wdc.PagedCacheC()
    import ctypes
    L, N = wdc.LIB, None
    assert L.wdc_op_quantize_fp8(N, N, 0, N, N, 1, 16, 1, N) == 1
    assert L.wdc_op_gemm_fp8(N, N, N, N, N, N, N, 1, 8, 16, 0, N, N, N) == 1
    assert L.wdc_op_qk_norm_rope(N, N, 0, 1, 1, 1, 64, ctypes.byref(n), N, N, N, N) == 1
    assert L.wdc_op_qk_norm_rope_append(N, N, 0, 1, 1, ctypes.byref(n), ctypes.byref(c), N, N, N) == 1
    assert L.wdc_op_attention_paged(N, N, ctypes.byref(c), N, 1, 1, 1, 1, N, N) == 1


def test_oracle_rounds_to_the_format():
    """The oracle's e4m3 against torch's conversion, over values of every exponent, ties and saturation included."""
    x = np.concatenate([np.linspace(-500, 500, 20001), np.exp2(np.linspace(-14, 9, 5000)), np.arange(0, 64) / 1024.0, [0.0]])
    want = torch.from_numpy(x).float().clamp(-448, 448).to(F8).double().numpy()
    assert np.array_equal(chunk.e4m3_round(x.astype(np.float32)), want)


def test_oracle_attention_of_a_dense_cache():
    """One page that holds the whole sequence, all of it visible: plain softmax attention."""
    r = np.random.default_rng(0)
    q, k, v = r.standard_normal((6, 2, 8)), r.standard_normal((1, 1, 6, 8)), r.standard_normal((1, 1, 6, 8))
    o, _ = chunk.attention_paged(q, k, v, [[0]], [6], [0, 6], 0)
    for h in range(2):
        s = q[:, h] @ k[0, 0].T / np.sqrt(8)
        p = np.exp(s) / np.exp(s).sum(1, keepdims=True)
        assert np.allclose(o[:, h], p @ v[0, 0])
    assert list(chunk.limits(4, 6, 1)) == [3, 4, 5, 6] and list(chunk.limits(4, 6, 4)) == [4, 4, 6, 6]
    assert list(chunk.limits(4, 2, 1)) == [0, 0, 1, 2]
