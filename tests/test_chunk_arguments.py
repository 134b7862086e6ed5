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


def test_sizes_beyond_an_int(ctx, monkeypatch):
    """What the C ABI's ints would cut off is refused, or (max_new, frame) means what a smaller one does."""
    f, m = torch.float32, lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device="meta")
    big = 2 ** 32 + 1
    with pytest.raises(ValueError, match="a size of"):
        ctx.op_quantize_fp8(m(big, 16), m(big, 16, dtype=F8), m(1, big, dtype=f))
    with pytest.raises(ValueError, match="a size of"):
        ctx.op_gemm_fp8(m(big, 16, dtype=F8), m(1, big, dtype=f), m(8, 16, dtype=F8), m(1, 1, dtype=f), m(big, 8))
    with pytest.raises(ValueError, match="a size of"):
        ctx.op_qk_norm_rope(m(big, 3 * 64), m(1, big, 64), m(1, big, 64))
    with pytest.raises(ValueError, match="a size of"):
        ctx.op_qk_norm_rope_append(m(big, 3 * 64), m(big, 1, 64), cache(), e(2, dtype=I32))
    with pytest.raises(ValueError, match="a size of"):
        ctx.op_attention_paged(m(big, 1, 64), cache(), e(2, dtype=I32), m(big, 64), 1)
    with pytest.raises(ValueError, match="a size of"):
        wdc.PagedCache(m(3, 1, 16, 64), m(3, 1, 16, 64, dtype=torch.half), m(1, big, dtype=I32), m(1, dtype=I32))
    seen = []
    monkeypatch.setattr(wdc.LIB, "wdc_op_attention_paged", lambda *a: seen.append(a[6:8]) or 0)
    monkeypatch.setattr(ctx, "_op_stream", lambda s: 0)
    for new, frame in [(2 ** 32 + 2, 2 ** 32), (-2 ** 32, 2 ** 31), (3, -2 ** 32)]:
        ctx.op_attention_paged(e(5, 2, 64), cache(), e(2, dtype=I32), e(5, 128), new, frame=frame)
    assert seen == [(5, 2 ** 31 - 1), (-1, 2 ** 31 - 1), (3, -1)]


@pytest.mark.parametrize("cname,struct", [("wdc_paged_cache", "PagedCacheC"), ("wdc_head_norm", "HeadNorm")])
def test_struct_layout_matches_a_c_compiler(tmp_path, cname, struct):
    import ctypes
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    s = getattr(wdc, struct)
    names = [n for n, _ in s._fields_]
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "wdc.h"\nint main(void) {'
                   + "".join(f'printf("%zu ", offsetof({cname}, {n}));' for n in names)
                   + f'printf("%zu", sizeof({cname})); return 0; }}')
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(s, n).offset for n in names] + [ctypes.sizeof(s)]


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


def test_heads_and_angles_beyond_an_int(ctx, monkeypatch):
    """A head's size, a block's rows, the positions and the pairs of the angles are ints of the C ABI as well."""
    f, m = torch.float32, lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device="meta")
    big = 2 ** 32 + 64
    monkeypatch.setattr(wdc.LIB, "wdc_op_qk_norm_rope", lambda *a: pytest.fail("called"))
    monkeypatch.setattr(wdc.LIB, "wdc_op_qk_norm_rope_append", lambda *a: pytest.fail("called"))
    monkeypatch.setattr(ctx, "_op_stream", lambda s: 0)
    monkeypatch.setattr(wdc.LIB, "wdc_op_quantize_fp8", lambda *a: pytest.fail("called"))
    for rows in (2 ** 32 + 1, 1 - 2 ** 32, 2 ** 32 + 128):         # (1 or 128 once cut off)
        for scale in (e(1, 1, dtype=f), e(1, 4, dtype=f)):
            with pytest.raises(ValueError):
                ctx.op_quantize_fp8(e(4, 64), e(4, 64, dtype=F8), scale, block_rows=rows)
    good = dict(qkv=e(5, 4 * 64), q=e(2, 5, 64), k=e(1, 5, 64))
    app = dict(qkv=e(5, 4 * 64), q=e(5, 2, 64), cache=cache(), q_start=e(2, dtype=I32))
    with pytest.raises(ValueError, match="a size of"):
        ctx.op_qk_norm_rope(m(1, 3 * big), m(1, 1, big), m(1, 1, big))
    for rot in (m(big, 16, 2, dtype=f), m(1, 2 ** 31 + 8, 2, dtype=f), m(1, 2 ** 30 + 8, 2, dtype=f)):
        with pytest.raises(ValueError, match="a size of"):
            ctx.op_qk_norm_rope(**good, rot=rot)
        with pytest.raises(ValueError, match="a size of"):
            ctx.op_qk_norm_rope_append(**app, rot=rot)
