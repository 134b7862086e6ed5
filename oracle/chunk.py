"""Chunk operators in fp64 from their definitions: e4m3 blocks, the product of
two such matrices, head norms with rotation, and attention over a paged cache."""
import numpy as np

E4M3_MAX = 448.0
BLOCK = 128


def e4m3_round(y):
    """Nearest e4m3 value (3 bits after the point, exponents from -6, ties to even), saturated."""
    y = np.asarray(y, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(y))), -6.0)
        e = np.where(y == 0, -6.0, e)
        step = np.exp2(e - 3)
        return np.clip(np.round(y / step) * step, -E4M3_MAX, E4M3_MAX)


def quantize(x, block_rows=1):
    """(values, scales): IEEE fp32 division for scale and quotient, as the operator defines them."""
    x = np.asarray(x, np.float32)
    M, K = x.shape
    mb, kb = -(-M // block_rows), -(-K // BLOCK)
    p = np.zeros((mb * block_rows, kb * BLOCK), np.float32)
    p[:M, :K] = x
    p = p.reshape(mb, block_rows, kb, BLOCK)
    s = (np.abs(p).max((1, 3)) / np.float32(E4M3_MAX)).astype(np.float32)
    with np.errstate(invalid="ignore"):
        q = p / np.where(s == 0, np.float32(1), s)[:, None, :, None]
    q = e4m3_round(q).reshape(mb * block_rows, kb * BLOCK)[:M, :K]
    return q, (s.T.copy() if block_rows == 1 else s)


def dequantize(q, s, block_rows):
    """Values times scales, in fp64 (scales laid out as quantize gives them)."""
    M, K = q.shape
    s = np.asarray(s, np.float64)
    s = s.T if block_rows == 1 else s
    return np.asarray(q, np.float64) * s.repeat(block_rows, 0)[:M].repeat(BLOCK, 1)[:, :K]


def norm_rotate(x, w, eps, rot, pos, interleaved):
    """x [T, heads, d]: RMS norm over d times w, then the first 2 * rot.shape[1] elements
    turned by rot[pos] (cos, sin)."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if w is not None:
        y = y * np.asarray(w, np.float64)
    if rot is None:
        return y
    half = rot.shape[1]
    cs = np.asarray(rot, np.float64)[pos][:, None]
    c, s = cs[..., 0], cs[..., 1]
    out = y.copy()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def limits(n, L, frame):
    """Tokens that each of a chunk's n tokens, the last of L, sees."""
    p = L - n + np.arange(n)
    if frame == 0:
        return np.full(n, L)
    return np.where(p < 0, 0, np.minimum(L, (p // frame + 1) * frame))


def attention_paged(q, k, v, table, length, start, frame):
    """q [T, heads, d] over pages k, v [pages, kv, page, d]; rows that no sequence owns are NaN.
    Also returns sum p |v| / sum p of each element, for error bounds."""
    T, H, d = q.shape
    kv, page = k.shape[1], k.shape[2]
    G = H // kv
    out, mag = np.full((T, H, d), np.nan), np.full((T, H, d), np.nan)
    for b in range(len(length)):
        n, L = start[b + 1] - start[b], length[b]
        rows = slice(start[b], start[b + 1])
        lim = limits(n, L, frame)
        pages = [table[b][i] for i in range(-(-L // page))]
        for g in range(kv):
            kk = np.concatenate([k[p, g] for p in pages])[:L].astype(np.float64) if L else np.zeros((0, d))
            vv = np.concatenate([v[p, g] for p in pages])[:L].astype(np.float64) if L else np.zeros((0, d))
            for h in range(g * G, (g + 1) * G):
                s = np.asarray(q[rows, h], np.float64) @ kk.T / np.sqrt(d)
                hide = np.arange(L)[None] >= lim[:, None]
                s = np.where(hide, -np.inf, s)
                top = s.max(1, initial=-np.inf, keepdims=True)
                e = np.exp(s - np.where(np.isfinite(top), top, 0.0))
                l = e.sum(1, keepdims=True)
                p = e / np.where(l == 0, 1.0, l)
                out[rows, h], mag[rows, h] = p @ vv, p @ np.abs(vv)
    return out, mag
