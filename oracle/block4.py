"""A block in four bits, in fp64 from the definitions: e2m1 rows with scales, the
products of such matrices, the residual's norm, and rotation by several axes."""
import numpy as np

from oracle import chunk, dit

PIECE = 512
ROW = np.float32(1) / np.float32(2688)


def e2m1_round(y):
    """Nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (one bit after the point, exponents from 0; ties to even), saturated."""
    y = np.asarray(y, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(y))), 0.0)
        step = np.exp2(np.where(y == 0, 0.0, e) - 1)
        return np.clip(np.round(y / step) * step, -6, 6)


def quantize(x):
    """(values of the codes [M, K], scales [M, K / 16], row scales [M]), every intermediate an fp32 number."""
    x = np.asarray(x, np.float32)
    M, K = x.shape
    f, b = np.float32, x.reshape(M, K // 16, 16)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(1)
        row = np.where(np.isfinite(top), np.where(top < f(2.0 ** -100), f(0), top * ROW), f(np.nan))
        live = row > 0
        t = np.abs(b).max(2) / np.where(live, f(6) * row, f(1))[:, None]
        s = np.where(live[:, None], chunk.e4m3_round(t), 0).astype(f)
        step = s * np.where(live, row, f(0))[:, None]
        by = np.where(step > 0, f(1) / np.where(step > 0, step, f(1)), f(0))
        y = np.where(live[:, None, None], b * by[:, :, None], f(0))
    return e2m1_round(y).reshape(M, K), s, row


def values(code, s, row):
    """What the codes stand for, in fp64."""
    return code * np.asarray(s, np.float64).repeat(16, 1) * np.asarray(row, np.float64)[:, None]


def pack(code):
    """[M, K / 2] bytes, the even column in the low four bits."""
    levels = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    c = np.searchsorted(levels, np.abs(code)).astype(np.uint8) + 8 * (np.asarray(code) < 0).astype(np.uint8)
    return c[:, ::2] | c[:, 1::2] << 4


def unpack(b):
    levels = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    levels = np.concatenate([levels, -levels])
    out = np.empty((b.shape[0], 2 * b.shape[1]))
    out[:, ::2], out[:, 1::2] = levels[b & 15], levels[b >> 4]
    return out


def places(M, n):
    """Indices [M, n] of the scales in pieces [ceil(M / 128), n / 4, 512]."""
    r, j = np.arange(M)[:, None], np.arange(n)[None]
    return r // 128, j // 4, r % 32 * 16 + r // 32 % 4 * 4 + j % 4


def to_pieces(s, fill=0.0):
    M, n = s.shape
    p = np.full((-(-M // 128), n // 4, PIECE), fill)
    p[places(M, n)] = s
    return p


def from_pieces(p, M):
    return np.asarray(p)[places(M, 4 * p.shape[1])]


def silu(x):
    return x / (1 + np.exp(-x))


def gated(g, u, gelu):
    return (dit.gelu_tanh(g) if gelu else silu(g)) * u


def add_norm(x, delta=None, gate=None, weight=None, offset=0.0, shift=None, center=False, eps=1e-6, rows_per_set=0):
    """(sum, result) in fp64; gate, weight and shift [sets, D]."""
    x = np.asarray(x, np.float64)
    pick = (lambda v: np.asarray(v, np.float64)[np.arange(len(x)) // rows_per_set if rows_per_set else np.zeros(len(x), int)])
    r = x if delta is None else x + (1.0 if gate is None else pick(gate)) * np.asarray(delta, np.float64)
    c = r - r.mean(1, keepdims=True) if center else r
    y = c / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    if weight is not None:
        y = y * (pick(weight) + offset)
    if shift is not None:
        y = y + pick(shift)
    return r, y


def axes_table(tables, coords):
    """cos and sin [T, all pairs, 2] of each token, section by section."""
    return np.concatenate([t[c] for t, c in zip(tables, np.asarray(coords).T)], 1)
