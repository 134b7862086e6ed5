"""Workloads of the operators that roll a model out chunk by chunk.

What a block does with the tokens of a new chunk, over a cache of the tokens
before them:

* ``quantize``  rows of activations (or 128 x 128 blocks of a weight) to e4m3
  with a scale for each block of 128 (``op_quantize_fp8``);
* ``gemm``      the product of two such matrices, with the epilogues of
  ``op_gemm`` (``op_gemm_fp8``);
* ``rotate``    the norms of queries and keys for each head and their rotation
  by position in one pass: into the operands of ``op_attention``
  (``op_qk_norm_rope``) or with keys and values appended to a paged cache
  (``op_qk_norm_rope_append``);
* ``attend``    the chunk's attention over that cache (``op_attention_paged``).

Where ``own`` is false ``run`` computes them from elementary torch operations
in 32 bits, rounded once at the end; where it is true it calls the framework.
``exact`` restates them in 64 bits.
"""
import math
import random

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0


def listed():
    return [
        # one new token for each of four streams, few heads: all latency
        dict(name="rotate_token", kind="rotate", form="append", dtype="bf16", heads=16, kv=4, d=64, rot=64, pairs=True,
             B=4, new=1, past=2000, ragged=True, page=16, mix=1),
        # one frame (30 x 45 tokens) of the 5B-scale model onto twelve frames of history
        dict(name="rotate_frame", kind="rotate", form="append", dtype="bf16", heads=48, kv=48, d=64, rot=64, pairs=True,
             B=1, new=1350, past=16200, ragged=False, page=64, mix=2),
        # a whole clip of the 5B-scale model's length for the dense attention, heads of 128, half-split pairs
        dict(name="rotate_clip", kind="rotate", form="dense", dtype="bf16", heads=24, kv=24, d=128, rot=128, pairs=False,
             B=1, new=17776, past=0, ragged=False, page=0, mix=3),
        # a frame and its 226 condition tokens, before a projection
        dict(name="quantize_frame", kind="quantize", dtype="bf16", M=1576, K=3072, rows=1),
        # the MLP's hidden rows of a 3-frame clip in fp32
        dict(name="quantize_hidden_f32", kind="quantize", dtype="f32", M=4276, K=12288, rows=1),
        # four single tokens through a QKV projection: the weights' bytes
        dict(name="gemm_token", kind="gemm", dtype="bf16", M=4, N=9216, K=3072, mode="store"),
        # a frame's MLP down-projection with the gated residual
        dict(name="gemm_frame", kind="gemm", dtype="bf16", M=1350, N=3072, K=12288, mode="resid"),
        # a whole clip's MLP up-projection
        dict(name="gemm_clip", kind="gemm", dtype="bf16", M=17776, N=12288, K=3072, mode="gelu"),
        # eight streams, one token each, up to 32k of history, four queries to a key head: the cache's bytes
        dict(name="attend_token", kind="attend", heads=32, kv=8, d=128, B=8, new=1, past=32767, ragged=True, page=64,
             frame=1, mix=4),
        # one frame onto twelve frames of history, each token sees its whole frame (5B-scale heads)
        dict(name="attend_frame", kind="attend", heads=48, kv=48, d=64, B=1, new=1350, past=16200, ragged=False, page=64,
             frame=1350, mix=5),
        # six streams with chunks of different lengths and odd ends, three queries to a key head, small pages
        dict(name="attend_ragged", kind="attend", heads=12, kv=4, d=128, B=6, new=701, past=5003, ragged=True, page=16,
             frame=1, mix=6),
        # two prompts from nothing, causal
        dict(name="attend_prompt", kind="attend", heads=24, kv=24, d=128, B=2, new=6001, past=0, ragged=False, page=128,
             frame=1, mix=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "quantize", "gemm", "attend"])
    if kind == "quantize":
        K = 16 * _log(rng, 8, 768)
        return dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), M=min(_log(rng, 1, 20000), (1 << 25) // K), K=K,
                    rows=rng.choice([1, 1, 1, 128]))
    if kind == "gemm":
        N, K = 8 * _log(rng, 16, 1536), 16 * _log(rng, 8, 768)
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                    M=min(_log(rng, 1, 16384), int(5e11 // (N * K))), N=N, K=K, mode=rng.choice(["store", "gelu", "resid"]))
    d = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 2, 3, 4, 6] if kv < 8 else [1, 2, 4])
    if kind == "rotate":
        form, pairs = rng.choice(["dense", "append", "append"]), rng.random() < 0.5
        dtype = "f32" if form == "dense" and rng.random() < 0.5 else "bf16"
        c = dict(kind=kind, form=form, dtype=dtype, heads=heads, kv=kv, d=d, rot=rng.choice([d, d, 32, d - 16]), pairs=pairs)
        if form == "dense":
            return dict(c, B=1, new=_log(rng, 1, 16384), past=0, ragged=False, page=0, mix=0)
        return dict(c, B=rng.randint(1, 6), new=_log(rng, 1, 2500), past=_log(rng, 1, 8000) - 1, ragged=rng.random() < 0.6,
                    page=rng.choice([16, 32, 64, 128]), mix=rng.randint(0, 9999))
    B, new, past = rng.randint(1, 8), rng.choice([1, _log(rng, 1, 3000)]), _log(rng, 1, 32000) - 1
    while B > 1 and B * heads * new * (new + past) > 1 << 30:
        B -= 1
    while heads * new * (new + past) > 1 << 30:
        past //= 2
        new = max(1, new * 3 // 4)
    return dict(kind=kind, heads=heads, kv=kv, d=d, B=B, new=new, past=past, ragged=B > 1 and rng.random() < 0.7,
                page=rng.choice([16, 32, 64, 128]), frame=rng.choice([0, 1, 1, rng.randint(2, 400)]), mix=rng.randint(0, 9999))


# ---------------------------------------------------------------- inputs
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt) % (1 << 62))


def _randn(seed, salt, *shape, std=1.0):
    t = torch.randn(*shape, device="cuda", generator=_gen(seed, salt))
    return t if std == 1.0 else t.mul_(std)


def _dtype(c):
    return torch.float32 if c.get("dtype") == "f32" else torch.bfloat16


def _lengths(c):
    """New and earlier tokens of each sequence."""
    r = random.Random(c["mix"])
    new, past = [c["new"]] * c["B"], [c["past"]] * c["B"]
    if c["ragged"]:
        new = [new[0]] + [r.randint(1, n) for n in new[1:]]
        past = [past[0]] + [r.randint(0, p) for p in past[1:]]
    return new, past


def _ceil(a, b):
    return -(-a // b)


def _activations(c, seed, salt, M, K, dtype):
    """Rows as a norm leaves them, with a few wide channels and one row of zeros in 64."""
    x = _randn(seed, salt, M, K)
    x *= torch.exp(_randn(seed, salt + 1, K, std=0.5))
    x *= (torch.arange(M, device="cuda") % 64 != 63)[:, None]
    return x.to(dtype)


def _to_e4m3(x):
    """Blocks of 128 x 128 of a weight in e4m3 and their scales."""
    N, K = x.shape
    nb, kb = _ceil(N, BLOCK), _ceil(K, BLOCK)
    p = torch.nn.functional.pad(x, (0, kb * BLOCK - K, 0, nb * BLOCK - N)).view(nb, BLOCK, kb, BLOCK)
    s = p.abs().amax((1, 3)) / E4M3_MAX
    q = (p / s[:, None, :, None]).nan_to_num_(0.0).view(nb * BLOCK, kb * BLOCK)[:N, :K]
    return q.to(torch.float8_e4m3fn).contiguous(), s


def _rows_to_e4m3(x):
    M, K = x.shape
    kb = _ceil(K, BLOCK)
    p = torch.nn.functional.pad(x.float(), (0, kb * BLOCK - K)).view(M, kb, BLOCK)
    s = p.abs().amax(2) / E4M3_MAX
    q = (p / s[:, :, None]).nan_to_num_(0.0).view(M, kb * BLOCK)[:, :K]
    return q.to(torch.float8_e4m3fn).contiguous(), s.t().contiguous()


def _gemm_inputs(c, seed):
    M, N, K = c["M"], c["N"], c["K"]
    A, sa = _rows_to_e4m3(_activations(c, seed, 1, M, K, torch.bfloat16))
    W, sw = _to_e4m3(_randn(seed, 3, N, K, std=K ** -0.5))
    bias = _randn(seed, 4, N, std=0.1)
    res = gate = None
    if c["mode"] == "resid":
        res, gate = _randn(seed, 5, M, N).to(_dtype(c)), _randn(seed, 6, N)
    return A, sa, W, sw, bias, res, gate


def _rotations(c, positions):
    """cos and sin of every position: a third of the pairs turn with the frame, the rest with row and column."""
    half = c["rot"] // 2
    p = torch.arange(positions, device="cuda", dtype=torch.float64)
    axes = torch.stack([p // 1350, p % 1350 // 45, p % 45])
    i = torch.arange(half, device="cuda")
    a = axes[i % 3].t() * 10000.0 ** (-(i // 3 * 3).double() / max(half, 1))
    return torch.stack([a.cos(), a.sin()], -1).float()


def _paging(c, seed, new, past):
    """A page table in random order, with a few pages that belong to nobody."""
    width = max(_ceil(n + p, c["page"]) for n, p in zip(new, past)) + 1
    total = c["B"] * width + 3
    order = torch.randperm(total, device="cuda", generator=_gen(seed, 90))[:c["B"] * width]
    length = torch.tensor([n + p for n, p in zip(new, past)], device="cuda", dtype=torch.int32)
    start = torch.tensor([sum(new[:b]) for b in range(c["B"] + 1)], device="cuda", dtype=torch.int32)
    return order.view(c["B"], width).int().contiguous(), total, length, start


def _pool(c, seed, pages):
    k = _randn(seed, 91, pages, c["kv"], c["page"], c["d"]).bfloat16()
    v = _randn(seed, 92, pages, c["kv"], c["page"], c["d"]).half()
    return k, v


def _rotate_inputs(c, seed, new):
    T, H, kv, d = sum(new), c["heads"], c["kv"], c["d"]
    qkv = _randn(seed, 1, T, (H + 2 * kv) * d, std=1.5).to(_dtype(c))
    return qkv, 1 + _randn(seed, 2, d, std=0.1), 1 + _randn(seed, 3, d, std=0.1)


_contexts = {}


def _context(dtype):
    """The program's context: one model of the type, as small as it gets."""
    if dtype not in _contexts:
        from paper_2608_01845_gb300 import wdc
        _contexts[dtype] = wdc.Context(wdc.make_config(
            layers=1, hidden=256, heads=4, head_dim=64, mlp=256, temb_dim=256, freq_dim=256, in_ch=16, frames=1, height=16,
            width=16, patch=2, cond_tokens=16, cond_dim=64, dtype=wdc.F32 if dtype == torch.float32 else wdc.BF16), 2)
    return _contexts[dtype]


def prepare(case, seed):
    c, kind = case, case["kind"]
    s = {"case": c}
    if kind == "quantize":
        s["x"] = _activations(c, seed, 1, c["M"], c["K"], _dtype(c))
        s["q"] = torch.empty(c["M"], c["K"], device="cuda", dtype=torch.float8_e4m3fn)
        kb = _ceil(c["K"], BLOCK)
        s["scale"] = torch.empty((kb, c["M"]) if c["rows"] == 1 else (_ceil(c["M"], BLOCK), kb), device="cuda")
    elif kind == "gemm":
        s["A"], s["sa"], s["W"], s["sw"], s["bias"], s["res"], s["gate"] = _gemm_inputs(c, seed)
        s["C"] = torch.empty(c["M"], c["N"], device="cuda", dtype=_dtype(c))
    else:
        new, past = _lengths(c)
        T = sum(new)
        if kind == "rotate":
            s["qkv"], s["wq"], s["wk"] = _rotate_inputs(c, seed, new)
            s["rot"] = _rotations(c, max(n + p for n, p in zip(new, past)))
        else:
            s["q"] = _randn(seed, 1, T, c["heads"], c["d"]).bfloat16()
            s["o"] = torch.empty(T, c["heads"] * c["d"], device="cuda", dtype=torch.bfloat16)
        if c["page"]:
            s["table"], pages, s["length"], s["start"] = _paging(c, seed, new, past)
            s["k"], s["v"] = _pool(c, seed, pages)
            if kind == "rotate":
                s["q"] = torch.empty(T, c["heads"], c["d"], device="cuda", dtype=torch.bfloat16)
        else:
            dt, ldv = _dtype(c), _ceil(T, 8) * 8 if c["dtype"] == "bf16" else T
            s["q"] = torch.empty(c["heads"], T, c["d"], device="cuda", dtype=dt)
            s["k"] = torch.empty(c["kv"], T, c["d"], device="cuda", dtype=dt)
            s["vt"] = torch.zeros(c["kv"], c["d"], ldv, device="cuda", dtype=torch.half if c["dtype"] == "bf16" else dt)
    if own:
        from paper_2608_01845_gb300 import wdc
        s["ctx"] = _context(_dtype(c))
        if c.get("page"):
            s["cache"] = wdc.PagedCache(s["k"], s["v"], s["table"], s["length"])
    return s


# ---------------------------------------------------------------- run
def _gelu(x):
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


def _plain_quantize(s):
    x, c = s["x"].float(), s["case"]
    M, K = x.shape
    kb, rows = s["scale"].shape[1 if c["rows"] != 1 else 0], c["rows"]
    mb = _ceil(M, rows)
    p = torch.nn.functional.pad(x, (0, kb * BLOCK - K, 0, mb * rows - M)).view(mb, rows, kb, BLOCK)
    scale = p.abs().amax((1, 3)) / E4M3_MAX
    q = p / torch.where(scale > 0, scale, 1.0)[:, None, :, None]
    q = q.clamp(-E4M3_MAX, E4M3_MAX).view(mb * rows, kb * BLOCK)[:M, :K].to(torch.float8_e4m3fn)
    return {"q": q, "scale": scale.t().contiguous() if rows == 1 else scale}


def _plain_gemm(s):
    c = s["case"]
    k = torch.arange(c["K"], device="cuda") // BLOCK
    n = torch.arange(c["N"], device="cuda") // BLOCK
    A = s["A"].float() * s["sa"].t()[:, k]
    W = s["W"].float() * s["sw"][n][:, k]
    y = A @ W.t() + s["bias"]
    if c["mode"] == "gelu":
        y = _gelu(y)
    elif c["mode"] == "resid":
        y = s["res"].float() + s["gate"] * y
    return y.to(s["C"].dtype)


def _plain_norm_rotate(x, w, rot, pos, pairs):
    """x [T, heads, d] in 32 bits: RMS norm over d, then the first rot dimensions turned by their position's angles."""
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
    cs, half = rot[pos][:, None], rot.shape[1]
    cos, sin = cs[..., 0], cs[..., 1]
    if pairs:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., 2 * half:]], -1)


def _plain_rotate(s):
    c = s["case"]
    T, H, kv, d = s["qkv"].shape[0], c["heads"], c["kv"], c["d"]
    x = s["qkv"].float().view(T, H + 2 * kv, d)
    t = torch.arange(T, device="cuda")
    if c["form"] == "append":
        b = torch.searchsorted(s["start"], t.int(), right=True) - 1
        pos = s["length"][b] - (s["start"][b + 1] - s["start"][b]) + t - s["start"][b]
        pos = pos.long()
    else:
        pos = t
    q = _plain_norm_rotate(x[:, :H], s["wq"], s["rot"], pos, c["pairs"]).to(_dtype(c))
    k = _plain_norm_rotate(x[:, H:H + kv], s["wk"], s["rot"], pos, c["pairs"]).to(_dtype(c))
    v = x[:, H + kv:].to(torch.half if c["dtype"] == "bf16" else torch.float32)
    if c["form"] == "append":
        page = s["table"][b, pos // c["page"]].long()
        s["k"][page, :, pos % c["page"]] = k
        s["v"][page, :, pos % c["page"]] = v
        return {"q": q, "k": s["k"], "v": s["v"]}
    s["vt"][:, :, :T] = v.permute(1, 2, 0)
    return {"q": q.transpose(0, 1).contiguous(), "k": k.transpose(0, 1).contiguous(), "vt": s["vt"]}


def _plain_attend(s):
    c = s["case"]
    H, kv, d, B, G = c["heads"], c["kv"], c["d"], c["B"], c["heads"] // c["kv"]
    T, new, longest = s["q"].shape[0], c["new"], c["new"] + c["past"]
    start, length = s["start"].long(), s["length"].long()
    count = start[1:] - start[:-1]
    i, j = torch.arange(new, device="cuda"), torch.arange(longest, device="cuda")
    # the cache's keys and values of each sequence, zeros behind its end
    page = s["table"][:, j // c["page"]].long()
    there = (j < length[:, None])[:, :, None, None]
    k = torch.where(there, s["k"][page, :, j % c["page"]].float(), 0.0).permute(0, 2, 3, 1)
    v = torch.where(there, s["v"][page, :, j % c["page"]].float(), 0.0).transpose(1, 2)
    row = (start[:-1, None] + i).clamp(max=T - 1)
    q = s["q"][row].float().view(B, new, kv, G, d).permute(0, 2, 3, 1, 4).reshape(B, kv, G * new, d)
    pos = (length - count)[:, None] + i
    seen = length[:, None] if c["frame"] == 0 else torch.minimum(length[:, None], (pos // c["frame"] + 1) * c["frame"])
    hide = (j >= seen.expand(B, new)[:, :, None])[:, None, None]
    x = (q @ k).mul_(d ** -0.5).view(B, kv, G, new, longest)
    x.masked_fill_(hide, -math.inf)
    p = x.sub_(x.amax(-1, keepdim=True)).exp_()
    o = (p.view(B, kv, G * new, longest) @ v).view(B, kv, G, new, d) / p.sum(-1, keepdim=True)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, new, H * d)[i < count[:, None]]
    return o.bfloat16()


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if not own:
        return {"quantize": _plain_quantize, "gemm": _plain_gemm, "rotate": _plain_rotate, "attend": _plain_attend}[kind](s)
    ctx = s["ctx"]
    if kind == "quantize":
        ctx.op_quantize_fp8(s["x"], s["q"], s["scale"], block_rows=c["rows"])
        return {"q": s["q"], "scale": s["scale"]}
    if kind == "gemm":
        ctx.op_gemm_fp8(s["A"], s["sa"], s["W"], s["sw"], s["C"], bias=s["bias"], gelu=c["mode"] == "gelu", res=s["res"],
                        gate=s["gate"])
        return s["C"]
    if kind == "rotate":
        kw = dict(q_weight=s["wq"], k_weight=s["wk"], eps=1e-6, rot=s["rot"], interleaved=c["pairs"])
        if c["form"] == "append":
            ctx.op_qk_norm_rope_append(s["qkv"], s["q"], s["cache"], s["start"], **kw)
            return {"q": s["q"], "k": s["k"], "v": s["v"]}
        ctx.op_qk_norm_rope(s["qkv"], s["q"], s["k"], vt=s["vt"], **kw)
        return {"q": s["q"], "k": s["k"], "vt": s["vt"]}
    ctx.op_attention_paged(s["q"], s["cache"], s["start"], s["o"], max_new=c["new"], frame=c["frame"])
    return s["o"]


# ---------------------------------------------------------------- work
def _seen(c):
    """Visible (query, key) pairs of one head, over all sequences."""
    total, F = 0, c["frame"]
    for n, p in zip(*_lengths(c)):
        L = n + p
        if F == 0:
            total += n * L
        else:
            total += sum(min(L, (x // F + 1) * F) for x in range(p, L))
    return total


def work(case):
    c, kind = case, case["kind"]
    es = 4 if c.get("dtype") == "f32" else 2
    if kind == "quantize":
        M, K = c["M"], c["K"]
        return {"bytes": (es + 1) * M * K + 4 * _ceil(M, c["rows"]) * _ceil(K, BLOCK), "flops": 3 * M * K}
    if kind == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        kb = _ceil(K, BLOCK)
        return {"bytes": M * K + N * K + es * M * N * (2 if c["mode"] == "resid" else 1) + 4 * kb * (M + _ceil(N, BLOCK)),
                "flops": 2 * M * N * K}
    new, past = _lengths(c)
    T, H, kv, d = sum(new), c["heads"], c["kv"], c["d"]
    if kind == "rotate":
        n = T * (H + 2 * kv) * d
        return {"bytes": 2 * es * n + 4 * c["rot"] * T, "flops": 8 * n}
    keys = sum(new) + sum(past)
    return {"bytes": 4 * T * H * d + 4 * keys * kv * d, "flops": 4 * d * H * _seen(c)}


# ---------------------------------------------------------------- 64 bits
def _e4m3(y):
    """The nearest value of the format (3 bits after the point, exponents from -6), ties to even."""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))).clamp(min=-6.0)
    step = torch.exp2(e - 3)
    return (torch.round(y / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantize(c, seed):
    x = _activations(c, seed, 1, c["M"], c["K"], _dtype(c)).double()
    R, (M, K) = c["rows"], x.shape
    q, scale = torch.empty_like(x), torch.empty(_ceil(M, R), _ceil(K, BLOCK), device="cuda", dtype=torch.float64)
    for j in range(scale.shape[1]):
        part = x[:, j * BLOCK:(j + 1) * BLOCK]
        top = part.abs().amax(1)
        if R != 1:
            top = torch.cat([t.amax().expand(t.shape[0]) for t in top.split(R)])
        step = top / E4M3_MAX
        q[:, j * BLOCK:(j + 1) * BLOCK] = _e4m3(part / torch.where(step == 0, 1.0, step)[:, None])
        scale[:, j] = step[::R]
    return {"q": q, "scale": scale.t().contiguous() if R == 1 else scale}


def _exact_gemm(c, seed):
    A, sa, W, sw, bias, res, gate = _gemm_inputs(c, seed)
    y = torch.zeros(c["M"], c["N"], device="cuda", dtype=torch.float64)
    wide = sw.double().repeat_interleave(BLOCK, 0)[:c["N"]]
    for j in range(sa.shape[0]):
        k = slice(j * BLOCK, (j + 1) * BLOCK)
        y += (A[:, k].double() * sa[j].double()[:, None]) @ (W[:, k].double() * wide[:, j:j + 1]).t()
    y += bias.double()
    if c["mode"] == "gelu":
        y = y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return y if res is None else res.double() + gate.double() * y


def _exact_turn(x, w, cs, pairs):
    """x [T, heads, d] in 64 bits; cs [T, rot / 2, 2]."""
    y = x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * w.double()
    out, half = y.clone(), cs.shape[1]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
        c, s = cs[:, None, i, 0].double(), cs[:, None, i, 1].double()
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return out


def _exact_rotate(c, seed):
    new, past = _lengths(c)
    H, kv, d = c["heads"], c["kv"], c["d"]
    qkv, wq, wk = _rotate_inputs(c, seed, new)
    rot = _rotations(c, max(n + p for n, p in zip(new, past)))
    x = qkv.double().view(-1, H + 2 * kv, d)
    at = torch.cat([torch.arange(p, p + n, device="cuda") for n, p in zip(new, past)])
    q, k = _exact_turn(x[:, :H], wq, rot[at], c["pairs"]), _exact_turn(x[:, H:H + kv], wk, rot[at], c["pairs"])
    v = x[:, H + kv:]
    if c["form"] == "dense":
        T = x.shape[0]
        vt = torch.zeros(kv, d, _ceil(T, 8) * 8 if c["dtype"] == "bf16" else T, device="cuda", dtype=torch.float64)
        vt[:, :, :T] = v.permute(1, 2, 0)
        return {"q": q.transpose(0, 1), "k": k.transpose(0, 1), "vt": vt}
    table, pages, _, _ = _paging(c, seed, new, past)
    pk, pv = (t.double() for t in _pool(c, seed, pages))
    t0 = 0
    for b, (n, p) in enumerate(zip(new, past)):
        for g in range(p // c["page"], _ceil(n + p, c["page"])):
            lo, hi = max(p, g * c["page"]), min(n + p, (g + 1) * c["page"])
            rows, slots = slice(t0 + lo - p, t0 + hi - p), slice(lo - g * c["page"], hi - g * c["page"])
            pk[table[b, g], :, slots] = k[rows].transpose(0, 1)
            pv[table[b, g], :, slots] = v[rows].transpose(0, 1)
        t0 += n
    return {"q": q, "k": pk, "v": pv}


def _exact_attend(c, seed):
    new, past = _lengths(c)
    H, kv, d, P, F = c["heads"], c["kv"], c["d"], c["page"], c["frame"]
    table, pages, _, _ = _paging(c, seed, new, past)
    K, V = _pool(c, seed, pages)
    q = _randn(seed, 1, sum(new), H, d).bfloat16()
    out, t0 = torch.empty(sum(new), H, d, device="cuda", dtype=torch.float64), 0
    for b, (n, p) in enumerate(zip(new, past)):
        L = n + p
        used = table[b, :_ceil(L, P)].long()
        at = torch.arange(p, L, device="cuda")
        last = torch.full_like(at, L) if F == 0 else ((at // F + 1) * F).clamp(max=L)
        for g in range(kv):
            k = K[used, g].reshape(-1, d)[:L].double()
            v = V[used, g].reshape(-1, d)[:L].double()
            for h in range(g * (H // kv), (g + 1) * (H // kv)):
                x = q[t0:t0 + n, h].double() @ k.t() / math.sqrt(d)
                x = torch.where(torch.arange(L, device="cuda") < last[:, None], x, -math.inf)
                out[t0:t0 + n, h] = torch.softmax(x, -1) @ v
        t0 += n
    return out.reshape(sum(new), H * d)


def exact(case, seed):
    c = case
    return {"quantize": _exact_quantize, "gemm": _exact_gemm, "rotate": _exact_rotate, "attend": _exact_attend}[c["kind"]](c, seed)
