"""Workloads of the operators of a chunk's block in four bits.

Between a chunk's attention and its projections a block adds a branch to the
residual, normalises and modulates it and hands it on in few bits; the products
then run in four bits, the MLP's with a gate, and the heads of a video are turned by
frame, row and column:

* ``quantize``  rows to e2m1 with an e4m3 scale for 16 columns and an fp32 scale for
  a row, and their values read back (``op_quantize_fp4``, ``op_dequantize_fp4``);
* ``gemm``      the product of two such matrices, with the epilogues of ``op_gemm``
  (``op_gemm_fp4``);
* ``gated``     a gated MLP's first half: both projections, the activation and their
  product (``op_gated_fp4``);
* ``norm``      the residual's sum, its root-mean-square or layer norm and modulation,
  in the model's type or in e4m3 with a scale for 128 columns (``op_add_norm``);
* ``rotate``    the norms of queries and keys and their rotation by a position of
  several axes, for the dense attention or appended to a paged cache
  (``op_qk_norm_rope``, ``op_qk_norm_rope_append`` with ``axes``).

Where ``own`` is false ``run`` computes them from elementary torch operations in 32
bits, rounded once at the end; where it is true it calls the framework.  ``exact``
restates them in 64 bits.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0
ROW = 1.0 / 2688                       # a row's scale of its largest magnitude: 6 * 448 steps
TINY = 2.0 ** -100                     # rows below it become zero
EPS = 1e-6


def listed():
    return [
        # four single tokens before a projection: all latency
        dict(name="quantize_token", kind="quantize", dtype="bf16", M=4, K=5120),
        # the MLP's hidden rows of a 3-frame clip in fp32
        dict(name="quantize_hidden_f32", kind="quantize", dtype="f32", M=4276, K=12288),
        # four single tokens through a QKV projection: the weights' bytes
        dict(name="gemm_token", kind="gemm", dtype="bf16", M=4, N=15360, K=5120, mode="store"),
        # a frame's MLP down-projection with the gated residual
        dict(name="gemm_frame", kind="gemm", dtype="bf16", M=1350, N=4096, K=16384, mode="resid"),
        # a whole clip's MLP up-projection
        dict(name="gemm_clip", kind="gemm", dtype="bf16", M=17776, N=16384, K=4096, mode="gelu"),
        # one token of each of three streams through a gated MLP
        dict(name="gated_token", kind="gated", dtype="bf16", M=3, N=13824, K=5120, act="silu"),
        # a frame and its 226 condition tokens through a gated MLP
        dict(name="gated_frame", kind="gated", dtype="bf16", M=1576, N=10240, K=4096, act="silu"),
        # four single tokens between a block's halves
        dict(name="norm_token", kind="norm", dtype="bf16", M=4, D=5120, center=False, add=True, mod=0, out="e4m3"),
        # three frames, each at its own noise level: layer norm, modulation and gate by frame
        dict(name="norm_frames", kind="norm", dtype="bf16", M=4050, D=4096, center=True, add=True, mod=1350, out="e4m3"),
        # a whole clip's rows, root-mean-square norm, for a bf16 projection
        dict(name="norm_clip", kind="norm", dtype="bf16", M=17776, D=5120, center=False, add=True, mod=0, out="same"),
        # one frame (30 x 45 tokens) onto twelve frames of history, heads of 128, pairs by frame, row and column
        dict(name="rotate_frame", kind="rotate", form="append", dtype="bf16", heads=24, kv=24, d=128, pairs="22,21,21",
             inter=True, B=1, new=1350, past=16200, page=64, mix=1),
        # a whole clip for the dense attention, heads of 64, half-split pairs
        dict(name="rotate_clip", kind="rotate", form="dense", dtype="bf16", heads=48, kv=48, d=64, pairs="12,10,10",
             inter=False, B=1, new=17776, past=0, page=0, mix=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "gemm", "gated", "norm", "rotate"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "quantize":
        K = 64 * _log(rng, 1, 256)
        return dict(kind=kind, dtype=dtype, M=min(_log(rng, 1, 20000), (1 << 25) // K), K=K)
    if kind in ("gemm", "gated"):
        N, K = 8 * _log(rng, 1, 2048), 64 * _log(rng, 1, 256)
        c = dict(kind=kind, dtype=dtype, M=min(_log(rng, 1, 17776), int(5e11 // (N * K))), N=N, K=K)
        return dict(c, mode=rng.choice(["store", "gelu", "resid"])) if kind == "gemm" else dict(c, act=rng.choice(["silu", "gelu"]))
    if kind == "norm":
        D = 16 * _log(rng, 4, 1024)
        M = min(_log(rng, 1, 20000), (1 << 25) // D)
        return dict(kind=kind, dtype=dtype, M=M, D=D, center=rng.random() < 0.5, add=rng.random() < 0.7,
                    mod=rng.choice([0, 0, rng.randint(1, M)]), out=rng.choice(["same", "e4m3"]))
    d, inter = rng.choice([64, 128]), rng.random() < 0.5
    kv = rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 2, 3, 4, 6] if kv < 8 else [1, 2, 4])
    rot = rng.choice([d, d, 48, d - 16]) // 2
    cut = sorted(rng.sample(range(rot + 1), rng.choice([1, 2, 2, 3])))
    pairs = ",".join(str(b - a) for a, b in zip([0] + cut, cut + [rot]))
    form = rng.choice(["dense", "append"])
    c = dict(kind=kind, form=form, dtype=dtype if form == "dense" else "bf16", heads=heads, kv=kv, d=d, pairs=pairs, inter=inter)
    if form == "dense":
        return dict(c, B=1, new=_log(rng, 1, 16384), past=0, page=0, mix=rng.randint(0, 9999))
    return dict(c, B=rng.randint(1, 6), new=_log(rng, 1, 2500), past=_log(rng, 1, 8000) - 1, page=rng.choice([16, 32, 64, 128]),
                mix=rng.randint(0, 9999))


# ---------------------------------------------------------------- inputs
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt) % (1 << 62))


def _randn(seed, salt, *shape, std=1.0):
    t = torch.randn(*shape, device="cuda", generator=_gen(seed, salt))
    return t if std == 1.0 else t.mul_(std)


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _ceil(a, b):
    return -(-a // b)


def _activations(c, seed, salt, M, K):
    """Rows as a block leaves them, with a few wide channels and one row of zeros in 64."""
    x = _randn(seed, salt, M, K)
    x *= torch.exp(_randn(seed, salt + 1, K, std=0.5))
    x *= (torch.arange(M, device="cuda") % 64 != 63)[:, None]
    return x.to(_dtype(c))


# Scales of 16 columns lie in pieces of 512 bytes, one for 128 rows and 64 columns:
# row r % 32, row r / 32 of 4, column block of 4.
def _to_pieces(s):
    M, n = s.shape
    mb = _ceil(M, 128)
    p = torch.nn.functional.pad(s.float(), (0, 0, 0, mb * 128 - M)).view(mb, 4, 32, n // 4, 4)
    return p.permute(0, 3, 2, 1, 4).reshape(mb, n // 4, 512).to(torch.float8_e4m3fn)


def _from_pieces(p, M):
    mb, n, _ = p.shape
    return p.float().view(mb, n, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(mb * 128, n * 4)[:M]


def _e2m1_codes(y):
    """0..7 for the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (ties to the even code), + 8 where y is below 0."""
    a = y.abs()
    code = (y < 0).to(torch.uint8) * 8
    for level, tie in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += a >= level if tie else a > level
    return code


def _levels():
    half = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return torch.tensor(half + [-v for v in half], device="cuda")


def _rows_to_fp4(x):
    """x [M, K] in 32 bits: codes [M, K], scales [M, K / 16] (values of e4m3), scale of each row."""
    M, K = x.shape
    top = x.abs().amax(1)
    row = torch.where(top < TINY, 0.0, top * ROW)
    b = x.view(M, K // 16, 16)
    s = (b.abs().amax(2) / torch.where(row > 0, 6.0 * row, 1.0)[:, None]).clamp(max=E4M3_MAX).to(torch.float8_e4m3fn).float()
    s = torch.where(row > 0, s.t(), 0.0).t()
    step = s * row[:, None]
    code = _e2m1_codes(b * torch.where(step > 0, 1.0 / step, 0.0)[:, :, None])
    return code.view(M, K), s, row


def _pack(code):
    return (code[:, 0::2] | code[:, 1::2] << 4).contiguous()


def _unpack(packed):
    return torch.stack([packed & 15, packed >> 4], -1).flatten(1).long()


def _fp4(x):
    code, s, row = _rows_to_fp4(x.float())
    return _pack(code), _to_pieces(s), row


def _matrix(c, seed, salt, rows):
    if salt == 1:
        return _fp4(_activations(c, seed, 1, rows, c["K"]))
    return _fp4(_randn(seed, salt, rows, c["K"], std=c["K"] ** -0.5))


def _gemm_inputs(c, seed):
    s = {"A": _matrix(c, seed, 1, c["M"]), "W": _matrix(c, seed, 3, c["N"]), "bias": _randn(seed, 4, c["N"], std=0.1)}
    if c["kind"] == "gated":
        s["U"], s["up_bias"] = _matrix(c, seed, 7, c["N"]), _randn(seed, 8, c["N"], std=0.1)
    elif c["mode"] == "resid":
        s["res"], s["gate"] = _randn(seed, 5, c["M"], c["N"]).to(_dtype(c)), _randn(seed, 6, c["N"])
    return s


def _norm_inputs(c, seed):
    M, D = c["M"], c["D"]
    sets = _ceil(M, c["mod"]) if c["mod"] else 1
    s = {"x": _activations(c, seed, 1, M, D), "weight": _randn(seed, 3, sets, D, std=0.2)}
    if c["center"]:
        s["shift"] = _randn(seed, 4, sets, D, std=0.2)
    if c["add"]:
        s["delta"], s["gate"] = _randn(seed, 5, M, D).to(_dtype(c)), _randn(seed, 6, sets, D, std=0.5)
    return s


def _pairs(c):
    return [int(n) for n in c["pairs"].split(",")]


def _counts(c):
    """New and earlier tokens of each sequence."""
    r = random.Random(c["mix"])
    return ([c["new"]] + [r.randint(1, c["new"]) for _ in range(c["B"] - 1)],
            [c["past"]] + [r.randint(0, c["past"]) for _ in range(c["B"] - 1)])


def _axes(c, new, past):
    """A table of cos and sin for each axis, and the place of each token on each: frame, row and column
    of 30 x 45 tokens, and for a fourth axis the sequence."""
    pairs = _pairs(c)
    at = torch.cat([torch.arange(p, p + n, device="cuda") for n, p in zip(new, past)])
    seq = torch.cat([torch.full((n,), b, device="cuda") for b, n in enumerate(new)])
    place = torch.stack([at // 1350, at % 1350 // 45, at % 45, seq][:len(pairs)], 1)
    tables = []
    for a, n in enumerate(pairs):
        rows = [max(x + y for x, y in zip(new, past)) // 1350 + 1, 30, 45, len(new)][a]
        f = 10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / max(n, 1))
        t = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * f
        tables.append(torch.stack([t.cos(), t.sin()], -1).float())
    return tables, place.int().contiguous()


def _heads(c, seed, new):
    d = c["d"]
    qkv = _randn(seed, 1, sum(new), (c["heads"] + 2 * c["kv"]) * d, std=1.5).to(_dtype(c))
    return qkv, 1 + _randn(seed, 2, d, std=0.1), 1 + _randn(seed, 3, d, std=0.1)


def _paging(c, seed, new, past):
    """A page table in random order, with a few pages that belong to nobody; the pool's old contents."""
    width = max(_ceil(n + p, c["page"]) for n, p in zip(new, past)) + 1
    total = c["B"] * width + 3
    table = torch.randperm(total, device="cuda", generator=_gen(seed, 90))[:c["B"] * width].view(c["B"], width).int()
    length = torch.tensor([n + p for n, p in zip(new, past)], device="cuda", dtype=torch.int32)
    start = torch.tensor([sum(new[:b]) for b in range(c["B"] + 1)], device="cuda", dtype=torch.int32)
    k = _randn(seed, 91, total, c["kv"], c["page"], c["d"]).bfloat16()
    v = _randn(seed, 92, total, c["kv"], c["page"], c["d"]).half()
    return table, length, start, k, v


_contexts = {}


def _context(dtype):
    """The program's context: one model of the type, as small as it gets."""
    if dtype not in _contexts:
        from paper_2608_01845_gb300 import wdc
        _contexts[dtype] = wdc.Context(wdc.make_config(
            layers=1, hidden=256, heads=4, head_dim=64, mlp=256, temb_dim=256, freq_dim=256, in_ch=16, frames=1, height=16,
            width=16, patch=2, cond_tokens=16, cond_dim=64, dtype=wdc.F32 if dtype == torch.float32 else wdc.BF16), 2)
    return _contexts[dtype]


def _empty(c, *shape, dtype=None):
    return torch.empty(*shape, device="cuda", dtype=dtype or _dtype(c))


def prepare(case, seed):
    c, kind = case, case["kind"]
    s = {"case": c}
    if kind == "quantize":
        M, K = c["M"], c["K"]
        s["x"] = _activations(c, seed, 1, M, K)
        s["Q"] = (_empty(c, M, K // 2, dtype=torch.uint8), _empty(c, _ceil(M, 128), K // 64, 512, dtype=torch.float8_e4m3fn),
                  _empty(c, M, dtype=torch.float32))
        s["back"] = _empty(c, M, K)
    elif kind in ("gemm", "gated"):
        s.update(_gemm_inputs(c, seed))
        s["C"] = _empty(c, c["M"], c["N"])
    elif kind == "norm":
        s.update(_norm_inputs(c, seed))
        s["sum"] = _empty(c, c["M"], c["D"])
        s["out"] = _empty(c, c["M"], c["D"], dtype=torch.float8_e4m3fn if c["out"] == "e4m3" else None)
        s["scale"] = _empty(c, _ceil(c["D"], 128), c["M"], dtype=torch.float32)
    else:
        new, past = _counts(c)
        T = sum(new)
        s["qkv"], s["wq"], s["wk"] = _heads(c, seed, new)
        s["tables"], s["place"] = _axes(c, new, past)
        if c["form"] == "append":
            s["table"], s["length"], s["start"], s["k"], s["v"] = _paging(c, seed, new, past)
            s["q"] = _empty(c, T, c["heads"], c["d"])
        else:
            bf16 = c["dtype"] == "bf16"
            s["q"], s["k"] = _empty(c, c["heads"], T, c["d"]), _empty(c, c["kv"], T, c["d"])
            s["vt"] = torch.zeros(c["kv"], c["d"], _ceil(T, 8) * 8 if bf16 else T, device="cuda", dtype=torch.half if bf16 else None)
    if own:
        from paper_2608_01845_gb300 import wdc
        s["ctx"] = _context(_dtype(c))
        for name in "QAWU":
            if name in s:
                s[name] = wdc.Fp4Matrix(*s[name])
        if kind == "rotate":
            s["axes"] = wdc.RotAxes(s["tables"], s["place"])
            if c["form"] == "append":
                s["cache"] = wdc.PagedCache(s["k"], s["v"], s["table"], s["length"])
    return s


# ---------------------------------------------------------------- run
def _gelu(x):
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


def _plain_quantize(s):
    x = s["x"].float()
    code, scale, row = _rows_to_fp4(x)
    step = scale * row[:, None]
    back = _levels()[code.long()].view(*scale.shape, 16) * step[:, :, None]
    return {"back": back.view(x.shape).to(s["x"].dtype), "scale": _to_pieces(scale), "row": row}


def _values(m):
    packed, pieces, row = m
    v = _levels()[_unpack(packed)]
    return (v.view(v.shape[0], -1, 16) * (_from_pieces(pieces, v.shape[0]) * row[:, None])[:, :, None]).view(v.shape)


def _plain_gemm(s):
    c = s["case"]
    y = _values(s["A"]) @ _values(s["W"]).t() + s["bias"]
    if c["mode"] == "gelu":
        y = _gelu(y)
    elif c["mode"] == "resid":
        y = s["res"].float() + s["gate"] * y
    return y.to(s["C"].dtype)


def _plain_gated(s):
    a = _values(s["A"])
    g, u = a @ _values(s["W"]).t() + s["bias"], a @ _values(s["U"]).t() + s["up_bias"]
    return ((g / (1 + torch.exp(-g)) if s["case"]["act"] == "silu" else _gelu(g)) * u).to(s["C"].dtype)


def _plain_norm(s):
    c = s["case"]
    m = torch.arange(c["M"], device="cuda") // c["mod"] if c["mod"] else torch.zeros(c["M"], device="cuda", dtype=torch.long)
    x = s["x"].float()
    if c["add"]:
        x = x + s["gate"][m] * s["delta"].float()
    r = {"sum": x.to(_dtype(c))} if c["add"] else {}
    if c["center"]:
        x = x - x.mean(1, keepdim=True)
    y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * (1 + s["weight"][m])
    if c["center"]:
        y = y + s["shift"][m]
    if c["out"] == "same":
        return dict(r, out=y.to(_dtype(c)))
    M, D = y.shape
    p = torch.nn.functional.pad(y, (0, _ceil(D, 128) * 128 - D)).view(M, -1, 128)
    scale = p.abs().amax(2) / E4M3_MAX
    q = (p / torch.where(scale > 0, scale, 1.0)[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(M, -1)[:, :D]
    return dict(r, out=q.to(torch.float8_e4m3fn), scale=scale.t().contiguous())


def _plain_turn(x, w, cs, inter):
    """x [T, heads, d] in 32 bits: root-mean-square norm over d, then its first pairs turned by cs [T, pairs, 2]."""
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    n, cos, sin = cs.shape[1], cs[:, None, :, 0], cs[:, None, :, 1]
    if inter:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., 2 * n:]], -1)


def _plain_rotate(s):
    c = s["case"]
    T, H, kv, d = s["qkv"].shape[0], c["heads"], c["kv"], c["d"]
    x = s["qkv"].float().view(T, H + 2 * kv, d)
    cs = torch.cat([t[p.long()] for t, p in zip(s["tables"], s["place"].t())], 1)
    q = _plain_turn(x[:, :H], s["wq"], cs, c["inter"]).to(_dtype(c))
    k = _plain_turn(x[:, H:H + kv], s["wk"], cs, c["inter"]).to(_dtype(c))
    v = x[:, H + kv:].to(torch.half if c["dtype"] == "bf16" else torch.float32)
    if c["form"] == "append":
        t = torch.arange(T, device="cuda")
        b = torch.searchsorted(s["start"], t.int(), right=True) - 1
        at = (s["length"][b] - (s["start"][b + 1] - s["start"][b]) + t - s["start"][b]).long()
        page = s["table"][b, at // c["page"]].long()
        s["k"][page, :, at % c["page"]] = k
        s["v"][page, :, at % c["page"]] = v
        return {"q": q, "k": s["k"], "v": s["v"]}
    s["vt"][:, :, :T] = v.permute(1, 2, 0)
    return {"q": q.transpose(0, 1).contiguous(), "k": k.transpose(0, 1).contiguous(), "vt": s["vt"]}


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if not own:
        return {"quantize": _plain_quantize, "gemm": _plain_gemm, "gated": _plain_gated, "norm": _plain_norm,
                "rotate": _plain_rotate}[kind](s)
    ctx = s["ctx"]
    if kind == "quantize":
        ctx.op_quantize_fp4(s["x"], s["Q"])
        ctx.op_dequantize_fp4(s["Q"], s["back"])
        return {"back": s["back"], "scale": s["Q"].scale, "row": s["Q"].row_scale}
    if kind == "gemm":
        ctx.op_gemm_fp4(s["A"], s["W"], s["C"], bias=s["bias"], gelu=c["mode"] == "gelu", res=s.get("res"), gate=s.get("gate"))
        return s["C"]
    if kind == "gated":
        ctx.op_gated_fp4(s["A"], s["W"], s["U"], s["C"], gate_bias=s["bias"], up_bias=s["up_bias"], gelu=c["act"] == "gelu")
        return s["C"]
    if kind == "norm":
        e4m3 = c["out"] == "e4m3"
        ctx.op_add_norm(s["x"], s["out"], delta=s.get("delta"), gate=s.get("gate"), total=s["sum"] if c["add"] else None,
                        weight=s["weight"], weight_offset=1.0, shift=s.get("shift"), center=c["center"], eps=EPS,
                        rows_per_set=c["mod"], scale=s["scale"] if e4m3 else None)
        r = {"sum": s["sum"]} if c["add"] else {}
        return dict(r, out=s["out"], scale=s["scale"]) if e4m3 else dict(r, out=s["out"])
    kw = dict(q_weight=s["wq"], k_weight=s["wk"], eps=EPS, axes=s["axes"], interleaved=c["inter"])
    if c["form"] == "append":
        ctx.op_qk_norm_rope_append(s["qkv"], s["q"], s["cache"], s["start"], **kw)
        return {"q": s["q"], "k": s["k"], "v": s["v"]}
    ctx.op_qk_norm_rope(s["qkv"], s["q"], s["k"], vt=s["vt"], **kw)
    return {"q": s["q"], "k": s["k"], "vt": s["vt"]}


# ---------------------------------------------------------------- work
def work(case):
    c, kind = case, case["kind"]
    es = 4 if c["dtype"] == "f32" else 2

    def fp4(rows, K):
        return rows * K // 2 + _ceil(rows, 128) * 128 * K // 16 + 4 * rows

    if kind == "quantize":
        n = c["M"] * c["K"]
        return {"bytes": 2 * es * n + 2 * fp4(c["M"], c["K"]), "flops": 4 * n}
    if kind in ("gemm", "gated"):
        M, N, K = c["M"], c["N"], c["K"]
        weights = 1 if kind == "gemm" else 2
        return {"bytes": fp4(M, K) + weights * fp4(N, K) + es * M * N * (2 if c.get("mode") == "resid" else 1) + 4 * weights * N,
                "flops": 2 * weights * M * N * K}
    if kind == "norm":
        n, e4m3 = c["M"] * c["D"], c["out"] == "e4m3"
        return {"bytes": n * (es * (3 if c["add"] else 1) + (1 if e4m3 else es)) + (4 * _ceil(c["D"], 128) * c["M"] if e4m3 else 0),
                "flops": 8 * n}
    T = sum(_counts(c)[0])
    n = T * (c["heads"] + 2 * c["kv"]) * c["d"]
    return {"bytes": 2 * es * n + 4 * T * len(_pairs(c)), "flops": 8 * n}


# ---------------------------------------------------------------- 64 bits
def _f32(x):
    """The fp32 number that the definition has at this place (scales, reciprocals and quotients are fp32 numbers)."""
    return x.float().double()


def _grid(y, bits, low, most):
    """The nearest value with `bits` bits after the point and exponents from `low`, ties to even, up to `most`."""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -40))).clamp(min=float(low))
    step = torch.exp2(e - bits)
    return (torch.round(y / step) * step).clamp(-most, most)


def _exact_quantize(c, seed):
    x = _activations(c, seed, 1, c["M"], c["K"]).double()
    M, K = x.shape
    top = x.abs().max(1).values
    row = _f32(top * torch.tensor(1 / 2688, device="cuda").double())
    row[top < TINY] = 0
    scale, back = torch.zeros(M, K // 16, device="cuda", dtype=torch.float64), torch.zeros_like(x)
    live = row > 0
    for j in range(K // 16):
        part = x[live, 16 * j:16 * j + 16]
        s = _grid(_f32(part.abs().max(1).values / _f32(6 * row[live])), 3, -6, 448.0)
        step = _f32(s * row[live])
        by = torch.where(step > 0, _f32(1 / torch.where(step > 0, step, 1.0)), 0.0)
        scale[live, j] = s
        back[live, 16 * j:16 * j + 16] = _grid(_f32(part * by[:, None]), 1, 0, 6.0) * step[:, None]
    pieces = torch.zeros(_ceil(M, 128), K // 64, 512, device="cuda", dtype=torch.float64)
    r, j = torch.arange(M, device="cuda")[:, None], torch.arange(K // 16, device="cuda")
    pieces[r // 128, j // 4, r % 32 * 16 + r % 128 // 32 * 4 + j % 4] = scale
    return {"back": back, "scale": pieces, "row": row}


def _exact_values(m):
    packed, pieces, row = m
    M, half = packed.shape
    v = torch.zeros(M, 2 * half, device="cuda", dtype=torch.float64)
    for i in range(2):
        code = packed >> 4 * i & 15
        e, m1 = (code >> 1 & 3).double(), (code & 1).double()
        size = torch.where(e == 0, 0.5 * m1, torch.exp2(e - 1) * (1 + 0.5 * m1))
        v[:, i::2] = torch.where(code > 7, -size, size)
    r, j = torch.arange(M, device="cuda")[:, None], torch.arange(half // 8, device="cuda")
    s = pieces.double()[r // 128, j // 4, r % 32 * 16 + r % 128 // 32 * 4 + j % 4]
    return v * s.repeat_interleave(16, 1) * row.double()[:, None]


def _exact_act(y, gelu):
    return y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))) if gelu else y * torch.sigmoid(y)


def _exact_product(c, seed):
    s = _gemm_inputs(c, seed)
    a = _exact_values(s["A"])
    y = a @ _exact_values(s["W"]).t() + s["bias"].double()
    if c["kind"] == "gated":
        u = a @ _exact_values(s["U"]).t() + s["up_bias"].double()
        return _exact_act(y, c["act"] == "gelu") * u
    if c["mode"] == "gelu":
        return _exact_act(y, True)
    return s["res"].double() + s["gate"].double() * y if c["mode"] == "resid" else y


def _exact_norm(c, seed):
    s = _norm_inputs(c, seed)
    per = c["mod"] or c["M"]
    out, total = [], []
    for i in range(0, c["M"], per):
        v = {k: t[i // per].double() for k, t in s.items() if k in ("weight", "shift", "gate")}
        x = s["x"][i:i + per].double()
        if c["add"]:
            x = x + v["gate"] * s["delta"][i:i + per].double()
        total.append(x)
        if c["center"]:
            x = x - x.sum(1, keepdim=True) / c["D"]
        y = x / ((x * x).sum(1, keepdim=True) / c["D"] + EPS).sqrt() * (1 + v["weight"])
        out.append(y + v["shift"] if c["center"] else y)
    r, y = ({"sum": torch.cat(total)} if c["add"] else {}), torch.cat(out)
    if c["out"] == "same":
        return dict(r, out=y)
    scale, q = torch.empty(_ceil(c["D"], 128), c["M"], device="cuda", dtype=torch.float64), torch.empty_like(y)
    for j in range(scale.shape[0]):
        part = y[:, 128 * j:128 * j + 128]
        scale[j] = part.abs().max(1).values / 448
        q[:, 128 * j:128 * j + 128] = _grid(part / torch.where(scale[j] > 0, scale[j], 1.0)[:, None], 3, -6, 448.0)
    return dict(r, out=q, scale=scale)


def _exact_turn(x, w, tables, place, inter):
    y = x / ((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()
    out, total, i = y.clone(), sum(t.shape[1] for t in tables), 0
    for a, t in enumerate(tables):
        cs = t.double()[place[:, a].long()]
        for j in range(t.shape[1]):
            p, q = (2 * i, 2 * i + 1) if inter else (i, i + total)
            c, s = cs[:, j, 0, None], cs[:, j, 1, None]
            out[..., p], out[..., q] = y[..., p] * c - y[..., q] * s, y[..., q] * c + y[..., p] * s
            i += 1
    return out


def _exact_rotate(c, seed):
    new, past = _counts(c)
    H, kv, page = c["heads"], c["kv"], c["page"]
    qkv, wq, wk = _heads(c, seed, new)
    tables, place = _axes(c, new, past)
    x = qkv.double().view(-1, H + 2 * kv, c["d"])
    q, k = _exact_turn(x[:, :H], wq, tables, place, c["inter"]), _exact_turn(x[:, H:H + kv], wk, tables, place, c["inter"])
    v = x[:, H + kv:]
    if c["form"] == "dense":
        T = x.shape[0]
        vt = torch.zeros(kv, c["d"], _ceil(T, 8) * 8 if c["dtype"] == "bf16" else T, device="cuda", dtype=torch.float64)
        vt[:, :, :T] = v.permute(1, 2, 0)
        return {"q": q.transpose(0, 1), "k": k.transpose(0, 1), "vt": vt}
    table, _, _, pk, pv = _paging(c, seed, new, past)
    pk, pv, t0 = pk.double(), pv.double(), 0
    for b, (n, p) in enumerate(zip(new, past)):
        for g in range(p // page, _ceil(n + p, page)):
            lo, hi = max(p, g * page), min(n + p, (g + 1) * page)
            rows, slots = slice(t0 + lo - p, t0 + hi - p), slice(lo - g * page, hi - g * page)
            pk[table[b, g], :, slots] = k[rows].transpose(0, 1)
            pv[table[b, g], :, slots] = v[rows].transpose(0, 1)
        t0 += n
    return {"q": q, "k": pk, "v": pv}


def exact(case, seed):
    return {"quantize": _exact_quantize, "gemm": _exact_product, "gated": _exact_product, "norm": _exact_norm,
            "rotate": _exact_rotate}[case["kind"]](case, seed)
