"""Timed cases of the operators around the attention of a shard: attention with modified scores, and the per-head
norms and rotations of its queries and keys, in their plain form and through the entry points of paper_2407_00611_amd.

  attn_fwd     the row spans of the step's documents, then attention of a query shard against one chunk of keys whose
               scores may be capped by a tanh, biased by distance and masked by documents and prefixes: O and lse
  attn_train   the same, then Delta and the gradients of Q, K and V
  rope_fwd     RMS norm of every query and key head and the rotation by their positions, on one or several axes
  rope_train   the same, then the gradients of the projections and of the norm weights from the fp32 gradients that the
               attention backward leaves

Values are i.i.d. normal, as projections leave them; shapes are this repository's benchmark configurations and
ordinary or odd sizes between them.
"""
import math

import torch

own = False

ATTN = {"op": "attn_fwd", "dtype": "bf16", "B": 1, "Hq": 32, "Hkv": 8, "D": 128, "Sq": 4096, "Sk": 4096, "q_offset": 0,
        "seg": 0, "q_offset2": 0, "k_offset": 0, "causal": True, "cap": 0.0, "alibi": False, "docs": 0, "prefix": False,
        "pad": "tail", "layout": "dense"}
ROPE = {"op": "rope_fwd", "dtype": "bf16", "B": 1, "Hq": 32, "Hkv": 8, "D": 128, "S": 4096, "rot": 128, "axes": 1,
        "pairs": "halves", "norm": True, "offset": 0, "seg": 0, "offset2": 0, "layout": "dense"}


def listed():
    return [
        # a new token of four sequences, left-padded to one length, distance bias: few rows, latency
        dict(ATTN, name="one_token_batch", B=4, Sq=1, Sk=8192, q_offset=8191, alibi=True, docs=1, pad="head"),
        # a new token against 128K keys, capped scores: bound by reading the keys and values
        dict(ATTN, name="one_token_long", Sq=1, Sk=131072, q_offset=131071, cap=50.0),
        # prompts packed into one row, each with a prefix that all of its tokens see
        dict(ATTN, name="packed_prompts", docs=8, prefix=True),
        # images of several sizes packed into one row, head size 64, no causal order
        dict(ATTN, name="packed_images_d64", Hq=24, Hkv=24, D=64, Sq=8192, Sk=8192, causal=False, docs=6),
        # fp32 training of a small layer whose head size fits no tile, everything at once
        dict(ATTN, name="train_f32", op="attn_train", dtype="f32", Hq=8, Hkv=2, D=80, Sq=500, Sk=500, cap=20.0, alibi=True, docs=3),
        # training of two packed rows of 1000 tokens, grouped heads, queries, keys and values in one buffer
        dict(ATTN, name="train_ragged", op="attn_train", B=2, Hq=12, Hkv=4, Sq=1000, Sk=1000, cap=30.0, docs=5, prefix=True,
             layout="packed"),
        # the load-balanced placement: an early and a late run of rows against one chunk of the ring, distance bias
        dict(ATTN, name="train_zigzag_alibi", op="attn_train", q_offset=4096, seg=2048, q_offset2=26624, k_offset=4096, Sk=2048,
             alibi=True),
        # a training row of 8192 tokens of packed documents, capped scores
        dict(ATTN, name="train_docs_capped", op="attn_train", Sq=8192, Sk=8192, cap=50.0, docs=3),
        # one new token of 16 sequences: latency
        dict(ROPE, name="rope_one_token", B=16, S=1, offset=8191),
        # latent video, 16 frames of 32 x 32 patches, three axes, head size 64
        dict(ROPE, name="rope_video", Hq=24, Hkv=24, D=64, S=16384, rot=64, axes=3),
        # training, two runs of rows of a 128K sequence, grouped heads, projections in one buffer
        dict(ROPE, name="rope_train_gqa", op="rope_train", S=4096, offset=28672, seg=2048, offset2=98304, layout="packed"),
        # fp32, part of an odd head size rotated, neighbouring pairs, far positions
        dict(ROPE, name="rope_train_f32", op="rope_train", dtype="f32", B=2, Hq=12, Hkv=4, D=80, S=1000, rot=64,
             pairs="neighbours", offset=500000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn_fwd", "attn_fwd", "attn_train", "attn_train", "attn_train", "rope_fwd", "rope_train"])
    f32 = rng.random() < 0.25
    g, hkv = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 8])
    c = {"op": op, "dtype": "f32" if f32 else "bf16", "B": rng.choice([1, 1, 2, 3]), "Hq": g * hkv, "Hkv": hkv}
    if op.startswith("rope"):
        d = rng.choice([32, 64, 80, 96, 128, 128, 192, 256])
        c.update(D=d, S=_log_int(rng, 1, 16384), rot=rng.choice([d, d, d // 2]), axes=rng.choice([1, 1, 2, 3]),
                 pairs=rng.choice(["halves", "neighbours"]), norm=rng.random() < 0.75, offset=_log_int(rng, 1, 1000000), seg=0,
                 offset2=0, layout=rng.choice(["dense", "packed", "heads_first"]))
        if c["axes"] == 1 and c["S"] > 2 and rng.random() < 0.4:
            c.update(seg=c["S"] // 2, offset2=c["offset"] + 2 * c["S"])
        return c
    # for training some keys a row, as the gradient of the scores of a single one is nothing but rounding
    sk = _log_int(rng, 16 if op == "attn_train" else 1, 700 if f32 else 8192)
    sq = sk if rng.random() < 0.6 else _log_int(rng, 1, 700 if f32 else 4096)
    docs = min(rng.choice([0, 0, 1, 2, 5, 16]), max(sk // 8, 1))
    c.update(D=rng.choice([32, 64, 80, 128, 256]) if f32 else rng.choice([64, 128, 128]), Sq=sq, Sk=sk,
             q_offset=max(0, sk - sq), seg=0, q_offset2=0, k_offset=0, causal=rng.random() < 0.7,
             cap=rng.choice([0.0, 0.0, 15.0, 50.0]), alibi=rng.random() < 0.4, docs=docs,
             prefix=docs > 0 and rng.random() < 0.4, pad=rng.choice(["tail", "head"]),
             layout=rng.choice(["dense", "packed" if sq == sk else "dense", "heads_first"]))
    if sq > 2 and rng.random() < 0.2:           # two runs of rows, the second one further on
        c.update(seg=sq // 2, q_offset2=c["q_offset"] + 2 * sq, docs=0, prefix=False)
    # the plain form holds the scores of all pairs
    while work(c)["flops"] > 6e11 or c["B"] * c["Hq"] * c["Sq"] * c["Sk"] > 2 ** 31 - 1:
        c.update(B=1, Hq=g * max(1, c["Hkv"] // 2), Hkv=max(1, c["Hkv"] // 2))
    return c


# ---------------------------------------------------------------------------------------------- shapes of a case

def _row_positions(c, device="cpu"):
    n, off, off2 = (c["Sq"], c["q_offset"], c["q_offset2"]) if c["op"].startswith("attn") else (c["S"], c["offset"], c["offset2"])
    i = torch.arange(n, dtype=torch.int64, device=device)
    return torch.where(i < c["seg"], off + i, off2 + i - c["seg"]) if c["seg"] else off + i


def _placement(offset, seg, offset2):
    return (offset, seg, offset2) if seg else offset


def _bounds(c):
    """[B, docs + 1] first positions of the documents of every packed row: lengths as 1 : 2 : 3 in turn, another one first
    in every row, beside some padding."""
    total = max(c["q_offset"] + c["Sq"], c["k_offset"] + c["Sk"])
    rows = []
    for b in range(c["B"]):
        part = [1 + (j + b) % 3 for j in range(c["docs"])]
        pad = total * (1 + b % 4) // 32
        ends = [(total - pad) * sum(part[:j]) // sum(part) for j in range(c["docs"] + 1)]
        rows.append([e + pad for e in ends] if c["pad"] == "head" else ends)
    return torch.tensor(rows, dtype=torch.int64)


def _prefix(c):
    """A quarter of every document."""
    b = _bounds(c)
    return (b[:, 1:] - b[:, :-1]) // 4


def _pairs(c):
    """Visible (row, key) pairs of one query head, all batch entries."""
    pos = _row_positions(c).expand(c["B"], -1)
    lo, hi = torch.zeros_like(pos), torch.full_like(pos, 1 << 60)
    if c["docs"]:
        b = _bounds(c)
        d = torch.searchsorted(b, pos.contiguous(), right=True) - 1
        inside = (d >= 0) & (d < c["docs"])
        d = d.clamp(0, c["docs"] - 1)
        lo, hi = b.gather(1, d), torch.where(inside, b.gather(1, d + 1), 0)
        if c["causal"]:
            first = pos + 1
            if c["prefix"]:
                first = torch.maximum(first, lo + _prefix(c).gather(1, d))
            hi = torch.minimum(hi, first)
    elif c["causal"]:
        hi = pos + 1
    return int((hi.clamp(max=c["k_offset"] + c["Sk"]) - lo.clamp(min=c["k_offset"])).clamp(min=0).sum())


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"].startswith("rope"):
        x = c["B"] * c["S"] * (c["Hq"] + c["Hkv"]) * c["D"]
        # forward: x in, y out; backward: x and the fp32 gradient in, the gradient of x out
        train = c["op"] == "rope_train"
        need_x = c["norm"] or not train
        return {"bytes": 2 * x * e + (x * (e * c["norm"] + 4 + e) if train else 0) + 8 * c["rot"], "flops": x * (22 if train else 8) * need_x}
    q, kv, rows = c["B"] * c["Sq"] * c["Hq"] * c["D"], 2 * c["B"] * c["Sk"] * c["Hkv"] * c["D"], c["B"] * c["Sq"] * c["Hq"]
    pairs = c["Hq"] * _pairs(c)
    fwd = (2 * q + kv) * e + 4 * rows
    if c["op"] == "attn_fwd":
        return {"bytes": fwd, "flops": 4 * c["D"] * pairs}
    # backward: Q, K, V, O, dO, lse in; dQ, dK, dV out
    return {"bytes": fwd + (4 * q + 2 * kv) * e + 4 * rows, "flops": 14 * c["D"] * pairs}


# ---------------------------------------------------------------------------------------------- inputs

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _heads(gen, c, S, heads, dtype):
    """[B, S, h, D] values for each h in `heads`, in one of the memory layouts projections leave them in."""
    B, D = c["B"], c["D"]
    if c["layout"] == "packed":
        x = torch.randn((B, S, sum(heads), D), generator=gen, device="cuda").to(dtype)
        return list(x.split(heads, dim=2))
    if c["layout"] == "heads_first":
        return [torch.randn((B, h, S, D), generator=gen, device="cuda").to(dtype).transpose(1, 2) for h in heads]
    return [torch.randn((B, S, h, D), generator=gen, device="cuda").to(dtype) for h in heads]


def _video_positions(c):
    """Frame, row and column of every patch of a clip as near to 16 : 32 : 32 as its patches allow; int32 [axes, B, S]."""
    i = torch.arange(c["S"], dtype=torch.int32, device="cuda") + c["offset"]
    axes = [i // 1024, i // 32 % 32, i % 32] if c["axes"] == 3 else [i // 32, i % 32]
    return torch.stack(axes)[:, None].expand(-1, c["B"], -1).contiguous()


def _axis_pairs(c):
    """Pairs that each axis turns: all of them, halves, or a quarter for the frames and the rest in halves."""
    n = c["rot"] // 2
    if c["axes"] == 1:
        return [n]
    return [n // 2, n - n // 2] if c["axes"] == 2 else [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2]


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _dtype(c)
    if c["op"].startswith("rope"):
        q, k = _heads(gen, c, c["S"], [c["Hq"], c["Hkv"]], dt)
        freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in _axis_pairs(c)])
        s = {"c": c, "q": q, "k": k, "freq": freq.cuda(), "positions": _video_positions(c) if c["axes"] > 1 else None,
             "q_weight": None, "k_weight": None}
        if c["norm"]:
            s["q_weight"], s["k_weight"] = (1 + 0.1 * torch.randn((2, c["D"]), generator=gen, device="cuda")).unbind()
        if c["op"] == "rope_train":
            s["dq"], s["dk"] = (torch.randn((c["B"], c["S"], h, c["D"]), generator=gen, device="cuda") for h in (c["Hq"], c["Hkv"]))
        return s
    if c["layout"] == "packed":
        q, k, v = _heads(gen, c, c["Sq"], [c["Hq"], c["Hkv"], c["Hkv"]], dt)
    else:
        q, = _heads(gen, c, c["Sq"], [c["Hq"]], dt)
        k, v = _heads(gen, c, c["Sk"], [c["Hkv"], c["Hkv"]], dt)
    s = {"c": c, "q": q, "k": k, "v": v, "scale": 1 / math.sqrt(c["D"]), "slopes": None, "bounds": None, "prefix": None}
    if c["cap"]:                    # scores that the cap bends: some units wide
        s["scale"] *= 4.0
    if c["alibi"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / c["Hq"]) for h in range(c["Hq"])], device="cuda")
    if c["docs"]:
        s["bounds"] = _bounds(c).cuda()
        s["prefix"] = _prefix(c).cuda() if c["prefix"] else None
    if c["op"] == "attn_train":
        s["d_o"] = torch.randn((c["B"], c["Sq"], c["Hq"], c["D"]), generator=gen, device="cuda").to(dt)
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    if own:
        return _own_rope(s) if s["c"]["op"].startswith("rope") else _own_attention(s)
    return _plain_rope(s) if s["c"]["op"].startswith("rope") else _plain_attention(s)


def _own_attention(s):
    import paper_2407_00611_amd as st
    c = s["c"]
    rows, causal, spans = _placement(c["q_offset"], c["seg"], c["q_offset2"]), c["causal"], None
    if s["bounds"] is not None:     # they hold the causal order too
        spans, causal = st.st_mask_spans(s["bounds"], c["Sq"], rows, causal, prefix=s["prefix"]), False
    mods = {"softcap": c["cap"], "slopes": s["slopes"], "spans": spans}
    o, lse = st.st_attn_score_fwd(s["q"], s["k"], s["v"], rows, c["k_offset"], causal, s["scale"], lowp=True, **mods)
    if c["op"] == "attn_fwd":
        return {"o": o, "lse": lse}
    delta = st.st_attn_delta(s["d_o"], o)
    dq, dk, dv = st.st_attn_score_bwd(s["q"], s["k"], s["v"], s["d_o"], lse, delta, rows, c["k_offset"], causal, s["scale"], **mods)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_rope(s):
    import paper_2407_00611_amd as st
    c = s["c"]
    how = {"freq": s["freq"], "offset": _placement(c["offset"], c["seg"], c["offset2"]), "positions": s["positions"],
           "axes": _axis_pairs(c), "pairs": c["pairs"], "norm": c["norm"], "q_weight": s["q_weight"], "k_weight": s["k_weight"]}
    q, k = st.st_qk_rope_fwd(s["q"], s["k"], **how)
    if c["op"] == "rope_fwd":
        return {"q": q, "k": k}
    dq, dk, dwq, dwk = st.st_qk_rope_bwd(s["q"], s["k"], s["dq"], s["dk"], **how)
    return {"q": q, "k": k, "dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def _visible(s, k_pos):
    """[B or 1, 1, Sq, Sk] truth values."""
    c = s["c"]
    pos = _row_positions(c, "cuda")
    if s["bounds"] is None:
        seen = k_pos <= pos[:, None] if c["causal"] else torch.ones((c["Sq"], c["Sk"]), dtype=torch.bool, device="cuda")
        return seen[None, None]
    def document(p):
        d = torch.searchsorted(s["bounds"], p.expand(c["B"], -1).contiguous(), right=True) - 1
        return torch.where(d < c["docs"], d, -1)
    dq, dk = document(pos), document(k_pos)
    seen = (dq[:, :, None] == dk[:, None, :]) & (dq >= 0)[:, :, None]
    if c["causal"]:
        early = k_pos <= pos[:, None]
        if s["prefix"] is not None:
            d = dq.clamp(min=0)
            early = early | (k_pos < (s["bounds"].gather(1, d) + s["prefix"].gather(1, d))[:, :, None])
        seen = seen & early
    return seen[:, None]


def _plain_attention(s):
    c, dt = s["c"], _dtype(s["c"])
    group = c["Hq"] // c["Hkv"]
    wide = lambda x: x.float().transpose(1, 2).repeat_interleave(c["Hq"] // x.shape[2], dim=1).contiguous()
    q, k, v = wide(s["q"]), wide(s["k"]), wide(s["v"])
    pos, k_pos = _row_positions(c, "cuda"), torch.arange(c["Sk"], device="cuda") + c["k_offset"]
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    slope = None
    if c["cap"]:
        x = torch.tanh(x / c["cap"])
        slope = 1 - x * x
        x = x * c["cap"]
    if s["slopes"] is not None:
        x = x - s["slopes"][None, :, None, None] * (pos[:, None] - k_pos).abs().float()
    x = x.masked_fill(~_visible(s, k_pos), -math.inf)
    top = x.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = torch.exp(x - top)
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total > 0, total, 1)
    o = torch.matmul(p, v)
    out = {"o": o.transpose(1, 2).to(dt).contiguous(), "lse": (top + torch.log(total)).squeeze(3)}
    if c["op"] == "attn_fwd":
        return out
    d_o = wide(s["d_o"])
    ds = p * (torch.matmul(d_o, v.transpose(2, 3).contiguous()) - (d_o * o).sum(3, keepdim=True))
    if slope is not None:
        ds = ds * slope
    ds = ds * s["scale"]
    narrow = lambda x: x.unflatten(1, (c["Hkv"], group)).sum(2).transpose(1, 2).to(dt).contiguous()
    out["dq"] = torch.matmul(ds, k).transpose(1, 2).to(dt).contiguous()
    out["dk"] = narrow(torch.matmul(ds.transpose(2, 3).contiguous(), q))
    out["dv"] = narrow(torch.matmul(p.transpose(2, 3).contiguous(), d_o))
    return out


def _angles(s):
    """[B or 1, S, 1, rot / 2] in 64 bits."""
    c = s["c"]
    if s["positions"] is None:
        return (_row_positions(c, "cuda")[:, None].double() * s["freq"])[None, :, None]
    axis = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(_axis_pairs(c))).cuda()
    return s["positions"][axis].permute(1, 2, 0)[:, :, None].double() * s["freq"]


def _split(x, c):
    """First and second values of the rotated pairs, and the rest."""
    r, n = x[..., :c["rot"]], c["rot"] // 2
    a, b = (r[..., :n], r[..., n:]) if c["pairs"] == "halves" else (r[..., 0::2], r[..., 1::2])
    return a, b, x[..., c["rot"]:]


def _join(a, b, rest, c):
    r = torch.cat([a, b], -1) if c["pairs"] == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _plain_rope(s):
    c, dt = s["c"], _dtype(s["c"])
    angle = _angles(s)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def forward(x, w):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        a, b, rest = _split(x, c)
        return _join(a * cos - b * sin, a * sin + b * cos, rest, c).to(dt)

    def backward(x, w, dy):
        a, b, rest = _split(dy, c)
        dn = _join(a * cos + b * sin, b * cos - a * sin, rest, c)
        if not c["norm"]:
            return dn.to(dt), None
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        x, g = x * r, dn * w
        return (r * (g - x * (g * x).mean(-1, keepdim=True))).to(dt), (dn * x).sum((0, 1, 2))

    out = {"q": forward(s["q"], s["q_weight"]), "k": forward(s["k"], s["k_weight"])}
    if c["op"] == "rope_train":
        out["dq"], out["dwq"] = backward(s["q"], s["q_weight"], s["dq"])
        out["dk"], out["dwk"] = backward(s["k"], s["k_weight"], s["dk"])
    return out


# ---------------------------------------------------------------------------------------------- from the definition, in 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    return _exact_rope(s) if c["op"].startswith("rope") else _exact_attention(s)


def _exact_attention(s):
    """One query head after the other, gradients by differentiation."""
    c, train = s["c"], s["c"]["op"] == "attn_train"
    q, k, v = (s[x].double().detach().requires_grad_(train) for x in "qkv")
    i, t = _row_positions(c, "cuda")[:, None], (torch.arange(c["Sk"], device="cuda") + c["k_offset"])[None, :]
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["B"], c["Hq"], c["Sq"]), dtype=torch.float64, device="cuda")
    bounds, prefix = _bounds(c) if c["docs"] else None, _prefix(c) if c["prefix"] else None
    for b in range(c["B"]):
        seen = (t <= i) if c["causal"] else (t == t).expand(c["Sq"], -1)
        if bounds is not None:
            order, seen = seen, torch.zeros_like(seen)
            for d in range(c["docs"]):
                lo, hi = int(bounds[b, d]), int(bounds[b, d + 1])
                early = order if prefix is None else order | (t < lo + int(prefix[b, d]))
                seen = seen | ((i >= lo) & (i < hi) & (t >= lo) & (t < hi) & early)
        for h in range(c["Hq"]):
            x = q[b, :, h] @ k[b, :, h * c["Hkv"] // c["Hq"]].T * s["scale"]
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * (i - t).abs()
            x = torch.where(seen, x, -math.inf)
            top = x.detach().amax(1, keepdim=True)
            top = torch.where(top == -math.inf, 0, top)
            e = torch.exp(x - top)
            total = e.sum(1, keepdim=True)
            y = e @ v[b, :, h * c["Hkv"] // c["Hq"]] / (total + (total == 0))
            if train:
                (y * s["d_o"][b, :, h].double()).sum().backward()
            o[b, :, h] = y.detach()
            lse[b, h] = (top + torch.log(total)).detach()[:, 0]
    out = {"o": o, "lse": lse}
    if train:
        out.update(dq=q.grad, dk=k.grad, dv=v.grad)
    return out


def _exact_rope(s):
    """Pairs as complex numbers, gradients by differentiation."""
    c, train = s["c"], s["c"]["op"] == "rope_train"
    n = c["rot"] // 2
    first = torch.arange(n, device="cuda") if c["pairs"] == "halves" else 2 * torch.arange(n, device="cuda")
    second = first + (n if c["pairs"] == "halves" else 1)
    angle = torch.zeros((c["B"], c["S"], n), dtype=torch.float64, device="cuda")
    at = 0
    for axis, m in enumerate(_axis_pairs(c)):
        p = _row_positions(c, "cuda").expand(c["B"], -1) if s["positions"] is None else s["positions"][axis].long()
        angle[:, :, at:at + m] = p[:, :, None] * s["freq"][at:at + m]
        at += m
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    out = {}
    for name in "qk":
        x = s[name].double().detach().requires_grad_(train)
        w = s[name + "_weight"].double().detach().requires_grad_(train) if c["norm"] else None
        y = x if w is None else x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        z = torch.complex(y[..., first], y[..., second]) * turn
        y = y.index_copy(-1, first, z.real).index_copy(-1, second, z.imag)
        out[name] = y.detach()
        if train:
            (y * s["d" + name].double()).sum().backward()
            out["d" + name], out["dw" + name] = x.grad, None if w is None else w.grad
    return out
