"""Timed cases of the operators that serve a model: a cache of keys and values in pages, in the storage type or in 8 bits with a
scale for each page and head, how new tokens get into it, how chunks come out of it, and the attention that reads it; in their
plain form and through the entry points of paper_2407_00611_amd.

  attn     attention of the new rows of a batch of sequences (one token each, a few, whole prompts, or both) against the cache,
           whose scores may be capped by a tanh, biased by distance and cut by a window: O and lse
  append   RMS norm of every query and key head, the rotation by the tokens' places, and keys and values into the cache; then the
           pages that have changed, read back as dense chunks
  read     a run of every sequence's tokens as dense chunks of keys and values, as the ring's attention takes them

A page in 8 bits holds e4m3 values times a power of two, 2^e, for each head: e is the least with which the largest new value of
the page is within 448 2^e, and never less than the page had with the rows before them.  Scales are stored as e + 127.

Values are i.i.d. normal, the cached ones of every page and head with a spread of their own; the pages of the sequences lie in no order.
"""
import math

import torch

own = False

ATTN = {"op": "attn", "dtype": "bf16", "cache": "e4m3", "B": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "len": 8192, "ragged": False,
        "rows": 1, "prompts": 0, "prompt_rows": 0, "causal": True, "window": 0, "cap": 0.0, "bias": False, "ahead": 0}
APPEND = {"op": "append", "dtype": "bf16", "cache": "e4m3", "B": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "len": 8192, "ragged": False,
          "rows": 1, "prompts": 0, "prompt_rows": 0, "rot": 128, "pairs": "halves", "norm": True, "offset": 0, "layout": "dense"}
READ = {"op": "read", "dtype": "bf16", "cache": "e4m3", "B": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "len": 8192, "ragged": False,
        "rows": 1, "prompts": 0, "prompt_rows": 0, "count": 8192}


def listed():
    return [
        # the next token of one short conversation: latency
        dict(ATTN, name="one_token_short", page=16, len=700),
        # the next token of one sequence of 128K tokens: reading the keys and values
        dict(ATTN, name="one_token_long", len=131072),
        # a serving batch of 64 sequences of very different lengths, one of them a free place
        dict(ATTN, name="batch_ragged", B=64, page=16, ragged=True),
        # a model of 24 heads of 64 with a cache in the storage type, every layer but some with a window
        dict(ATTN, name="batch_window_d64", cache="bf16", B=32, Hq=24, Hkv=24, D=64, page=32, len=4096, ragged=True, window=1000),
        # five drafted tokens of each of 16 sequences are looked over at once, capped scores
        dict(ATTN, name="drafts_capped", B=16, Hq=12, Hkv=4, page=32, len=4096, ragged=True, rows=5, cap=30.0),
        # a piece of a long prompt behind the 16K tokens that the cache holds
        dict(ATTN, name="prompt_piece", len=18432, rows=2048),
        # two prompts among sequences that go on by a token, distance bias, cache in the storage type
        dict(ATTN, name="mixed_bias", cache="bf16", B=24, page=16, len=2000, ragged=True, prompts=2, prompt_rows=700, bias=True),
        # fp32, a head size that fits no tile
        dict(ATTN, name="batch_f32", dtype="f32", cache="f32", B=4, Hq=8, Hkv=2, D=80, page=16, len=2000, ragged=True, rows=3),
        # the next token of 16 sequences: latency
        dict(APPEND, name="append_one_token", B=16, ragged=True),
        # prompts of 6000, 3000 and 2000 tokens, projections in one buffer
        dict(APPEND, name="append_prompts", B=3, len=6000, ragged=True, rows=2000, prompts=2, prompt_rows=6000, layout="packed"),
        # a shard of a 128K sequence for the ring
        dict(READ, name="read_shard", len=131072, count=32768),
        # the cached beginnings of 16 sequences, fp32 chunks of an odd head size
        dict(READ, name="read_f32", dtype="f32", B=16, Hq=8, Hkv=2, D=80, page=16, len=1000, ragged=True, count=1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "attn", "append", "append", "read"])
    f32 = rng.random() < 0.2
    g, hkv = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 8])
    c = {"op": op, "dtype": "f32" if f32 else "bf16", "B": _log_int(rng, 1, 64), "Hq": g * hkv, "Hkv": hkv,
         "page": rng.choice([16, 16, 32, 64, 128, 256]), "len": _log_int(rng, 16, 4000 if f32 else 32768), "ragged": rng.random() < 0.7,
         "rows": 1, "prompts": 0, "prompt_rows": 0}
    c["cache"] = rng.choice(["e4m3", c["dtype"]]) if op != "attn" or f32 else rng.choice(["e4m3", "e4m3", "bf16"])
    if op == "read":
        c.update(D=rng.choice([32, 64, 80, 128, 128, 256]), count=_log_int(rng, 1, c["len"]))
    else:
        if rng.random() < 0.5:                      # some rows more, or prompts among single tokens
            if rng.random() < 0.5:
                c.update(rows=_log_int(rng, 2, min(c["len"], 600 if f32 else 2000)))
            else:
                c.update(prompts=rng.randint(1, 3), prompt_rows=_log_int(rng, 2, min(c["len"], 600 if f32 else 2000)))
        if op == "append":
            d = rng.choice([32, 64, 80, 128, 128, 256])
            c.update(D=d, rot=rng.choice([d, d, d // 2, 0]), pairs=rng.choice(["halves", "neighbours"]), norm=rng.random() < 0.6,
                     offset=_log_int(rng, 1, 1000000), layout=rng.choice(["dense", "packed"]))
        else:
            c.update(D=rng.choice([32, 64, 80, 128, 256]) if f32 else rng.choice([64, 128, 128]), causal=rng.random() < 0.8,
                     window=rng.choice([0, 0, 0, _log_int(rng, 4, 4000)]), cap=rng.choice([0.0, 0.0, 15.0, 50.0]),
                     bias=rng.random() < 0.25, ahead=rng.choice([0, 0, 0, _log_int(rng, 1, 100000)]))
            if c["ahead"]:                          # far rows with a bias have scores that 32 bits are too few for
                c["bias"] = False
            if c["ahead"] and c["window"]:          # a share that the window has left behind would see nothing at all
                c["ahead"] = c["window"] // 2
    # the plain form holds the keys and values in 32 bits, padded to the longest sequence, and the scores of all pairs
    def too_much():
        w = work(c)
        return c["B"] * c["len"] * c["Hkv"] * c["D"] > 2 ** 29 or c["B"] * c["len"] * c["Hq"] * _most_rows(c) > 2 ** 30 or \
            w["bytes"] > 5e8 or w["flops"] > 5e11
    while too_much():
        if c["B"] > 1:
            c["B"] //= 2
        else:
            c.update(rows=max(1, c["rows"] // 2), prompt_rows=max(1, c["prompt_rows"] // 2), len=max(16, c["len"] * 3 // 4))
    return c


# ---------------------------------------------------------------------------------------------- shapes of a case

def _counts(c):
    """New rows of every sequence: prompts first, each half as long as the one before."""
    return [max(c["prompt_rows"] >> b, 1) if b < c["prompts"] else c["rows"] for b in range(c["B"])]


def _most_rows(c):
    return max(_counts(c))


def _lens(c):
    """Tokens of every sequence, the new ones among them: all alike, or spread over the range, and one sequence of none where
    there are many."""
    n = _counts(c)
    if not c["ragged"]:
        return [max(c["len"], x) for x in n]
    lens = [max(int(c["len"] * (1 - 0.95 * (b * 0.6180339887 % 1))), n[b]) for b in range(c["B"])]
    if c["B"] >= 32 and c["op"] == "attn":
        lens[c["B"] // 2] = 0
    return lens


def _first(c):
    """First rows of what is read back: the page where the new tokens begin; of a read, a place on the way to the end."""
    if c["op"] == "append":
        return [(x - n) // c["page"] * c["page"] for x, n in zip(_lens(c), _counts(c))]
    return [max(x - c["count"], 0) // 2 for x in _lens(c)]


def _count(c):
    return max(x - f for x, f in zip(_lens(c), _first(c))) if c["op"] == "append" else c["count"]


def _width(c):
    return max((x + c["page"] - 1) // c["page"] for x in _lens(c)) + 1


def _size(kind):
    return {"e4m3": 1, "bf16": 2, "f32": 4}[kind]


def work(c):
    e, s = _size(c["dtype"]), _size(c["cache"])
    lens, n, T, kv = _lens(c), _counts(c), sum(_counts(c)), 2 * c["Hkv"] * c["D"]
    tables = 8 * c["B"] + 4 * sum((x + c["page"] - 1) // c["page"] for x in lens)
    if c["op"] == "read":
        rows = sum(min(max(x - f, 0), c["count"]) for x, f in zip(lens, _first(c)))
        return {"bytes": rows * kv * s + c["B"] * c["count"] * kv * e + tables, "flops": rows * kv}
    if c["op"] == "append":
        back = sum(min(x - f, _count(c)) for x, f in zip(lens, _first(c)))
        q = T * c["Hq"] * c["D"]
        return {"bytes": (2 * q + T * kv) * e + T * kv * s + back * kv * s + c["B"] * _count(c) * kv * e + tables,
                "flops": 10 * (q + T * kv)}
    seen = pairs = 0
    for x, m in zip(lens, n):
        p0 = (x if c["ahead"] else x - m) + c["ahead"]                    # place of the first row
        lo = lambda p: max(0, min(p - c["window"] + 1, x)) if c["window"] else 0
        hi = lambda p: max(0, min(p + 1, x)) if c["causal"] else x
        seen += max(0, hi(p0 + m - 1) - lo(p0))
        pairs += sum(max(0, hi(p) - lo(p)) for p in range(p0, p0 + m))
    q = T * c["Hq"] * c["D"]
    return {"bytes": seen * kv * s + 2 * q * e + 4 * T * c["Hq"] + tables, "flops": 4 * c["D"] * c["Hq"] * pairs}


# ---------------------------------------------------------------------------------------------- inputs

def _dtype(kind):
    return {"e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16, "f32": torch.float32}[kind]


def _exponent(top):
    """The least e with top <= 448 2^e, of 2^-126 .. 2^127; float of whole numbers."""
    m, x = torch.frexp(top)                                             # top = m 2^x, 1/2 <= m < 1
    return torch.where(top > 0, x - 9 + (m > 0.875), -126).clamp(-126, 127)


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt, B, page, width = _dtype(c["dtype"]), c["B"], c["page"], _width(c)
    n_pages = B * width + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda")[:B * width].to(torch.int32).reshape(B, width)
    starts = torch.tensor([0] + _counts(c)).cumsum(0).to(torch.int32).cuda()
    s = {"c": c, "table": order.contiguous(), "lens": torch.tensor(_lens(c), dtype=torch.int32, device="cuda"), "starts": starts}
    for name in "kv":
        spread = torch.exp2(torch.rand((n_pages, 1, c["Hkv"], 1), generator=gen, device="cuda") * 2 - 1)
        x = torch.randn((n_pages, page, c["Hkv"], c["D"]), generator=gen, device="cuda").mul_(spread)
        if c["cache"] == "e4m3":
            e = _exponent(x.abs().amax((1, 3)))
            x = x.mul_(torch.exp2(-e.float())[:, None, :, None])
            s[name + "_scale"] = (e + 127).to(torch.uint8)
        s[name + "_cache"] = x.to(_dtype(c["cache"]))
    T = int(sum(_counts(c)))
    if c["op"] == "attn":
        s["q"] = torch.randn((1, T, c["Hq"], c["D"]), generator=gen, device="cuda").to(dt)
        s["scale"] = (4.0 if c["cap"] else 1.0) / math.sqrt(c["D"])     # with a cap, scores that it bends
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / c["Hq"]) for h in range(c["Hq"])], device="cuda") if c["bias"] else None
        s["q_first"] = s["lens"].long() + c["ahead"] if c["ahead"] else None
        return s
    s["first"] = torch.tensor(_first(c), dtype=torch.int32, device="cuda")
    if c["op"] == "append":
        heads = [c["Hq"], c["Hkv"], c["Hkv"]]
        if c["layout"] == "packed":
            s["q"], s["k"], s["v"] = torch.randn((1, T, sum(heads), c["D"]), generator=gen, device="cuda").to(dt).split(heads, dim=2)
        else:
            s["q"], s["k"], s["v"] = (torch.randn((1, T, h, c["D"]), generator=gen, device="cuda").to(dt) for h in heads)
        s["freq"] = 10000.0 ** (-torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda") / max(c["rot"] // 2, 1))
        s["q_weight"] = s["k_weight"] = None
        if c["norm"]:
            s["q_weight"], s["k_weight"] = (1 + 0.1 * torch.randn((2, c["D"]), generator=gen, device="cuda")).unbind()
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    return _own(s) if own else {"attn": _plain_attention, "append": _plain_append, "read": _plain_read}[s["c"]["op"]](s)


def _own(s):
    import paper_2407_00611_amd as st
    c = s["c"]
    cache = st.KVCache(s["k_cache"], s["v_cache"], s["table"], s["lens"], s.get("k_scale"), s.get("v_scale"))
    if c["op"] == "attn":
        o, lse = st.st_attn_cache(s["q"], s["starts"], cache, c["causal"], s["scale"], max_rows=_most_rows(c), window=c["window"],
                                  softcap=c["cap"], slopes=s["slopes"], q_first=s["q_first"], lowp=True)
        return {"o": o, "lse": lse}
    if c["op"] == "append":
        q = st.st_cache_append(s["q"], s["k"], s["v"], s["starts"], cache, s["freq"], offset=c["offset"], pairs=c["pairs"], norm=c["norm"],
                               q_weight=s["q_weight"], k_weight=s["k_weight"])
        k, v = st.st_cache_read(cache, s["first"], _count(c), dtype=s["q"].dtype)
        return {"q": q, "k": k, "v": v}
    k, v = st.st_cache_read(cache, s["first"], c["count"], dtype=_dtype(c["dtype"]))
    return {"k": k, "v": v}


def _tokens(s, name, places):
    """Values in 32 bits of the tokens at `places` [B, n] of every sequence (those past the table read its last page)."""
    c = s["c"]
    at = s["table"].gather(1, (places // c["page"]).clamp(max=s["table"].shape[1] - 1)).long()
    x = s[name + "_cache"][at, places % c["page"]].float()              # [B, n, Hkv, D]
    if c["cache"] == "e4m3":
        x = x * torch.exp2(s[name + "_scale"][at].float() - 127)[..., None]
    return x


def _plain_read(s):
    c = s["c"]
    places = s["first"].long()[:, None] + torch.arange(_count(c), device="cuda")
    there = (places < s["lens"][:, None])[:, :, None, None]
    return {name: torch.where(there, _tokens(s, name, places), 0).to(_dtype(c["dtype"])) for name in "kv"}


def _rows(s):
    """Sequence and number in it of every packed row."""
    t = torch.arange(sum(_counts(s["c"])), device="cuda")
    b = torch.searchsorted(s["starts"].long(), t, right=True) - 1
    return b, t - s["starts"].long()[b]


def _plain_append(s):
    c, dt = s["c"], _dtype(s["c"]["dtype"])
    b, i = _rows(s)
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    place = (s["lens"].long() - new)[b] + i
    angle = (place + c["offset"])[:, None].double() * s["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turned(x, w):
        x = x[0].float()
        if c["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        n, r = c["rot"] // 2, x[..., :c["rot"]]
        p, q = (r[..., :n], r[..., n:]) if c["pairs"] == "halves" else (r[..., 0::2], r[..., 1::2])
        y, z = p * cos - q * sin, p * sin + q * cos
        r = torch.cat([y, z], -1) if c["pairs"] == "halves" else torch.stack([y, z], -1).flatten(-2)
        return torch.cat([r, x[..., c["rot"]:]], -1)

    page = s["table"][b, place // c["page"]].long()
    for name, x in (("k", turned(s["k"], s["k_weight"])), ("v", s["v"][0].float())):
        cache = s[name + "_cache"]
        if c["cache"] != "e4m3":
            cache[page, place % c["page"]] = x.to(cache.dtype)
            continue
        scale, n_pages = s[name + "_scale"], cache.shape[0]
        top = torch.zeros((n_pages, c["Hkv"]), device="cuda").scatter_reduce_(0, page[:, None].expand(-1, c["Hkv"]), x.abs().amax(-1), "amax")
        # pages with new rows, and rows of theirs that were there before
        begun = torch.full((n_pages,), c["page"], device="cuda").scatter_reduce_(0, page, place % c["page"], "amin")
        touched = begun < c["page"]
        e_old = scale.int() - 127
        e = torch.where((begun > 0)[:, None], torch.maximum(e_old, _exponent(top)), _exponent(top))
        at = touched.nonzero()[:, 0]
        cache[at] = (cache[at].float() * torch.exp2((e_old - e)[at].float())[:, None, :, None]).to(cache.dtype)
        scale[at] = (e[at] + 127).to(torch.uint8)
        cache[page, place % c["page"]] = (x * torch.exp2(-e[page].float())[..., None]).to(cache.dtype)
    return {"q": turned(s["q"], s["q_weight"]).to(dt)[None], **_plain_read(s)}


def _plain_attention(s):
    c, dt = s["c"], _dtype(s["c"]["dtype"])
    B, Hkv, D, L, n, G = c["B"], c["Hkv"], c["D"], max(max(_lens(c)), 1), _most_rows(c), c["Hq"] // c["Hkv"]
    b, i = _rows(s)
    key = torch.arange(L, device="cuda")
    k, v = (_tokens(s, name, key.expand(B, -1)).permute(0, 2, 1, 3).contiguous() for name in "kv")    # [B, Hkv, L, D]
    q = torch.zeros((B, n, c["Hq"], D), device="cuda")
    q[b, i] = s["q"][0].float()
    q = q.unflatten(2, (Hkv, G)).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).unflatten(2, (G, n)) * s["scale"]             # [B, Hkv, G, n, L]
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    first = s["q_first"] if s["q_first"] is not None else s["lens"].long() - new
    pos = (first[:, None] + torch.arange(n, device="cuda"))[:, :, None]                                # [B, n, 1]
    if s["slopes"] is not None:
        x = x - s["slopes"].reshape(Hkv, G, 1, 1) * (pos - key).abs().float()[:, None, None]
    seen = (key < s["lens"][:, None, None]).expand(B, n, L)
    if c["causal"]:
        seen = seen & (key <= pos)
    if c["window"]:
        seen = seen & (pos - key < c["window"])
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1)
    # stale values of pages whose end no sequence has reached stay out
    v = torch.where((key < s["lens"][:, None])[:, None, :, None], v, 0)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (G, n)).permute(0, 3, 1, 2, 4).flatten(2, 3)     # [B, n, Hq, D]
    lse = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).flatten(2, 3)                           # [B, n, Hq]
    return {"o": o[b, i].to(dt)[None], "lse": lse[b, i].t()[None].contiguous()}


# ---------------------------------------------------------------------------------------------- from the definition, in 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    return {"attn": _exact_attention, "append": _exact_append, "read": _exact_read}[c["op"]](s)


def _e4m3_values():
    """The 256 values: sign, four bits of exponent (bias 7), three of mantissa; 2^-9 steps where the exponent is zero."""
    code = torch.arange(256, dtype=torch.float64)
    sign, low = torch.where(code >= 128, -1.0, 1.0), code % 128
    e, m = torch.div(low, 8, rounding_mode="floor"), low % 8
    x = sign * torch.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7), m * 2.0 ** -9)
    x[[127, 255]] = math.nan
    return x.cuda()


def _held(s, name, b):
    """[len, Hkv, D] in 64 bits: what the cache holds of sequence b."""
    c, n = s["c"], _lens(s["c"])[b]
    pages = s["table"][b, :(n + c["page"] - 1) // c["page"]].long()
    x = s[name + "_cache"][pages]
    if c["cache"] == "e4m3":
        x = _e4m3_values()[x.view(torch.uint8).long()] * (2.0 ** (s[name + "_scale"][pages].double() - 127))[:, None, :, None]
    return x.double().flatten(0, 1)[:n]


def _chunks(s, held):
    """Dense chunks from what the sequences hold."""
    c = s["c"]
    out = {name: torch.zeros((c["B"], _count(c), c["Hkv"], c["D"]), dtype=torch.float64, device="cuda") for name in "kv"}
    for b, f in enumerate(_first(c)):
        for name in "kv":
            x = held(name, b)[f:f + _count(c)]
            out[name][b, :x.shape[0]] = x
    return out


def _exact_read(s):
    return _chunks(s, lambda name, b: _held(s, name, b))


def _e4m3_near(x):
    """The nearest e4m3 value, ties to an even mantissa; |x| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    c = s["c"]
    n, at = _counts(c), 0
    first = torch.arange(c["rot"] // 2, device="cuda") * (1 if c["pairs"] == "halves" else 2)
    second = first + (c["rot"] // 2 if c["pairs"] == "halves" else 1)
    q_out, rows = [], {}
    for b in range(c["B"]):
        place = torch.arange(_lens(c)[b] - n[b], _lens(c)[b], device="cuda")
        angle = (place + c["offset"]).double()[:, None] * s["freq"]
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        for name in "qkv":
            x = s[name][0, at:at + n[b]].double()
            if name != "v":
                if c["norm"]:
                    x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * s[name + "_weight"].double()
                z = torch.complex(x[..., first], x[..., second]) * turn
                x = x.index_copy(-1, first, z.real).index_copy(-1, second, z.imag)
            if name == "q":
                q_out.append(x)
            else:
                rows[name, b] = x
        at += n[b]

    def held(name, b):
        x, had = _held(s, name, b), _lens(c)[b] - n[b]
        if c["cache"] != "e4m3":
            x[had:] = rows[name, b].to(_dtype(c["cache"])).double()
            return x
        for j in range(had // c["page"], (_lens(c)[b] - 1) // c["page"] + 1):
            lo, hi = j * c["page"], min((j + 1) * c["page"], _lens(c)[b])
            m = max(lo, had)
            y = rows[name, b][m - had:hi - had]
            e = torch.ceil(torch.log2(y.abs().amax((0, 2)) / 448)).clamp(-126, 127)
            if m > lo:
                e = torch.maximum(e, s[name + "_scale"][int(s["table"][b, j])].double() - 127)
            unit = (2.0 ** e)[:, None]
            x[lo:m] = _e4m3_near(x[lo:m] / unit) * unit
            x[m:hi] = _e4m3_near(y / unit) * unit
        return x

    return {"q": torch.cat(q_out)[None], **_chunks(s, held)}


def _exact_attention(s):
    """One sequence and KV head after the other."""
    c, at = s["c"], 0
    G, n, lens = c["Hq"] // c["Hkv"], _counts(c), _lens(c)
    T = sum(n)
    o = torch.zeros((1, T, c["Hq"], c["D"]), dtype=torch.float64, device="cuda")
    lse = torch.full((1, c["Hq"], T), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        k, v = _held(s, "k", b), _held(s, "v", b)
        p = torch.arange(n[b], device="cuda")[:, None] + (lens[b] + c["ahead"] if c["ahead"] else lens[b] - n[b])
        t = torch.arange(lens[b], device="cuda")
        hidden = torch.zeros((n[b], lens[b]), dtype=torch.bool, device="cuda")
        if c["causal"]:
            hidden = hidden | (t > p)
        if c["window"]:
            hidden = hidden | (t <= p - c["window"])
        for h in range(c["Hq"] if lens[b] else 0):
            x = s["q"][0, at:at + n[b], h].double() @ k[:, h // G].T * s["scale"]
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * (p - t).abs()
            x = x.masked_fill(hidden, -math.inf)
            norm = torch.logsumexp(x, 1)
            lse[0, h, at:at + n[b]] = norm
            some = torch.isfinite(norm)[:, None]
            o[0, at:at + n[b], h] = torch.where(some, torch.exp(x - torch.where(some, norm[:, None], 0)), 0) @ v[:, h // G]
        at += n[b]
    return {"o": o, "lse": lse}
