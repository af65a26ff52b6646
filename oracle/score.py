"""Attention with modified scores and the norms and rotations of its queries and keys, in 64 bits, from the definitions
(torch float64, on whatever device the inputs are; test infrastructure, shares no code with the kernels)."""
import math

import torch


def spans(bounds, positions, causal, prefix=None):
    """Row spans of packed documents, row by row: [B, Sq, 2] nested lists of positions."""
    out = []
    for b, ends in enumerate(bounds):
        rows = []
        for p in positions:
            span = (0, 0)
            for d in range(len(ends) - 1):
                if ends[d] <= p < ends[d + 1]:
                    hi = ends[d + 1]
                    if causal:
                        first = ends[d] + (prefix[b][d] if prefix is not None else 0)
                        hi = min(hi, max(p + 1, first))
                    span = (ends[d], hi)
            rows.append(span)
        out.append(rows)
    return out


def visible(positions, key_positions, causal, span=None):
    """[B or 1, Sq, Sk]; span int64 [B, Sq, 2] or None."""
    i, t = positions[:, None], key_positions[None, :]
    seen = (t <= i) if causal else torch.ones((len(positions), len(key_positions)), dtype=torch.bool, device=positions.device)
    seen = seen[None]
    if span is not None:
        seen = seen & (key_positions >= span[..., 0:1]) & (key_positions < span[..., 1:2])
    return seen


def _wide(x, heads):
    x = x.double().transpose(1, 2)
    return x.repeat_interleave(heads // x.shape[1], dim=1).contiguous()


def _scores(q, k, positions, key_positions, seen, scale, cap, slopes):
    u = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    t = torch.tanh(u / cap) if cap else None
    s = cap * t if cap else u
    if slopes is not None:
        s = s - slopes.double()[None, :, None, None] * (positions[:, None] - key_positions[None, :]).abs().double()
    return torch.where(seen[:, None], s, -math.inf), (1 - t * t if cap else None)


def forward(q, k, v, positions, key_positions, causal, scale, cap=0.0, slopes=None, span=None):
    """O [B,Sq,Hq,D] and lse [B,Hq,Sq]."""
    heads = q.shape[2]
    s, _ = _scores(_wide(q, heads), _wide(k, heads), positions, key_positions, visible(positions, key_positions, causal, span), scale, cap, slopes)
    lse = torch.logsumexp(s, 3) if s.shape[3] else torch.full(s.shape[:3], -math.inf, dtype=torch.float64, device=s.device)
    p = torch.where(s == -math.inf, 0.0, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None]))
    return torch.matmul(p, _wide(v, heads)).transpose(1, 2), lse


def backward(q, k, v, d_o, lse, delta, positions, key_positions, causal, scale, cap=0.0, slopes=None, span=None):
    """dQ [B,Sq,Hq,D], dK and dV [B,Sk,Hkv,D], from the final lse and Delta."""
    heads, kv_heads = q.shape[2], k.shape[2]
    Q, K, V, dO = (_wide(x, heads) for x in (q, k, v, d_o))
    s, bend = _scores(Q, K, positions, key_positions, visible(positions, key_positions, causal, span), scale, cap, slopes)
    l = lse.double()[..., None]
    p = torch.where((s == -math.inf) | (l == -math.inf), 0.0, torch.exp(s - torch.where(l == -math.inf, 0.0, l)))
    ds = p * (torch.matmul(dO, V.transpose(2, 3).contiguous()) - delta.double()[..., None])
    if bend is not None:
        ds = ds * bend
    ds = ds * scale
    fold = lambda x: x.unflatten(1, (kv_heads, heads // kv_heads)).sum(2).transpose(1, 2)
    return (torch.matmul(ds, K).transpose(1, 2), fold(torch.matmul(ds.transpose(2, 3).contiguous(), Q)),
            fold(torch.matmul(p.transpose(2, 3).contiguous(), dO)))


def magnitudes(q, k, v, d_o, lse, positions, key_positions, causal, scale, cap=0.0, slopes=None, span=None):
    """Of every element of O, dQ, dK and dV the sum of the sizes of the terms that make it: what a relative error of each term is
    taken of.  A score's gradient has the terms P |dO| |V| (of dP) and P |dO| sum P |V| (of Delta)."""
    heads, kv_heads = q.shape[2], k.shape[2]
    Q, K, V, dO = (_wide(x, heads) for x in (q, k, v, d_o))
    s, _ = _scores(Q, K, positions, key_positions, visible(positions, key_positions, causal, span), scale, cap, slopes)
    l = lse.double()[..., None]
    p = torch.where((s == -math.inf) | (l == -math.inf), 0.0, torch.exp(s - torch.where(l == -math.inf, 0.0, l)))
    Q, K, V, dO = Q.abs(), K.abs(), V.abs(), dO.abs()
    o = torch.matmul(p, V)
    ds = scale * p * (torch.matmul(dO, V.transpose(2, 3).contiguous()) + (dO * o).sum(3, keepdim=True))
    fold = lambda x: x.unflatten(1, (kv_heads, heads // kv_heads)).sum(2).transpose(1, 2)
    return (o.transpose(1, 2), torch.matmul(ds, K).transpose(1, 2), fold(torch.matmul(ds.transpose(2, 3).contiguous(), Q)),
            fold(torch.matmul(p.transpose(2, 3).contiguous(), dO)))


def delta(d_o, o):
    return (d_o.double() * o.double()).sum(3).transpose(1, 2)


def rope(x, weight, freq, positions, pairs, norm, eps=1e-6):
    """x [B,S,H,D]; positions [n, B, S] with one row for every pair, freq [n]."""
    y = x.double()
    if norm:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * weight.double()
    n = len(freq)
    first = torch.arange(n, device=x.device) * (2 if pairs == "neighbours" else 1)
    second = first + (1 if pairs == "neighbours" else n)
    t = (positions.double() * freq.double()[:, None, None]).permute(1, 2, 0)[:, :, None]
    a, b = y[..., first], y[..., second]
    y = y.index_copy(-1, first, a * torch.cos(t) - b * torch.sin(t))
    return y.index_copy(-1, second, a * torch.sin(t) + b * torch.cos(t))
