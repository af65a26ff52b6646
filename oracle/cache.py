"""A cache of keys and values in pages, and the attention that reads it, in 64 bits, from the definitions, one token after the other
(torch float64 on the CPU; test infrastructure, shares no code with the kernels)."""
import math

import torch


def e4m3_values():
    """The 256 values by code: sign, four bits of exponent (bias 7), three of mantissa; 127 and 255 are NaN."""
    out = []
    for code in range(256):
        e, m = code % 128 // 8, code % 8
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m * 2.0 ** -9
        out.append(math.nan if code % 128 == 127 else -x if code >= 128 else x)
    return torch.tensor(out, dtype=torch.float64)


def e4m3_near(x):
    """The nearest of those values, ties to an even last bit (|x| <= 448, or not finite: NaN)."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.where(torch.isfinite(x), torch.round(x / step) * step, math.nan)


def least_exponent(rows):
    """The least e (not below -126) with every finite |x| <= 448 2^e."""
    top = float(torch.where(torch.isfinite(rows), rows.abs(), 0.0).max()) if rows.numel() else 0.0
    e = -126
    while top > 448 * 2.0 ** e:
        e += 1
    return e


class Pages:
    """Keys or values of a cache: [n_pages, page, Hkv, D] values less their scale, and the exponents of the scales."""

    def __init__(self, values, exponents=None):
        self.x, self.e = values.double().clone(), exponents.clone() if exponents is not None else None

    def append(self, table, lens, starts, rows):
        """rows [T, Hkv, D]: as they would be without any rounding but the page's."""
        n_pages, page, heads, _ = self.x.shape
        for b in range(len(lens)):
            n, pieces = int(starts[b + 1] - starts[b]), {}
            for i in range(n):
                token = int(lens[b]) - n + i
                if token < 0 or token // page >= table.shape[1] or not 0 <= int(table[b, token // page]) < n_pages:
                    continue
                pieces.setdefault(token // page, []).append((token % page, int(starts[b]) + i))
            for j, piece in pieces.items():
                at = int(table[b, j])
                begun = piece[0][0]
                for h in range(heads):
                    new = torch.stack([rows[t, h] for _, t in piece]).double()
                    if self.e is None:
                        for (r, _), x in zip(piece, new):
                            self.x[at, r, h] = x
                        continue
                    e = least_exponent(new)
                    if begun:
                        had = int(self.e[at, h])
                        e = max(e, had)
                        if e > had:
                            self.x[at, :begun, h] = e4m3_near(self.x[at, :begun, h] * 2.0 ** (had - e))
                    self.e[at, h] = e
                    for (r, _), x in zip(piece, new):
                        self.x[at, r, h] = e4m3_near(x * 2.0 ** -e)

    def held(self, table, lens, b):
        """[len, Hkv, D], and which of the tokens are there."""
        n_pages, page, heads, D = self.x.shape
        n = max(0, min(int(lens[b]), table.shape[1] * page))
        out, there = torch.zeros((n, heads, D), dtype=torch.float64), torch.zeros(n, dtype=torch.bool)
        for x in range(n):
            at = int(table[b, x // page])
            if 0 <= at < n_pages:
                there[x] = True
                out[x] = self.x[at, x % page]
                if self.e is not None:
                    out[x] *= torch.exp2(self.e[at].double())[:, None]
        return out, there


def attention(q, k, v, there, positions, causal, scale, window=0, cap=0.0, slopes=None):
    """Rows q [n, Hq, D] of one sequence at `positions` against its tokens k, v [len, Hkv, D]: O [n, Hq, D], lse [n, Hq], and for bounds of
    errors sum p |v| [n, Hq, D] and the largest sum |q k| scale that a row meets [n, Hq]."""
    n, heads, D = q.shape
    o, mass = torch.zeros((2, n, heads, D), dtype=torch.float64)
    lse, size = torch.full((n, heads), -math.inf, dtype=torch.float64), torch.zeros((n, heads), dtype=torch.float64)
    token = torch.arange(k.shape[0])
    for i in range(n):
        p = int(positions[i])
        seen = there.clone()
        if causal:
            seen &= token <= p
        if window:
            seen &= p - token < window
        if not seen.any():
            continue
        for h in range(heads):
            kk, vv = k[seen, h * k.shape[1] // heads], v[seen, h * k.shape[1] // heads]
            s = kk @ q[i, h].double() * scale
            if cap:
                s = cap * torch.tanh(s / cap)
            if slopes is not None:
                s = s - float(slopes[h]) * (p - token[seen]).abs().double()
            lse[i, h] = torch.logsumexp(s, 0)
            w = torch.exp(s - lse[i, h])
            o[i, h], mass[i, h] = w @ vv, w @ vv.abs()
            size[i, h] = (kk.abs() @ q[i, h].double().abs()).max() * scale
    return o, lse, mass, size
