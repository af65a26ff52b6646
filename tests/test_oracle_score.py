"""Pins of the 64-bit oracle of attention with modified scores and of norms with rotations (CPU)."""
import math

import pytest
import torch

from oracle import score as so


def _case(seed=0, B=2, Hq=4, Hkv=2, Sq=9, Sk=13, D=8):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    return r(B, Sq, Hq, D), r(B, Sk, Hkv, D), r(B, Sk, Hkv, D), r(B, Sq, Hq, D)


@pytest.mark.parametrize("causal,cap,slope", [(False, 0.0, False), (True, 2.0, True), (True, 0.0, True), (False, 1.5, False)])
def test_forward_is_the_loop_over_rows_and_keys(causal, cap, slope):
    q, k, v, _ = _case()
    pos, kpos = torch.arange(9) + 6, torch.arange(13) + 2
    slopes = torch.tensor([0.5, 0.25, 0.125, 0.0625]) if slope else None
    span = torch.tensor([[(int(p) % 5, int(p) + 3 * (b + 1)) for p in pos] for b in range(2)])
    o, lse = so.forward(q, k, v, pos, kpos, causal, 0.3, cap, slopes, span)
    for b in range(2):
        for h in range(4):
            for i in range(9):
                s, rows = [], []
                for t in range(13):
                    if not (span[b, i, 0] <= kpos[t] < span[b, i, 1]) or (causal and kpos[t] > pos[i]):
                        continue
                    x = 0.3 * float(q[b, i, h] @ k[b, t, h // 2])
                    x = cap * math.tanh(x / cap) if cap else x
                    s.append(x - (float(slopes[h]) * abs(int(pos[i]) - int(kpos[t])) if slope else 0))
                    rows.append(v[b, t, h // 2])
                if not s:
                    assert lse[b, h, i] == -math.inf and not o[b, i, h].any()
                    continue
                z = sum(math.exp(x) for x in s)
                assert abs(float(lse[b, h, i]) - math.log(z)) < 1e-12
                assert torch.allclose(o[b, i, h], sum(math.exp(x) / z * y for x, y in zip(s, rows)), atol=1e-12)


def test_backward_is_the_derivative():
    q, k, v, d_o = (x.requires_grad_() for x in _case(1))
    pos, kpos = torch.arange(9) + 4, torch.arange(13)
    span = torch.stack([torch.zeros(2, 9, dtype=torch.int64), pos.expand(2, -1) - torch.arange(9) % 4], -1)
    mods = dict(cap=1.2, slopes=torch.tensor([0.3, 0.2, 0.1, 0.05]), span=span)
    o, lse = so.forward(q, k, v, pos, kpos, True, 0.4, **mods)
    (o * d_o).sum().backward()
    dq, dk, dv = so.backward(q.detach(), k.detach(), v.detach(), d_o.detach(), lse.detach(), so.delta(d_o.detach(), o.detach()), pos, kpos, True, 0.4, **mods)
    for x, y in ((q.grad, dq), (k.grad, dk), (v.grad, dv)):
        assert torch.allclose(x, y, atol=1e-12)
    # and a difference quotient of one element
    with torch.no_grad():
        def loss(step):
            z = q.detach().clone()
            z[1, 3, 2, 5] += step
            return float((so.forward(z, k, v, pos, kpos, True, 0.4, **mods)[0] * d_o).sum())
        assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - float(dq[1, 3, 2, 5])) < 1e-8


def test_spans_of_documents_and_prefixes():
    got = so.spans([[2, 5, 5, 9]], [0, 2, 4, 5, 7, 8, 9], True, [[2, 0, 3]])[0]
    assert got == [(0, 0), (2, 4), (2, 5), (5, 8), (5, 8), (5, 9), (0, 0)]
    assert so.spans([[2, 5, 5, 9]], [4, 6], False)[0] == [(2, 5), (5, 9)]


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_rope_is_a_rotation_by_position(pairs):
    g = torch.Generator().manual_seed(3)
    x = torch.randn((1, 5, 2, 12), generator=g, dtype=torch.float64)
    freq = torch.tensor([1.0, 0.5, 0.25, 0.1], dtype=torch.float64)
    at = lambda p: so.rope(x, None, freq, torch.full((4, 1, 5), p), pairs, False)
    assert torch.equal(at(0), x)
    assert torch.allclose(at(7).square().sum(-1), x.square().sum(-1))
    # products of rotated vectors depend on the difference of the positions alone
    assert torch.allclose((at(7) * at(3)).sum(-1), (at(104) * at(100)).sum(-1))
    i = (1, 2 if pairs == "neighbours" else 1, 3 if pairs == "neighbours" else 5)
    y = at(3)[0, 0, 0]
    t = 3 * 0.5
    assert abs(float(y[i[1]]) - float(x[0, 0, 0, i[1]] * math.cos(t) - x[0, 0, 0, i[2]] * math.sin(t))) < 1e-12
    n = so.rope(x, torch.full((12,), 2.0), freq, torch.zeros((4, 1, 5)), pairs, True, 0.0)
    assert torch.allclose(n.square().mean(-1), torch.full((1, 5, 2), 4.0, dtype=torch.float64))
