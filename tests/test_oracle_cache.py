"""Pins of the cache's oracle (CPU): the 8-bit values against torch's type, scales, pages, and attention against torch's softmax."""
import math

import torch

from oracle import cache as oc


def test_the_values_are_those_of_the_type():
    codes = torch.arange(256, dtype=torch.uint8)
    ours, theirs = oc.e4m3_values(), codes.view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.isnan(ours), torch.isnan(theirs)) and torch.equal(ours.nan_to_num(), theirs.nan_to_num())


def test_rounding_takes_the_nearest_and_even_ones():
    values = oc.e4m3_values()
    values = values[torch.isfinite(values)].unique()
    mid = (values[1:] + values[:-1]) / 2
    x = torch.cat([values, mid, mid + 1e-9, mid - 1e-9, torch.linspace(-448, 448, 10007, dtype=torch.float64)])
    near = oc.e4m3_near(x)
    assert torch.isin(near, values).all()
    assert torch.equal((near - x).abs(), (values[None] - x[:, None]).abs().min(1).values)
    assert torch.equal(near[:2 * len(values) - 1], x[:2 * len(values) - 1].float().to(torch.float8_e4m3fn).double())
    assert torch.isnan(oc.e4m3_near(torch.tensor([math.inf, -math.inf, math.nan]).double())).all()


def test_the_least_exponent():
    for top, e in ((448.0, 0), (448.1, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, -126), (1e-45, -126)):
        assert oc.least_exponent(torch.tensor([[top, -top / 2]], dtype=torch.float64)) == e, top
    assert oc.least_exponent(torch.tensor([math.inf, 1.0, math.nan]).double()) == -8


def test_appending_one_by_one_or_at_once():
    g = torch.Generator().manual_seed(1)
    rows = torch.randn((20, 2, 16), generator=g, dtype=torch.float64) * torch.exp2(torch.arange(20.0).double() / 4)[:, None, None]
    table, zero = torch.tensor([[2, 0]]), torch.zeros((3, 2), dtype=torch.int64)
    once, steps = (oc.Pages(torch.full((3, 16, 2, 16), math.nan), zero) for _ in range(2))
    once.append(table, [20], [0, 20], rows)
    for i in range(20):
        steps.append(table, [i + 1], [0, 1], rows[i:i + 1])
    a, there = once.held(table, [20], 0)
    b, _ = steps.held(table, [20], 0)
    assert there.all() and torch.equal(once.e, steps.e)
    # half a step of the least value twice over, of the page's last scale
    assert (a - b).abs().max() <= 2.0 ** -9 * 2.0 ** int(once.e.max())
    assert ((a - rows).abs() <= 2.0 ** -4 * rows.abs() + 2.0 ** -10 * torch.exp2(once.e.double())[[2] * 16 + [0] * 4][..., None]).all()


def test_tokens_of_no_page_are_dropped():
    pages = oc.Pages(torch.zeros((2, 16, 1, 8)))
    table = torch.tensor([[1, -1, 5]])
    pages.append(table, [60], [0, 60], torch.ones((60, 1, 8)))
    x, there = pages.held(table, [60], 0)
    assert x.shape[0] == 48 and there.sum() == 16 and x.sum() == 16 * 8 and pages.x[0].sum() == 0


def test_attention_is_a_softmax():
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 4, 8), (10, 2, 8), (10, 2, 8)))
    there = torch.ones(10, dtype=torch.bool)
    o, lse, _, _ = oc.attention(q, k, v, there, [7, 8, 9], True, 0.3)
    s = torch.einsum("ihd,thd->hit", q, k.repeat_interleave(2, 1)) * 0.3
    s = s.masked_fill(torch.arange(10)[None, None] > torch.tensor([7, 8, 9])[None, :, None], -math.inf)
    assert torch.allclose(o, torch.einsum("hit,thd->ihd", s.softmax(-1), v.repeat_interleave(2, 1)))
    assert torch.allclose(lse, s.logsumexp(-1).t())
    o, lse, _, _ = oc.attention(q, k, v, there, [50, 51, 52], True, 0.3, window=20)
    assert (o == 0).all() and (lse == -math.inf).all()
    one, _, _, _ = oc.attention(q, k, v, there, [9, 9, 9], True, 0.3, window=1)
    assert torch.allclose(one, v[9].repeat_interleave(2, 0).expand(3, 4, 8))
