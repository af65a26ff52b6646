"""Appending to a cache of pages and reading chunks of it (st_cache_append, st_cache_read) against the 64-bit oracle.

What is stored has to be the oracle's, bit by bit, in 8 bits (keys are made in 64 bits there, and two evaluations in 64 bits that differ
by 2^-50 round to one e4m3 value but for one in 2^-45) and for values, which are copied; keys in fp32 and queries are fp32 arithmetic
rounded once, with the tolerances of st_qk_rope_fwd's tests (keys in bf16, made in 64 bits too, are within them)."""
import math

import pytest
import torch

import paper_2407_00611_amd as st
from cache_cases import TYPES, Case, rows_of
from oracle import score as so

pytestmark = pytest.mark.gpu


def _near(x, ref, dtype, what):
    x, ref = x.double().cpu(), ref.double().cpu()
    assert x.shape == ref.shape and torch.equal(torch.isfinite(x), torch.isfinite(ref)), what
    norm = float(ref.norm())
    rms = norm / math.sqrt(max(ref.numel(), 1))
    assert float((x - ref).norm()) <= (2e-6 if dtype == torch.float32 else 2.0 ** -8) * norm + 1e-12, what
    worst = float(((x - ref).abs() / ref.abs().clamp(min=rms + 1e-30)).max()) if ref.numel() else 0.0
    assert worst <= (2e-5 if dtype == torch.float32 else 2.0 ** -8 + 2e-5), f"{what}: an element {worst:.3e} off"


def _stored(case, i):
    x = (case.k, case.v)[i].double().cpu()
    return x, case.scales[i].cpu().int() - 127 if case.scales[i] is not None else None


def _check_pages(case, rows, starts, lens, dtype, table=None):
    table = case.table if table is None else table
    for i, x in enumerate(rows):
        case.oracle[i].append(table, lens, starts, x.cpu())
        got, e = _stored(case, i)
        want = case.oracle[i].x
        if e is not None:
            assert torch.equal(e.long(), case.oracle[i].e), "scales"
        if case.kind == "e4m3" or i == 1:
            assert int((torch.isnan(got) != torch.isnan(want)).sum()) == 0, "kv"[i]
            if case.kind != "e4m3":
                want = want.to(dtype).double()
            differ = (got.nan_to_num(0.0) != want.nan_to_num(0.0)).sum()
            assert differ == 0, f"{'kv'[i]}: {differ} values differ"
        else:
            keep = torch.isnan(want)
            assert torch.equal(torch.isnan(got), keep)
            _near(got.nan_to_num(0.0), want.nan_to_num(0.0), dtype, "k")
            case.oracle[i].x = torch.where(keep, torch.nan, got)


def _append(dtype, kind, lens, counts, page=16, Hq=4, Hkv=2, D=64, rot=None, pairs="halves", norm=True, weights=True, offset=0, layout="dense", axes=None,
            rows="dense", grow=0.0, more_rows=0, in_place=False, seed=0):
    dt = TYPES[dtype]
    case = Case(seed, kind, [n - c for n, c in zip(lens, counts)], page, Hkv, D, layout, more=-(-max(counts) // page) + 1)
    g, T = case.g, sum(counts) + more_rows
    r = lambda *s: torch.randn(s, generator=g)
    if rows == "packed":
        q, k, v = r(1, T, Hq + 2 * Hkv, D).to(dt).cuda().split([Hq, Hkv, Hkv], 2)
    elif rows == "heads_first":
        q, k, v = (r(1, h, T, D).to(dt).cuda().transpose(1, 2) for h in (max(Hq, 1), Hkv, Hkv))
    else:
        q, k, v = (r(1, T, h, D).to(dt).cuda() for h in (max(Hq, 1), Hkv, Hkv))
    if grow:
        k, v = (x * torch.exp2(torch.arange(T, device="cuda") * grow)[None, :, None, None].to(dt) for x in (k, v))
    if not Hq:
        q = None
    rot = D if rot is None else rot
    freq = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))).cuda()
    wq, wk = ((1 + 0.3 * r(D)).cuda() if norm and weights else None for _ in range(2))
    starts = rows_of(counts)
    place = torch.zeros(T, dtype=torch.int64)
    for b, c in enumerate(counts):
        place[int(starts[b]):int(starts[b]) + c] = torch.arange(lens[b] - c, lens[b]) + offset
    table, each = None, place.expand(rot // 2, 1, T).cuda()
    if axes is not None:
        table = torch.randint(-50, 100000, (len(axes), 1, T), generator=g, dtype=torch.int32).cuda()
        each = table.long()[torch.repeat_interleave(torch.arange(len(axes)), torch.tensor(axes)).cuda()]
    print(f"[{dtype} in {kind}, {lens} by {counts}, page {page}, {Hq}/{Hkv} D{D} rot {rot} {axes} {pairs} norm {norm} {layout} {rows}]", flush=True)
    before, held = (q.clone(), q) if q is not None else (None, None)
    how = dict(offset=offset, positions=table, axes=axes, pairs=pairs, norm=norm, q_weight=wq if Hq else None, k_weight=wk)
    cache = case.cache(lens)
    q_out = held if in_place else torch.full_like(held, 7.0) if held is not None else None
    got = st.st_cache_append(q, k, v, starts.cuda(), cache, freq, q_out=q_out, **how)
    n = sum(counts)
    exact = lambda x, w: so.rope(x.double(), w.double() if w is not None else None, freq, each, pairs, norm)
    if Hq:
        assert got is q_out
        _near(got[:, :n], exact(before, wq)[:, :n], dt, "q")
        assert torch.equal(got[:, n:], (before if in_place else torch.full_like(before, 7.0))[:, n:]), "rows of no sequence"
    else:
        assert got is None
    new = [exact(k, wk)[0], v[0].double()]
    _check_pages(case, new, starts, lens, dt)
    if not in_place:                                 # once more: nothing changes
        pages = [case.k.clone(), case.v.clone()] + [s.clone() for s in case.scales if s is not None]
        again = st.st_cache_append(q, k, v, starts.cuda(), cache, freq, **how)
        bits = lambda x: x.contiguous().view(torch.uint8)
        for x, y in zip([case.k, case.v] + [s for s in case.scales if s is not None], pages):
            assert torch.equal(bits(x), bits(y))
        if Hq:
            assert torch.equal(again[:, :n], got[:, :n])
    return case, cache


APPENDS = [
    dict(lens=[1], counts=[1]),
    dict(lens=[16, 17, 5], counts=[1, 1, 1]),                                     # the last row of a page, the first, one inside
    dict(lens=[40, 7, 33], counts=[20, 0, 33], page=16, grow=0.25),               # whole pages, a sequence that gets none, scales that grow
    dict(lens=[300], counts=[270], page=256, Hq=3, Hkv=1, D=128, rows="packed"),
    dict(lens=[100, 70], counts=[70, 70], page=32, Hq=12, Hkv=4, D=80, rot=40, pairs="neighbours", offset=500000, grow=-0.1),
    dict(lens=[64], counts=[64], page=64, Hq=0, D=128, norm=False),
    dict(lens=[20, 40], counts=[3, 5], page=128, Hq=32, Hkv=8, D=128, layout="heads_first", more_rows=4),
    dict(lens=[20, 40], counts=[3, 5], Hq=2, Hkv=1, D=256, rot=250, layout="together", weights=False),
    dict(lens=[50], counts=[37], D=32, rot=0, norm=False, rows="heads_first"),
    dict(lens=[50, 60], counts=[7, 9], D=96, axes=[12, 20, 16], in_place=True),
    dict(lens=[2 ** 5] * 300, counts=[1] * 300, Hq=1, Hkv=1, D=32),               # more sequences than a workgroup has threads
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
@pytest.mark.parametrize("dtype,kind", [("bf16", "e4m3"), ("bf16", "bf16"), ("f32", "e4m3"), ("f32", "f32")])
def test_appending(dtype, kind, case):
    _append(dtype, kind, seed=case, **APPENDS[case])


@pytest.mark.parametrize("pairs,rot", [("halves", 128), ("neighbours", 64)])
def test_bf16_keys_are_those_of_64_bits(pairs, rot):
    """Made in 64 bits, to fp32, to bf16: two evaluations in 64 bits that differ by 2^-48 end in one value but for one in 2^-24 (of fp32
    steps) by 2^-16 (where that step is a tie of bf16); of 2^18 values none differ."""
    g, T, D, offset = torch.Generator().manual_seed(40), 512, 128, 100000
    q, k, v = (torch.randn((1, T, 4, D), generator=g).bfloat16().cuda() for _ in range(3))
    w = (1 + 0.3 * torch.randn(D, generator=g)).cuda()
    freq = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).cuda()
    case = Case(41, "bf16", [0], 64, 4, D, more=T // 64)
    cache = case.cache([T])
    st.st_cache_append(q, k, v, rows_of([T]).cuda(), cache, freq, offset=offset, pairs=pairs, q_weight=w, k_weight=w)
    place = (torch.arange(T, dtype=torch.int64) + offset).expand(rot // 2, 1, T).cuda()
    want = so.rope(k.double(), w.double(), freq, place, pairs, True).float().bfloat16()
    got, _ = st.st_cache_read(cache, None, T)
    assert torch.equal(got, want.to(got.device))


def test_one_by_one_and_growing():
    """A page filled by single tokens: its scale grows, and the rows that are there with it."""
    case = Case(3, "e4m3", [0, 5], 16, 2, 64, more=3)
    freq = torch.zeros(0, dtype=torch.float64).cuda()
    starts = rows_of([1, 1])
    for i in range(20):
        lens = [1 + i, 6 + i]
        k, v = (torch.randn((1, 2, 2, 64), generator=case.g).mul(2.0 ** (i / 3 - 4)).bfloat16().cuda() for _ in range(2))
        st.st_cache_append(None, k, v, starts.cuda(), case.cache(lens), freq, norm=False)
        _check_pages(case, [k[0].double(), v[0].double()], starts, lens, torch.bfloat16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite_and_far_ones(dtype):
    dt = TYPES[dtype]
    case = Case(4, "e4m3", [3], 16, 1, 64)
    k, v = (torch.randn((1, 8, 1, 64), generator=case.g).to(dt).cuda() for _ in range(2))
    k[0, 1, 0, 3], k[0, 2, 0, 5], v[0, 4, 0, 7], v[0, 5] = math.inf, math.nan, -math.inf, 0
    v[0, 6], k[0, 7] = 3e38, 1e-38
    freq = torch.zeros(0, dtype=torch.float64).cuda()
    st.st_cache_append(None, k, v, rows_of([8]).cuda(), case.cache([11]), freq, norm=False)
    _check_pages(case, [k[0].double(), v[0].double()], rows_of([8]), [11], dt)
    case = Case(5, "e4m3", [0], 16, 1, 64)                                        # nothing but zeros, and then something
    z = torch.zeros((1, 4, 1, 64), dtype=dt).cuda()
    st.st_cache_append(None, z, z, rows_of([4]).cuda(), case.cache([4]), freq, norm=False)
    _check_pages(case, [z[0].double()] * 2, rows_of([4]), [4], dt)
    st.st_cache_append(None, k[:, :1], v[:, :1], rows_of([1]).cuda(), case.cache([5]), freq, norm=False)
    _check_pages(case, [k[0, :1].double(), v[0, :1].double()], rows_of([1]), [5], dt)


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_places_without_a_page(kind):
    """Pages that the table does not name, tokens behind its end and before the sequence's beginning: dropped, and nothing else is touched."""
    case = Case(6, kind, [0, 0, 0], 16, 2, 64, more=3)
    table = case.table.clone()
    table[0, 1], table[1, 0] = -1, 10 ** 6
    lens, counts = [40, 30, 2], [40, 20, 5]                                       # the last: more rows than tokens
    k, v = (torch.randn((1, 65, 2, 64), generator=case.g).bfloat16().cuda() for _ in range(2))
    freq = torch.zeros(0, dtype=torch.float64).cuda()
    st.st_cache_append(None, k, v, rows_of(counts).cuda(), case.cache(lens, table), freq, norm=False)
    _check_pages(case, [k[0].double(), v[0].double()], rows_of(counts), lens, torch.bfloat16, table)
    wide = Case(7, kind, [0], 16, 2, 64, more=1)                                  # a table of two pages, 50 tokens
    st.st_cache_append(None, k[:, :50], v[:, :50], rows_of([50]).cuda(), wide.cache([50]), freq, norm=False)
    _check_pages(wide, [k[0].double(), v[0].double()], rows_of([50]), [50], torch.bfloat16)


@pytest.mark.parametrize("kind,dtype", [("e4m3", "bf16"), ("e4m3", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("page,Hkv,D,layout", [(16, 2, 64, "dense"), (64, 3, 80, "heads_first"), (256, 1, 256, "together")])
def test_reading(kind, dtype, page, Hkv, D, layout):
    lens = [0, 1, 37, 300, 64]
    case = Case(8, kind, lens, page, Hkv, D, layout)
    table = case.table.clone()
    table[3, 0] = -5
    dt = TYPES[dtype]
    for first, count in (([0, 0, 0, 0, 0], 300), ([0, 5, 36, 17, -3], 9), (None, 1)):
        outs = torch.full((5, count, 2 * Hkv, D), 7.0, dtype=dt, device="cuda").split(Hkv, 2)
        f = torch.tensor(first, dtype=torch.int32).cuda() if first is not None else None
        k, v = st.st_cache_read(case.cache(table=table), f, count, dtype=dt)
        st.st_cache_read(case.cache(table=table), f, count, k_out=outs[0], v_out=outs[1])
        assert torch.equal(outs[0], k) and torch.equal(outs[1], v)
        for i, x in enumerate((k, v)):
            for b in range(5):
                held = case.held(b, table=table)[i]
                want = torch.zeros((count, Hkv, D), dtype=torch.float64)
                for y in range(count):
                    token = y + (first[b] if first is not None else 0)
                    if 0 <= token < lens[b]:
                        want[y] = held[token]
                assert torch.equal(x[b].double().cpu(), want), (b, "kv"[i])
