"""Where a cache's attention and appending can go wrong at the ends of what they take: scales of pages without a token, infinities and NaN
wherever they lie, values beyond fp32, pages of the highest scales, keys beside a tie, scores near the
ends of fp32, probabilities in two parts whatever the batch."""
import math

import numpy as np
import pytest
import torch

import paper_2407_00611_amd as st
from cache_cases import TYPES, Case, check_attention, rows_of
from test_gpu_cache_attn import _attend

pytestmark = pytest.mark.gpu


# ---- scales of pages that hold no token

@pytest.mark.parametrize("byte", [255, 0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_scales_of_pages_without_a_token_are_not_used(dtype, D, byte):
    """What a program has not set yet: of the page behind a sequence's end, in the same block of keys, and of page 0, which stands in for
    those that are not there."""
    seed = next(s for s in range(200) if 0 not in torch.randperm(10, generator=torch.Generator().manual_seed(s))[[0, 1, 2, 4, 5, 6]])
    change = lambda case: case.spoil_scales(byte)
    for counts in ([1, 1], [5, 3], [40, 20], [41, 1]):
        how = dict(Hq=4, Hkv=1, D=D, seed=seed, change=change)
        case, *_ = _attend(dtype, "e4m3", [41, 33], counts, **how)
        assert not (case.scales[0][0] != byte).any()
        table = case.table.clone()
        table[0, 1], table[1, 0] = -1, 10 ** 6
        _attend(dtype, "e4m3", [41, 33], counts, table=table, **how)
        _attend(dtype, "e4m3", [41, 33], counts, causal=False, window=20, **how)
    how = dict(Hq=4, Hkv=1, D=D, change=change)
    _attend(dtype, "e4m3", [200, 130], [110, 90], **how)
    _attend(dtype, "e4m3", [5001, 1200], [1, 1], **how)                           # walks in shares


# ---- infinities and NaN, wherever the token lies

def _plant(case, token, d, x, b=0):
    case.v[int(case.table[b, token // case.page]), token % case.page, 0, d] = torch.tensor(x, device="cuda").to(case.v.dtype)


WALKS = [(400, 1), (400, 3), (400, 20), (5000, 1), (5000, 7), (20000, 2), (400, 100), (3000, 90)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,n", WALKS)
def test_an_infinity_is_one_wherever_its_token_lies(dtype, L, n):
    """Early tokens, which all rows see, and one at the edge of what they see: a row has what the definition says in the columns that such a
    token has, and in the others, bit by bit, what it has without."""
    D = 64
    case = Case(21, dtype, [L], 16, 1, D)
    q = torch.randn((1, n, 4, D), generator=case.g).to(TYPES[dtype]).cuda()
    print(f"[{dtype}, {n} rows of {L}]", flush=True)
    run = lambda: st.st_attn_cache(q, rows_of([n]).cuda(), case.cache(), True, 0.125)
    o0, l0 = run()
    edge = L - (n + 1) // 2                                                      # seen by the last rows only
    for token, d, x in ((40, 3, math.inf), (41, 60, -math.inf), (17, 9, math.inf), (300, 9, math.inf), (90, 10, math.inf), (L - n - 1, 10, -math.inf),
                        (100, 11, math.nan), (101, 11, math.inf), (edge, 12, math.inf), (5, 13, math.inf), (edge, 13, -math.inf)):
        _plant(case, token, d, x)
    o, lse = run()
    assert torch.equal(lse, l0)
    late = (torch.arange(n, device="cuda") >= edge - (L - n))[:, None].expand(n, 4)
    assert (o[0, :, :, 3] == math.inf).all() and (o[0, :, :, 60] == -math.inf).all() and (o[0, :, :, 9] == math.inf).all()
    assert torch.isnan(o[0, :, :, 10]).all() and torch.isnan(o[0, :, :, 11]).all()
    assert (o[0, :, :, 12][late] == math.inf).all() and torch.isfinite(o[0, :, :, 12][~late]).all()
    assert torch.isnan(o[0, :, :, 13][late]).all() and (o[0, :, :, 13][~late] == math.inf).all()
    keep = torch.ones(D, dtype=torch.bool, device="cuda")
    keep[[3, 60, 9, 10, 11, 12, 13]] = False
    # (tiles of prompts at the edge take another way: no more than its roundings apart)
    if n * 4 > 256 and dtype == "bf16":
        assert float((o[..., keep] - o0[..., keep]).abs().max()) <= 2.0 ** -8 * float(o0[..., keep].abs().max())
    else:
        assert torch.equal(o[..., keep], o0[..., keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 150.0])
@pytest.mark.parametrize("L,n", WALKS)
def test_an_infinity_of_no_weight_to_speak_of(dtype, cap, L, n):
    """A token whose probability is e^-120 and less, no number of fp32: what is infinite times it is infinite all the same."""
    D = 64
    case = Case(22, dtype, [L], 16, 1, D)
    q = torch.randn((1, n, 4, D), generator=case.g)
    q[..., 0] = 16.0
    q = q.to(TYPES[dtype]).cuda()
    case.k[..., 0] = 0.0
    tokens = (40, L // 2, L - n - 1, L - n)
    for x, token in enumerate(tokens):
        case.k[int(case.table[0, token // 16]), token % 16, 0, 0] = -100.0         # a score of -200, or what the cap leaves of it
        _plant(case, token, 5 + x, -math.inf if x == 2 else math.inf)
    print(f"[{dtype}, {n} rows of {L}, cap {cap}]", flush=True)
    o, lse = st.st_attn_cache(q, rows_of([n]).cuda(), case.cache(), True, 0.125, softcap=cap)
    assert torch.isfinite(lse).all()
    for x in range(4):
        assert (o[0, :, :, 5 + x] == (-math.inf if x == 2 else math.inf)).all(), x
    keep = torch.ones(D, dtype=torch.bool, device="cuda")
    keep[5:9] = False
    assert torch.isfinite(o[..., keep]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,n", WALKS)
def test_values_beyond_fp32_reach_those_who_see_them(dtype, L, n):
    """e4m3 values times a scale so high that fp32 does not hold the product, which is an infinity then: of a token that the last rows see, and
    of one that all see."""
    D = 64
    case = Case(23, "e4m3", [L], 16, 1, D)
    q = torch.randn((1, n, 4, D), generator=case.g).to(TYPES[dtype]).cuda()
    edge = L - (n + 1) // 2
    late = (torch.arange(n, device="cuda") >= edge - (L - n))[:, None].expand(n, 4)
    run = lambda: st.st_attn_cache(q, rows_of([n]).cuda(), case.cache(), True, 0.125)
    for byte, code in ((247, 256.0), (250, 32.0), (250, 448.0), (254, 2.0)):
        print(f"[{dtype}, {n} rows of {L}, {code} times 2^{byte - 127}]", flush=True)
        for page in {int(case.table[0, edge // 16]), int(case.table[0, 2])}:
            case.v[page] = 0
            case.scales[1][page] = byte
        _plant(case, edge, 12, code)
        _plant(case, 40, 3, -code)
        _plant(case, 41, 4, 2.0 ** -9)
        o, lse = run()
        assert torch.isfinite(lse).all()
        assert (o[0, :, :, 3] == -math.inf).all() and torch.isfinite(o[0, :, :, 4]).all()
        assert (o[0, :, :, 12][late] == math.inf).all() and torch.isfinite(o[0, :, :, 12][~late]).all()
        k, v = st.st_cache_read(case.cache(), None, L)
        assert v[0, 40, 0, 3] == -math.inf and v[0, edge, 0, 12] == math.inf and torch.isfinite(v[0, 41]).all()


# ---- appending

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("byte", [254, 253, 200, 1])
def test_appending_to_a_page_of_any_scale(dtype, byte):
    """A program's own page, begun with a scale at the ends of what there are: new rows are stored in it."""
    case = Case(24, "e4m3", [3], 16, 1, 64)
    for i, pages in enumerate((case.k, case.v)):
        case.scales[i].fill_(byte)
        case.oracle[i].e.fill_(byte - 127)
    k, v = (torch.randn((1, 5, 1, 64), generator=case.g).to(TYPES[dtype]).cuda() for _ in range(2))
    k[0, 0], v[0, 2], k[0, 1, 0, :9], v[0, 4, 0, 5:20] = 1e38, -3e37, 2e36, 1.5e38
    starts, lens = rows_of([5]), [8]
    st.st_cache_append(None, k, v, starts.cuda(), case.cache(lens), torch.zeros(0, dtype=torch.float64).cuda(), norm=False)
    for i, x in enumerate((k, v)):
        case.oracle[i].append(case.table, lens, starts, x[0].double().cpu())
        page = int(case.table[0, 0])
        assert int(case.scales[i][page, 0]) - 127 == int(case.oracle[i].e[page, 0])
        got = (case.k, case.v)[i][page, :8].double().cpu()
        assert torch.equal(got, case.oracle[i].x[page, :8])
        assert (got[3:] != 0).any()


def test_keys_beside_a_tie():
    """Rotated keys that are 2^-43 of themselves above or below the middle of two e4m3 values, at every place of a page and for every 64th
    of a turn: angles, sines and cosines made in 64 bits decide them rightly, those that are 2^-41 off do not."""
    n, rng = 256, np.random.default_rng(1)
    freq = 1.0
    a = np.zeros((n, 2)), np.zeros((n, 2))
    for place in range(n):
        sn, cs = math.sin(place * freq), math.cos(place * freq)
        if abs(sn) < 0.3:                                                        # (little to choose b by)
            continue
        x = rng.uniform(0.3, 0.9, 1 << 18).astype(np.float32).astype(np.float64)
        tie = 1.0625
        b = ((x * cs - tie) / sn).astype(np.float32).astype(np.float64)
        off = ((x.astype(np.longdouble) * np.longdouble(cs) - b.astype(np.longdouble) * np.longdouble(sn)) - np.longdouble(tie)).astype(np.float64)
        for side in range(2):
            good = np.where(off > 0, off, np.inf) if side == 0 else np.where(off < 0, -off, np.inf)
            good = np.where(good < 2.0 ** -43, np.inf, good)
            i = int(good.argmin())
            assert good[i] < 2.0 ** -38
            a[0][place, side], a[1][place, side] = x[i], b[i]
    k = torch.zeros((1, n, 2, 32))
    k[0, :, :, 0], k[0, :, :, 1] = torch.tensor(a[0]), torch.tensor(a[1])
    k[0, :, :, 2] = 448.0                                                        # (the scale is 1)
    k = k.cuda()
    case = Case(25, "e4m3", [0], 256, 2, 32, more=1)
    st.st_cache_append(None, k, k, rows_of([n]).cuda(), case.cache([n]), torch.tensor([freq], dtype=torch.float64).cuda(), norm=False, pairs="neighbours")
    page = int(case.table[0, 0])
    assert (case.scales[0][page] == 127).all()
    got = case.k[page, :, :, 0].float().cpu()
    for place in range(n):
        if a[0][place, 0]:
            assert got[place].tolist() == [1.125, 1.0], place


# ---- scores near the ends of fp32

@pytest.mark.parametrize("dtype,kind", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32"), ("f32", "e4m3")])
@pytest.mark.parametrize("L,n", WALKS + [(1, 1), (33, 2)])
def test_scores_near_the_ends_of_fp32(dtype, kind, L, n):
    """A row whose scores are all far below zero still has a softmax: of all tokens alike, the mean of the values."""
    D, Hq = 64, 4
    case = Case(26, kind, [L], 16, 1, D)
    q = torch.zeros((1, n, Hq, D))
    q[..., 0] = torch.tensor([1.0, -1.0, 2.0 ** 10, 0.0])[None, None]
    q = q.mul(2.0 ** 60).to(TYPES[dtype]).cuda()
    case.k[..., 0] = torch.tensor(-256.0, device="cuda").to(case.k.dtype)
    if kind == "e4m3":
        case.scales[0].fill_(127 + 40)
    else:
        case.k[..., 0] = torch.tensor(-2.0 ** 48, device="cuda").to(case.k.dtype)
    o, lse = st.st_attn_cache(q, rows_of([n]).cuda(), case.cache(), True, 1.0)
    s = torch.tensor([-1.0, 1.0, -2.0 ** 10, 0.0]).double() * 2.0 ** 108
    _, v, _ = case.held(0)
    v = v[:, 0]
    for i in range(n):
        seen = v[:L - n + i + 1]
        mean, mass = seen.mean(0), seen.abs().mean(0)
        bound = mass * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) + 1e-30
        for h in range(Hq):
            assert ((o[0, i, h].double().cpu() - mean).abs() <= bound).all(), (i, h)
            assert abs(float(lse[0, h, i]) - float(s[h] + math.log(len(seen)))) <= 2.0 ** -20 * abs(float(s[h])) + 1e-5


# ---- the precision of the probabilities

def _two_parts(dtype, kind, lens, counts, held, Hq=4, Hkv=1, D=64, T=None, max_rows=None, seed=31):
    """Sequences `held` to the bound of probabilities in two parts, fp32 O."""
    case = Case(seed, kind, lens, 16, Hkv, D)
    T = sum(counts) if T is None else T
    q = torch.randn((1, T, Hq, D), generator=case.g).to(TYPES[dtype]).cuda()
    starts = rows_of(counts)
    print(f"[{dtype} from {kind}, {lens} by {counts}, {Hq}/{Hkv} D{D}, T {T}, max_rows {max_rows}]", flush=True)
    o, lse = st.st_attn_cache(q, starts.cuda(), case.cache(), True, 1 / math.sqrt(D), max_rows=max_rows)
    check_attention(case, q, starts, o, lse, True, 1 / math.sqrt(D), max_rows=max_rows, two_parts=held)


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("counts,Hq,Hkv", [([1, 1], 8, 2), ([1], 4, 4), ([5, 3], 4, 1), ([20, 7], 4, 1), ([32, 16], 4, 1), ([64, 3], 4, 1)])
def test_probabilities_in_two_parts(kind, D, counts, Hq, Hkv):
    for lens in ([90] * len(counts), [1700, 64][:len(counts)]):
        _two_parts("bf16", kind, lens, counts, range(len(counts)), Hq, Hkv, D, max_rows=max(counts))


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("counts,Hq,Hkv,held", [([5, 200, 20, 1], 4, 1, [0, 2, 3]), ([32, 33, 70], 4, 1, [0]), ([1] * 9, 32, 1, range(9)),
                                                ([8, 100, 1], 16, 1, [0, 2]), ([128, 129], 1, 1, [0]), ([60, 128, 300], 2, 2, [0]),
                                                ([20], 4, 1, [0]), ([1], 32, 1, [0])])
def test_precision_does_not_depend_on_the_batch(kind, D, counts, Hq, Hkv, held):
    """Up to 128 rows of a group: two parts, beside prompts, and with max_rows left at what the call could have."""
    for more in (0, 400):
        _two_parts("bf16", kind, [c + 150 for c in counts], counts, held, Hq, Hkv, D, T=sum(counts) + more)
