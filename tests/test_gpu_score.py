"""Attention with modified scores (st_attn_score_fwd / _bwd) and row spans (st_mask_spans) against the 64-bit oracle.

Tolerances.  fp32: sums of up to some hundred products and terms, each step rounded by 2^-24 relative, 1e-5 in the norm as for the
other fp32 kernels.  bf16: the products are exact and everything up to P is fp32; P and dU are rounded once, by 2^-8 relative at most
(half a step), and so are the results in bf16; Delta comes from an O with the rounding of P in it.  That is at most one rounding for
O in fp32, two for O and dV in bf16, three for dQ and dK: of each element's terms, and of the norm of a tensor whose terms do not
cancel on the whole."""
import math

import pytest
import torch

import paper_2407_00611_amd as st
from oracle import score as so

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -8


def _near(x, ref, bound, what, size=None):
    """2-norm of the difference within bound of the reference's, and each element within bound of the sizes of its terms (None: of
    the element itself, or eight times the root mean square of all); -inf alike."""
    x, ref = x.double(), ref.double()
    assert x.shape == ref.shape, what
    assert torch.equal(x == -math.inf, ref == -math.inf), f"{what}: -inf elsewhere"
    fine = ref != -math.inf
    size = size[fine] if size is not None else None
    x, ref = x[fine], ref[fine]
    assert torch.isfinite(x).all(), f"{what}: not finite"
    if not ref.numel():
        return
    rms = float(ref.square().mean().sqrt())
    off = float((x - ref).square().mean().sqrt())
    assert off <= bound * rms + 1e-7, f"{what}: {off / max(rms, 1e-30):.3e} off, {bound:.1e} allowed"
    size = size + ref.abs() if size is not None else ref.abs().clamp(min=8 * rms)
    worst = float(((x - ref).abs() / (size * bound + 1e-6)).max())
    assert worst <= 1, f"{what}: an element {worst:.3e} times what is allowed off"


def _positions(where, n):
    i = torch.arange(n)
    if isinstance(where, tuple):
        return torch.where(i < where[1], where[0] + i, where[2] + i - where[1]).cuda()
    return (where + i).cuda()


def _random(g, dtype, layout, B, S, H, D):
    if layout == "heads_first":
        return torch.randn((B, H, S, D), generator=g).to(dtype).cuda().transpose(1, 2)
    if layout == "wide":                             # a slice of a buffer with other tensors before and behind
        return torch.randn((B, S, H + 3, D + 16), generator=g).to(dtype).cuda()[:, :, 1:H + 1, 8:D + 8]
    return torch.randn((B, S, H, D), generator=g).to(dtype).cuda()


def _spans(kind, g, pos, Sk, k0, B):
    n = len(pos)
    if kind is None:
        return None
    if kind == "random":                             # any intervals: empty, reversed, beyond the chunk, a single key
        a = torch.randint(k0 - 5, k0 + Sk + 5, (B, n, 2), generator=g)
        a[:, ::7, 1] = a[:, ::7, 0] + 1
        a[:, 3::11] = torch.tensor([-(1 << 62), 1 << 62])
        return a.cuda()
    if kind == "window":
        p = pos.cpu()
        return torch.stack([p - 9, p + 3], -1).expand(B, -1, -1).contiguous().cuda()
    if kind == "none":
        return torch.zeros((B, n, 2), dtype=torch.int64).cuda()
    raise AssertionError(kind)


def _run(dtype, B, Hq, Hkv, D, Sq, Sk, where=0, k0=0, causal=False, cap=0.0, alibi=False, spans=None, layout="dense", scale=None, backward=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v, d_o = (_random(g, t, layout, B, S, H, D) for S, H in ((Sq, Hq), (Sk, Hkv), (Sk, Hkv), (Sq, Hq)))
    pos, kpos = _positions(where, Sq), _positions(k0, Sk)
    span = _spans(spans, g, pos, Sk, k0, B)
    slopes = (2.0 ** (-8.0 * (torch.arange(Hq) + 1) / Hq)).cuda() if alibi else None
    scale = scale or 1 / math.sqrt(D)
    print(f"[{dtype} B{B} {Hq}/{Hkv} D{D} {Sq}x{Sk} at {where} on {k0} causal {causal} cap {cap} alibi {alibi} spans {spans} {layout}]", flush=True)
    mods = dict(softcap=cap, slopes=slopes, spans=span)
    olow = torch.empty((B, Sq, Hq, D), dtype=t, device="cuda")
    o, lse = st.st_attn_score_fwd(q, k, v, where, k0, causal, scale, o_part=torch.empty((B, Sq, Hq, D), device="cuda"), o_lowp=olow, **mods)
    ref = dict(cap=cap, slopes=slopes, span=span)
    o_ref, lse_ref = so.forward(q, k, v, pos, kpos, causal, scale, **ref)
    one = 1e-5 if dtype == "f32" else STEP
    size = so.magnitudes(q, k, v, d_o, lse_ref, pos, kpos, causal, scale, **ref)
    _near(o, o_ref, one, "o", size[0])
    _near(olow, o_ref, one if dtype == "f32" else 2 * STEP, "o in the storage type", size[0])
    _near(lse, lse_ref, 1e-5, "lse")
    if not backward:
        return
    delta = st.st_attn_delta(d_o, o)
    dq, dk, dv = st.st_attn_score_bwd(q, k, v, d_o, lse, delta, where, k0, causal, scale, **mods)
    want = so.backward(q, k, v, d_o, lse_ref, so.delta(d_o, o_ref), pos, kpos, causal, scale, **ref)
    bounds = (4e-5, 4e-5, 1e-5) if dtype == "f32" else (3 * STEP, 3 * STEP, 2 * STEP)
    # P of the backward is exp(s - lse), and lse a value of fp32: half a step of it, 2^-24 |lse|, is an error of the exponent.  It
    # shows where a bias puts the only keys of a row a million units away.
    far = 2.0 ** -24 * float(lse_ref[lse_ref != -math.inf].abs().max()) if bool((lse_ref != -math.inf).any()) else 0.0
    bounds = tuple(x + far for x in bounds)
    for x, y, s, bound, name in zip((dq, dk, dv), want, size[1:], bounds, ("dq", "dk", "dv")):
        assert x.dtype == t
        # what cancels: dP - Delta of rows that see one key or two is rounding of terms of this size
        floor = bound * float(want[2].abs().mean()) * 0.05 if Sk else 0.0
        _near(x, y, bound, name, s) if float(y.abs().max() if y.numel() else 0) > floor else None
    # added to what is there, twice, bit for bit the same
    acc = [torch.full(s, 3.0, device="cuda") for s in (q.shape, k.shape, v.shape)]
    again = [x.clone() for x in acc]
    for a in (acc, again):
        st.st_attn_score_bwd(q, k, v, d_o, lse, delta, where, k0, causal, scale, dq_acc=a[0], dk_acc=a[1], dv_acc=a[2], **mods)
    for x, y, z, s, bound, name in zip(acc, again, want, size[1:], bounds, ("dq", "dk", "dv")):
        assert torch.equal(x, y), name
        _near(x, z + 3.0, bound, name + " added", s + 3.0)


CASES = [
    # one token, one key, nothing at all
    dict(B=1, Hq=1, Hkv=1, Sq=1, Sk=1),
    dict(B=2, Hq=4, Hkv=2, Sq=1, Sk=70, where=69, causal=True, alibi=True, cap=3.0),
    dict(B=1, Hq=2, Hkv=1, Sq=5, Sk=0),
    dict(B=1, Hq=2, Hkv=1, Sq=33, Sk=64, spans="none"),
    # a chunk behind the rows, before them, far before them
    dict(B=1, Hq=2, Hkv=2, Sq=40, Sk=50, where=0, k0=100, causal=True),
    dict(B=1, Hq=2, Hkv=2, Sq=40, Sk=50, where=45, k0=10, causal=True, alibi=True),
    dict(B=1, Hq=8, Hkv=2, Sq=70, Sk=65, where=1000000, k0=100, causal=True, alibi=True),
    dict(B=1, Hq=8, Hkv=2, Sq=70, Sk=65, where=5 << 32, k0=(5 << 32) - 17, causal=True, cap=4.0),
    # keys on both sides of the row
    dict(B=2, Hq=3, Hkv=3, Sq=100, Sk=130, where=20, alibi=True),
    dict(B=1, Hq=3, Hkv=1, Sq=129, Sk=257, where=100, causal=True, cap=2.0),
    # two runs of rows
    dict(B=1, Hq=6, Hkv=2, Sq=77, Sk=90, where=(10, 30, 300), k0=5, causal=True, alibi=True, cap=10.0),
    dict(B=1, Hq=2, Hkv=2, Sq=200, Sk=300, where=(10, 130, 200), causal=True),
    # spans of any kind, alone and with the causal order
    dict(B=2, Hq=4, Hkv=2, Sq=150, Sk=200, spans="random", alibi=True),
    dict(B=2, Hq=4, Hkv=1, Sq=150, Sk=333, where=150, spans="random", causal=True, cap=5.0),
    dict(B=1, Hq=5, Hkv=1, Sq=300, Sk=300, spans="window", k0=0),
    dict(B=1, Hq=40, Hkv=1, Sq=19, Sk=131, where=112, causal=True, alibi=True, cap=20.0),
    # memory layouts, several tiles
    dict(B=2, Hq=4, Hkv=2, Sq=257, Sk=129, layout="heads_first", cap=3.0),
    dict(B=2, Hq=4, Hkv=2, Sq=130, Sk=190, where=60, causal=True, layout="wide", alibi=True),
    # scores far from unit scale, with and without a cap
    dict(B=1, Hq=2, Hkv=2, Sq=96, Sk=160, scale=0.3),
    dict(B=1, Hq=2, Hkv=2, Sq=96, Sk=160, scale=40.0, cap=30.0),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 40)])
def test_against_the_definition(dtype, D, case):
    _run(dtype, D=D, seed=len(str(case)), **case)


@pytest.mark.parametrize("D", [8, 32, 96, 128, 192, 256])
def test_head_sizes_of_fp32(D):
    _run("f32", B=1, Hq=4, Hkv=2, D=D, Sq=75, Sk=101, where=26, causal=True, cap=6.0, alibi=True)
    _run("f32", B=2, Hq=2, Hkv=1, D=D, Sq=40, Sk=70, spans="random")


@pytest.mark.parametrize("dtype,D,Sq,Sk,Hq,Hkv", [("bf16", 128, 1, 5000, 8, 1), ("bf16", 64, 3, 20000, 16, 2), ("bf16", 128, 700, 900, 4, 1),
                                                  ("f32", 64, 2, 3001, 4, 2), ("bf16", 128, 40, 4097, 2, 2)])
def test_split_launches(dtype, D, Sq, Sk, Hq, Hkv):
    """Few rows or few keys: shares of a tile's walk, joined afterwards."""
    _run(dtype, 1, Hq, Hkv, D, Sq, Sk, where=Sk - Sq, causal=True, alibi=True, cap=8.0)
    _run(dtype, 1, Hq, Hkv, D, Sq, Sk, spans="random")


def test_more_row_blocks_than_a_list_holds():
    """Key tiles walk their rows through a list of 1024 blocks at a time; 257 key tiles, so that no launch is split."""
    _run("bf16", 1, 16, 1, 64, 2100, 32800, where=0, spans="window", alibi=True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("with_prefix", [False, True])
def test_mask_spans(causal, with_prefix):
    g = torch.Generator().manual_seed(5)
    for B, n_docs, Sq, where in [(1, 0, 4, 0), (3, 1, 20, 3), (2, 7, 300, 0), (2, 40, 77, (5, 30, 200)), (1, 1, 1, 1 << 40)]:
        ends = torch.sort(torch.randint(0, 280, (B, n_docs + 1), generator=g), dim=1).values       # equal ones: empty documents
        if Sq == 1:
            ends = torch.tensor([[(1 << 40) - 5, (1 << 40) + 7]])
        pre = torch.randint(-2, 60, (B, n_docs), generator=g) if with_prefix else None
        got = st.st_mask_spans(ends.cuda(), Sq, where, causal, prefix=pre.cuda() if with_prefix else None)
        lists = [[max(x, 0) for x in row] for row in pre.tolist()] if with_prefix else None
        assert got.tolist() == [[list(s) for s in rows] for rows in so.spans(ends.tolist(), _positions(where, Sq).tolist(), causal, lists)]


def _packed(seed, dtype, B=2, Hq=6, Hkv=2, D=64, S=390):
    g = torch.Generator().manual_seed(seed)
    q, k, v, d_o = (torch.randn((B, S, h, D), generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv, Hq))
    bounds = torch.tensor([[0, 100, 101, 260, 370], [30, 95, 200, 200, 390]]).cuda()
    return q, k, v, d_o, bounds


def _all(q, k, v, d_o, where, k0, scale, mods, causal=False):
    o, lse = st.st_attn_score_fwd(q, k, v, where, k0, causal, scale, **mods)
    return (o, lse) + st.st_attn_score_bwd(q, k, v, d_o, lse, st.st_attn_delta(d_o, o), where, k0, causal, scale, **mods)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_nobody_sees_may_hold_anything(dtype):
    """Infinities and NaN in the padding, and of one document: the others' results stay as they are, bit for bit."""
    q, k, v, d_o, bounds = _packed(1, dtype)
    spans = st.st_mask_spans(bounds, q.shape[1], 0, True)
    mods = dict(softcap=7.0, slopes=torch.full((6,), 0.01).cuda(), spans=spans)
    # what lies in no document is rewritten, then a document too
    clean = _all(q, k, v, d_o, 0, 0, 0.2, mods)
    i = torch.arange(q.shape[1], device="cuda")
    outside = (i < bounds[:, :1]) | (i >= bounds[:, -1:])
    one = (i >= bounds[:, 2:3]) & (i < bounds[:, 3:4])
    one[1] = False
    for bad, what in ((outside, "padding"), (outside | one, "a document")):
        for value in (math.nan, math.inf, -math.inf):
            x = [t.clone() for t in (q, k, v, d_o)]
            for t in x:
                t[bad] = value
            got = _all(*x, 0, 0, 0.2, mods)
            for a, b, name in zip(clean, got, ("o", "lse", "dq", "dk", "dv")):
                rows = (~bad)[:, None].expand(-1, 6, -1) if name == "lse" else ~bad
                assert torch.equal(a[rows], b[rows]), f"{what}, {value}: {name}"
                if name != "lse":
                    assert not torch.isnan(b[outside]).any(), f"{what}, {value}: {name} of the padding"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_is_seen_reaches_who_sees_it(dtype):
    q, k, v, d_o, bounds = _packed(2, dtype)
    spans = st.st_mask_spans(bounds, q.shape[1], 0, True)
    clean, lse = st.st_attn_score_fwd(q, k, v, 0, 0, False, 0.125, spans=spans)
    for key in (100, 130, 255):                      # in entry 0: a document of one token, and inside one
        x = v.clone()
        x[0, key, 1, 5] = math.inf
        o, _ = st.st_attn_score_fwd(q, k, x, 0, 0, False, 0.125, spans=spans)
        sees = (spans[0, :, 0] <= key) & (key < spans[0, :, 1])
        assert (o[0, sees][:, 3:, 5] == math.inf).all(), key
        o[0, sees] = 0
        same = clean.clone()
        same[0, sees] = 0
        assert torch.equal(o, same), key


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_chunks_of_a_ring_fold_to_the_whole(dtype):
    """A step as a training program makes it: spans, every delivered chunk, merge, Delta, gradients chunk by chunk, two runs of rows."""
    B, Hq, Hkv, D, Sk, n = 2, 4, 2, 64, 96, 4
    g = torch.Generator().manual_seed(9)
    where, Sq = (48, 70, 250), 140
    q, d_o = (torch.randn((B, Sq, Hq, D), generator=g).to(dtype).cuda() for _ in range(2))
    ks, vs = ([torch.randn((B, Sk, Hkv, D), generator=g).to(dtype).cuda() for _ in range(n)] for _ in range(2))
    bounds = torch.tensor([[0, 60, 300, 384], [20, 110, 111, 350]]).cuda()
    prefix = torch.tensor([[10, 200, 0], [0, 1, 80]]).cuda()
    spans = st.st_mask_spans(bounds, Sq, where, True, prefix=prefix)
    mods = dict(softcap=9.0, slopes=torch.tensor([0.5, 0.1, 0.02, 0.004]).cuda(), spans=spans)
    o = torch.zeros((B, Sq, Hq, D), device="cuda")
    lse = torch.full((B, Hq, Sq), -math.inf, device="cuda")
    low = torch.empty_like(q)
    for j in (2, 0, 3, 1):
        part = st.st_attn_score_fwd(q, ks[j], vs[j], where, j * Sk, False, 0.2, **mods)
        st.st_attn_merge(o, lse, *part, out_dtype=st.ST_BF16 if dtype == torch.bfloat16 else st.ST_F32, o_out_lowp=low)
    pos, kpos = _positions(where, Sq), _positions(0, n * Sk)
    ref = dict(cap=9.0, slopes=mods["slopes"], span=spans)
    k, v = torch.cat(ks, 1), torch.cat(vs, 1)
    o_ref, lse_ref = so.forward(q, k, v, pos, kpos, False, 0.2, **ref)
    one = STEP if dtype == torch.bfloat16 else 1e-5
    _near(o, o_ref, one, "o")
    _near(lse, lse_ref, 1e-5, "lse")
    delta = st.st_attn_delta(d_o, o)
    dq = torch.zeros((B, Sq, Hq, D), device="cuda")
    dk, dv = torch.empty(k.shape, device="cuda"), torch.empty(k.shape, device="cuda")
    for j in (2, 0, 3, 1):
        a, b = torch.zeros(ks[j].shape, device="cuda"), torch.zeros(ks[j].shape, device="cuda")
        st.st_attn_score_bwd(q, ks[j], vs[j], d_o, lse, delta, where, j * Sk, False, 0.2, dq_acc=dq, dk_acc=a, dv_acc=b, **mods)
        dk[:, j * Sk:(j + 1) * Sk], dv[:, j * Sk:(j + 1) * Sk] = a, b
    want = so.backward(q, k, v, d_o, lse_ref, so.delta(d_o, o_ref), pos, kpos, False, 0.2, **ref)
    for x, y, name in zip((dq, dk, dv), want, ("dq", "dk", "dv")):
        _near(x, y, 3 * one, name)


def test_captured_on_a_stream_and_replayed():
    """Two captured graphs with workspaces of their own, replayed between eager work; an eager call on another stream agrees."""
    q, k, v, d_o, bounds = _packed(4, torch.bfloat16, D=128)
    slopes = torch.full((6,), 0.05).cuda()
    what = []
    for cap in (0.0, 5.0):
        spans = torch.empty((2, q.shape[1], 2), dtype=torch.int64, device="cuda")
        out = dict(o_part=torch.empty(q.shape, device="cuda"), lse_part=torch.empty((2, 6, q.shape[1]), device="cuda"))
        acc = [torch.empty(t.shape, device="cuda") for t in (q, k, v)]
        delta = torch.empty_like(out["lse_part"])
        mods = dict(softcap=cap, slopes=slopes, spans=spans)
        sizes = [st.st_attn_score_workspace_bytes(q, k, v, 0, 0, False, 0.1, backward=b, **mods) for b in (False, True)]
        ws = [torch.empty(n + 256, dtype=torch.uint8, device="cuda") for n in sizes]

        def step(spans=spans, out=out, acc=acc, delta=delta, mods=mods, ws=ws):
            st.st_mask_spans(bounds, q.shape[1], 0, True, spans=spans)
            st.st_attn_score_fwd(q, k, v, 0, 0, False, 0.1, workspace=ws[0], **out, **mods)
            st.st_attn_delta(d_o, out["o_part"], delta)
            st.st_attn_score_bwd(q, k, v, d_o, out["lse_part"], delta, 0, 0, False, 0.1, dq_acc=acc[0], dk_acc=acc[1], dv_acc=acc[2], assign=True,
                                 workspace=ws[1], **mods)
        step()
        torch.cuda.synchronize()
        eager = [t.clone() for t in list(out.values()) + acc]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        what.append((graph, list(out.values()) + acc, eager, step))          # (step holds the buffers that the graph works on)
    other = torch.cuda.Stream()
    for _ in range(3):
        for graph, tensors, eager, _ in what:
            for t in tensors:
                t.fill_(-1.0)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(tensors, eager):
                assert torch.equal(a, b)
        for cap, (_, _, eager, _) in zip((0.0, 5.0), what):
            spans = st.st_mask_spans(bounds, q.shape[1], 0, True)
            other.wait_stream(torch.cuda.current_stream())
            o, lse = st.st_attn_score_fwd(q, k, v, 0, 0, False, 0.1, softcap=cap, slopes=slopes, spans=spans, stream=other)
            other.synchronize()
            assert torch.equal(o, eager[0]) and torch.equal(lse, eager[1])


def test_plain_scores_agree_with_the_block_kernels():
    g = torch.Generator().manual_seed(11)
    q, k, v = (torch.randn((1, 300, 4, 128), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    o, lse = st.st_attn_score_fwd(q, k, v, 0, 0, True, 0.1)
    o2, lse2 = st.st_attn_block_fwd(q, k, v, 0, 0, True, 0.1)
    # the block kernel rounds Q scale log2 e to bf16: 2^-8 of the scores, which are about 1.1 wide
    assert float((lse - lse2).abs().max()) < 2e-2 and float((o - o2).norm() / o.norm()) < 2 * STEP
