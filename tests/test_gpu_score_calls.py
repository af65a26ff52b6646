"""Calls of the modified scores, norms and rotations as programs make them: through either half of the wrapper, several at once, with
more row tiles than the chip holds, with rows that have no gradient."""
import math

import pytest
import torch

import paper_2407_00611_amd as st
from oracle import score as so
from paper_2407_00611_amd import api
from test_gpu_score import _all, _packed, _positions, _run

pytestmark = pytest.mark.gpu


def _step(q, k, v, d_o, bounds, slopes, freq, weight, acc):
    """One of every entry point; with acc also the forms that add."""
    S, D = q.shape[1], q.shape[3]
    spans = st.st_mask_spans(bounds, S, 0, True)
    rope = dict(freq=freq, q_weight=weight, k_weight=weight)
    rq, rk = st.st_qk_rope_fwd(q, k, **rope)
    mods = dict(softcap=6.0, slopes=slopes, spans=spans)
    o, lse = st.st_attn_score_fwd(rq, rk, v, 0, 0, False, 0.3, lowp=True, **mods)
    delta = st.st_attn_delta(d_o, o)
    grads = st.st_attn_score_bwd(rq, rk, v, d_o, lse, delta, 0, 0, False, 0.3, **mods)
    out = st.st_qk_rope_bwd(q, k, grads[0], grads[1], **rope)
    if acc:
        part, pl = torch.empty(q.shape, device="cuda"), torch.empty_like(lse)
        st.st_attn_score_fwd(rq, rk, v, 0, 0, False, 0.3, o_part=part, lse_part=pl, **mods)
        sums = [torch.ones(t.shape, device="cuda") for t in (q, k, v)]
        st.st_attn_score_bwd(rq, rk, v, d_o, lse, delta, 0, 0, False, 0.3, dq_acc=sums[0], dk_acc=sums[1], dv_acc=sums[2], **mods)
        out = out + (part, pl) + tuple(sums)
    return (spans, rq, rk, o, lse) + grads + out


def _inputs(dtype, seed=21, **kw):
    q, k, v, d_o, bounds = _packed(seed, dtype, **kw)
    D = q.shape[3]
    freq = (10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).cuda()
    return q, k, v, d_o, bounds, torch.full((q.shape[2],), 0.02).cuda(), freq, torch.linspace(0.5, 1.5, D).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_both_halves_make_the_same_calls(dtype, monkeypatch):
    """The native half takes plain tensors and numbers, the ctypes half every other accepted form; their results agree bit for bit."""
    x = _inputs(dtype)
    native, took = api._binding, set()

    class Watched:
        def __getattr__(self, name):
            def call(*args):
                done = getattr(native, name)(*args)
                if done is not None:
                    took.add(name)
                return done
            return call

    class Declines:
        def __getattr__(self, _):
            return lambda *a: None
    monkeypatch.setattr(api, "_binding", Watched())
    short = _step(*x, acc=True)
    assert took >= {"mask_spans", "score_fwd", "score_bwd", "rope_fwd", "rope_bwd", "delta"}
    monkeypatch.setattr(api, "_binding", Declines())
    for a, b in zip(short, _step(*x, acc=True)):
        assert torch.equal(a, b)
    # a stream of one's own, as an object and as its handle
    monkeypatch.setattr(api, "_binding", native)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        spans = st.st_mask_spans(x[4], x[0].shape[1], 0, True, stream=stream)
        rq, rk = st.st_qk_rope_fwd(x[0], x[1], freq=x[6], q_weight=x[7], k_weight=x[7], stream=stream)
        o, lse = st.st_attn_score_fwd(rq, rk, x[2], 0, 0, False, 0.3, softcap=6.0, slopes=x[5], spans=spans, lowp=True, stream=stream)
        side.synchronize()
        for a, b in zip(short, (spans, rq, rk, o, lse)):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls with outputs and workspaces of their own share nothing."""
    jobs = [_inputs(torch.bfloat16, seed, D=128) for seed in (31, 32)]
    alone = [_step(*x, acc=True) for x in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(3):
        for n, (x, s) in enumerate(zip(jobs, streams)):
            with torch.cuda.stream(s):
                got[n].append(_step(*x, acc=True))
    torch.cuda.synchronize()
    for want, runs in zip(alone, got):
        for run in runs:
            for a, b in zip(want, run):
                assert torch.equal(a, b)


@pytest.mark.parametrize("spans", ["random", "window"])
def test_more_row_tiles_than_the_chip_holds(spans):
    """263 row tiles of two KV heads, spans: the workgroups take them in an order of their own, 256 at a time."""
    _run("bf16", 1, 32, 2, 64, 2100, 70, where=0, spans=spans, alibi=spans == "window")


def test_documents_of_unlike_lengths():
    """Row tiles that hold the end of a document and the start of the next; 528 workgroups a head group, and a batch entry of padding."""
    B, Hq, Hkv, D, S = 3, 24, 24, 64, 1000
    g = torch.Generator().manual_seed(3)
    q, k, v, d_o = (torch.randn((B, S, Hq, D), generator=g).to(torch.bfloat16).cuda() for _ in range(4))
    bounds = torch.tensor([[0, 3, 150, 151, 610, 700, 990], [100, 500, 500, 650, 652, 900, 1000], [5, 5, 5, 5, 5, 5, 5]]).cuda()
    spans = st.st_mask_spans(bounds, S, 0, False)
    got = _all(q, k, v, d_o, 0, 0, 0.125, dict(spans=spans))
    pos = _positions(0, S)
    o_ref, lse_ref = so.forward(q, k, v, pos, pos, False, 0.125, span=spans)
    want = (o_ref, lse_ref) + tuple(so.backward(q, k, v, d_o, lse_ref, so.delta(d_o, o_ref), pos, pos, False, 0.125, span=spans))
    outside = spans[..., 1] <= spans[..., 0]
    assert (got[0][outside] == 0).all() and (got[1].transpose(1, 2)[outside] == -math.inf).all() and (got[2][outside] == 0).all()
    # P, dU, O and the results are rounded once each, by 2^-8 at most: one rounding for O (fp32), two for dV, three for dQ and dK
    for x, y, n in zip(got, want, (1, 0, 3, 3, 2)):
        x, y = x.double(), y.double()
        fine = torch.isfinite(y)
        assert torch.equal(torch.isfinite(x), fine)
        assert float((x - y)[fine].norm()) <= (n * 2.0 ** -8 + 1e-5) * float(y[fine].norm())


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 80)])
def test_rows_whose_lse_says_that_they_are_empty(dtype, D):
    """lse = -inf: no gradient, whatever the row's dO and Delta hold, also where its span is not empty."""
    g = torch.Generator().manual_seed(13)
    q, k, v, d_o = (torch.randn((2, S, h, D), generator=g).to(dtype).cuda() for S, h in ((200, 4), (300, 2), (300, 2), (200, 4)))
    o, lse = st.st_attn_score_fwd(q, k, v, 0, 0, False, 0.1)
    delta = st.st_attn_delta(d_o, o)
    gone = torch.zeros((2, 200, 4), dtype=torch.bool, device="cuda")
    gone[0, 40:45, 1], gone[1, 199, 3], gone[1, 0, 2] = True, True, True
    lse[gone.transpose(1, 2)] = -math.inf
    quiet, loud = d_o.clone(), d_o.clone()
    quiet[gone], loud[gone] = 0.0, math.nan
    none, bad = delta.clone(), delta.clone()
    none[gone.transpose(1, 2)], bad[gone.transpose(1, 2)] = 0.0, math.nan
    want = st.st_attn_score_bwd(q, k, v, quiet, lse, none, 0, 0, False, 0.1)
    got = st.st_attn_score_bwd(q, k, v, loud, lse, bad, 0, 0, False, 0.1)
    for a, b, name in zip(want, got, ("dq", "dk", "dv")):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b), name
    assert (got[0][gone] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_in_tiles_with_an_edge(D, value):
    """One key's V, one row's dO, one row's Q: who sees them and who does not, in tiles that a document's edge crosses."""
    q, k, v, d_o, bounds = _packed(17, torch.bfloat16, D=D)
    spans = st.st_mask_spans(bounds, q.shape[1], 0, False)
    clean = _all(q, k, v, d_o, 0, 0, 0.1, dict(spans=spans))
    at = 120                                         # of entry 0: in the document 101 .. 259
    seen = (spans[0, :, 0] <= at) & (at < spans[0, :, 1])
    for what in "vdq":
        x = dict(q=q.clone(), v=v.clone(), d=d_o.clone())
        x[what][0, at, 1] = value
        o, lse, dq, dk, dv = _all(x["q"], k, x["v"], x["d"], 0, 0, 0.1, dict(spans=spans))
        for a, b, name in zip((o, dq, dk, dv), (clean[0],) + clean[2:], ("o", "dq", "dk", "dv")):
            assert torch.equal(a[1], b[1]) and torch.equal(a[0, ~seen], b[0, ~seen]), f"{what}: {name} of those that see nothing of it"
        if what == "v":                              # head 1 of K and V: query heads 3, 4, 5
            assert not torch.isfinite(o[0, seen][:, 3:]).any() and torch.equal(o[0, seen][:, :3], clean[0][0, seen][:, :3])
        elif what == "d":                            # query head 1: KV head 0
            assert not torch.isfinite(dv[0, seen][:, 0]).any() and not torch.isfinite(dq[0, at, 1]).any() and torch.equal(o, clean[0])
        else:
            assert not torch.isfinite(dk[0, seen][:, 0]).any() and not torch.isfinite(dq[0, at, 1]).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_that_pass_32_bits(dtype):
    """Heads of a buffer of more than 2^31 elements: as those of dense copies, bit for bit."""
    S, heads, D, Sq = 70000, 264, 128, 40
    big = torch.empty((1, S, heads, D), dtype=dtype, device="cuda")
    assert big.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(4)
    places = {"q": (0, 2), "k": (10, 11), "v": (262, 263), "d": (260, 262)}
    for a, b in places.values():
        big[:, :, a:b] = torch.randn((1, S, b - a, D), generator=g, device="cuda").to(dtype)
    wide = {n: big[:, :, a:b] for n, (a, b) in places.items()}
    wide["q"], wide["d"] = wide["q"][:, S - Sq:], wide["d"][:, S - Sq:]
    dense = {n: t.contiguous() for n, t in wide.items()}
    freq = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    spans = st.st_mask_spans(torch.tensor([[3, 30000, S - 20, S]]).cuda(), Sq, S - Sq, True)
    runs = []
    for x in (wide, dense):
        lse = st.st_attn_score_fwd(x["q"], x["k"], x["v"], S - Sq, 0, True, 0.1, softcap=9.0)[1]
        o = st.st_attn_score_fwd(x["q"], x["k"], x["v"], S - Sq, 0, False, 0.1, spans=spans, lowp=True)
        delta = st.st_attn_delta(x["d"], o[0])
        runs.append((lse,) + tuple(o) + tuple(st.st_attn_score_bwd(x["q"], x["k"], x["v"], x["d"], o[1], delta, S - Sq, 0, False, 0.1, spans=spans)) +
                    tuple(st.st_qk_rope_fwd(x["q"], x["v"][:, S - Sq:], freq=freq, offset=S - Sq)))
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    dk = runs[0][4]                                  # what the spans leave: the last two documents' keys from row S - 40 on
    assert float(dk[0, 30000:].float().norm()) > 0 and not dk[0, :30000].any()


@pytest.mark.parametrize("dtype,cap", [("bf16", 1024.0), ("f32", 1e6)])
def test_caps_far_above_the_scores(dtype, cap):
    """A cap that hardly bends anything: 1 - 2 / (1 + e^2x) cancels there, in the bf16 kernels 2^-22 cap of a score is lost."""
    g = torch.Generator().manual_seed(29)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v = (torch.randn((1, 200, h, 64), generator=g).to(t).cuda() for h in (4, 2, 2))
    pos = _positions(0, 200)
    o, lse = st.st_attn_score_fwd(q, k, v, 0, 0, True, 0.125, softcap=cap)
    o_ref, lse_ref = so.forward(q, k, v, pos, pos, True, 0.125, cap=cap)
    off = 2.0 ** -22 * cap if dtype == "bf16" else 1e-5
    assert float((lse - lse_ref).abs().max()) <= off + 1e-5
    # the errors of a row's scores change P by as much, beside its rounding by 2^-8 in bf16 and the sums' in fp32
    assert float((o - o_ref).norm()) <= ((2.0 ** -8 if dtype == "bf16" else 1e-5) + 2 * off) * float(o_ref.norm())
