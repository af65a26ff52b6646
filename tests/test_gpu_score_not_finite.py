"""Rows whose scores are NaN: they stay NaN where their walk is split or their states are folded, and nobody else changes.  Rows are
compared bit for bit, so there is no tolerance."""
import math

import pytest
import torch

import paper_2407_00611_amd as st
from test_gpu_score import _all, _packed

pytestmark = pytest.mark.gpu


def _forward_shares(q, k, v, where, causal, **mods):
    """Shares of the keys of every row tile, from the workspace: as many fp32 O and lse, each rounded up to 256 bytes."""
    need = st.st_attn_score_workspace_bytes(q, k, v, where, 0, causal, 0.1, **mods)
    up = lambda n: (n + 255) // 256 * 256
    rows = q.shape[0] * q.shape[1] * q.shape[2]
    fits = [n for n in range(2, 65) if up(n * rows * q.shape[3] * 4) + up(n * rows * 4) == need]
    assert need == 0 or len(fits) == 1
    return fits[0] if need else 1


# one to 64 shares of one token's keys, three of some rows'
SPLITS = [("bf16", 128, 1, 512, 2), ("bf16", 64, 1, 1024, 4), ("bf16", 128, 1, 4096, 16), ("bf16", 64, 1, 10000, 39), ("bf16", 128, 1, 16384, 64),
          ("bf16", 128, 90, 900, 3), ("bf16", 128, 1, 255, 1),
          ("f32", 64, 1, 512, 2), ("f32", 80, 1, 1000, 4), ("f32", 128, 1, 4096, 16), ("f32", 64, 1, 16384, 32), ("f32", 64, 90, 900, 3),
          ("f32", 64, 1, 200, 1)]


@pytest.mark.parametrize("dtype,D,Sq,Sk,shares", SPLITS)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_rows_whose_scores_are_nan(dtype, D, Sq, Sk, shares, value):
    """Q of one head, and K of one key that one entry sees in a span inside a single share.  One entry of two stays clean."""
    Hq, Hkv = (8, 1) if Sq == 1 else (16, 2) if dtype == "bf16" else (12, 2)
    g = torch.Generator().manual_seed(Sk)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v, d_o = (torch.randn((2, S, h, D), generator=g).to(t).cuda() for S, h in ((Sq, Hq), (Sk, Hkv), (Sk, Hkv), (Sq, Hq)))
    where = Sk - Sq
    one = torch.tensor([Sk // 3, Sk // 3 + 5]).expand(2, Sq, 2).contiguous().cuda()
    for spans, causal in ((None, True), (one, False)):
        mods = dict(spans=spans, softcap=0.0)
        assert _forward_shares(q, k, v, where, causal, **mods) == shares
        clean = st.st_attn_score_fwd(q, k, v, where, 0, causal, 0.1, **mods)
        for what in ("q", "k"):
            x = {"q": q.clone(), "k": k.clone()}
            at = Sk // 3 + 2
            if what == "q":
                x["q"][1, Sq // 2, 3] = value
                bad = torch.zeros((2, Sq, Hq), dtype=torch.bool, device="cuda")
                bad[1, Sq // 2, 3] = True
            else:
                x["k"][1, at, 0] = math.nan          # (an infinite key's scores may all be -inf)
                bad = torch.zeros((2, Sq, Hq), dtype=torch.bool, device="cuda")
                bad[1, :, :Hq // Hkv] = True
            for low in (False, True):
                o, lse = st.st_attn_score_fwd(x["q"], x["k"], v, where, 0, causal, 0.1, lowp=low, **mods)
                assert o[bad].isnan().all(), f"{what}, {shares} shares: O of the rows that see it"
                assert lse.transpose(1, 2)[bad].isnan().all(), f"{what}, {shares} shares: lse"
                same = clean[0] if not low else clean[0].to(t)
                assert torch.equal(o[~bad], same[~bad]) and torch.equal(lse.transpose(1, 2)[~bad], clean[1].transpose(1, 2)[~bad])
            if what == "k" and causal:
                continue
            # the row has gradients, all of them NaN, and gives its keys such ones
            dq, dk, dv = st.st_attn_score_bwd(x["q"], x["k"], v, d_o, lse, st.st_attn_delta(d_o, o), where, 0, causal, 0.1, **mods)
            assert dq[bad].isnan().all() and not dq[~bad].isnan().any()
            seen = torch.zeros((2, Sk, Hkv), dtype=torch.bool, device="cuda")
            seen[1, :where + Sq // 2 + 1 if causal else None, int(bad[1, Sq // 2].nonzero()[0]) // (Hq // Hkv)] = True
            if spans is not None:
                seen[:, :Sk // 3] = seen[:, Sk // 3 + 5:] = False
            assert dk[seen].isnan().all() and dv[seen].isnan().all() and not dk[~seen].isnan().any() and not dv[~seen].isnan().any()


@pytest.mark.parametrize("n", [2, 4, 5, 8, 9, 16, 17, 40])
def test_combining_a_state_of_nan(n):
    """Every way of the combine: states of rows that are NaN in one of them and empty in all others, NaN in all, empty in all."""
    g = torch.Generator().manual_seed(n)
    o = [torch.randn((1, 12, 2, 40), generator=g).cuda() for _ in range(n)]
    lse = [torch.randn((1, 2, 12), generator=g).cuda() for _ in range(n)]
    for x in range(n):
        lse[x][0, 0, 3] = math.nan if x == n - 1 else -math.inf
        lse[x][0, 1, 4] = math.nan if x == 0 else -math.inf
        lse[x][0, 1, 5] = math.nan
        lse[x][0, 0, 6] = -math.inf
        o[x][0, 6, 0] = math.nan                     # (an empty state's O may hold anything)
    low = torch.empty((1, 12, 2, 40), dtype=torch.bfloat16, device="cuda")
    got, l = st.st_attn_combine(o, lse, out_dtype=st.ST_BF16, o_out_lowp=low)
    gone = torch.zeros((1, 12, 2), dtype=torch.bool, device="cuda")
    gone[0, 3, 0] = gone[0, 4, 1] = gone[0, 5, 1] = True
    assert got[gone].isnan().all() and low[gone].isnan().all() and l.transpose(1, 2)[gone].isnan().all()
    assert not got[~gone].isnan().any() and not low[~gone].isnan().any() and not l.transpose(1, 2)[~gone].isnan().any()
    assert (got[0, 6, 0] == 0).all() and l[0, 0, 6] == -math.inf


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_chunks_with_nan_fold_to_nan(dtype):
    """A fold starts from the empty state, and some chunks hold nothing for a row: a chunk in which its scores are NaN still shows."""
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((2, 40, h, 64), generator=g).to(dtype).cuda() for h in (4, 2, 2))
    spans = torch.tensor([[50, 60]] * 40).expand(2, 40, 2).contiguous().cuda()          # in the second of three chunks
    bad = q.clone()
    bad[0, 7, 2] = math.nan
    for order in ((0, 1, 2), (1, 0, 2), (2, 0, 1)):
        parts = [[st.st_attn_score_fwd(x, k, v, 0, 40 * j, False, 0.1, spans=spans) for j in order] for x in (q, bad)]
        out = []
        for p in parts:
            o, lse = torch.zeros(q.shape, device="cuda"), torch.full((2, 4, 40), -math.inf, device="cuda")
            for part in p:
                st.st_attn_merge(o, lse, *part)
            out.append((o, lse))
            both = st.st_attn_combine([x[0] for x in p], [x[1] for x in p])
            assert both[0].isnan().equal(o.isnan()) and both[1].isnan().equal(lse.isnan())
        (o, lse), (o2, lse2) = out
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()
        assert o2[0, 7, 2].isnan().all() and lse2[0, 2, 7].isnan()
        o2[0, 7, 2], lse2[0, 2, 7] = o[0, 7, 2], lse[0, 2, 7]
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("D", [64, 80, 96, 192, 200, 256])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_fp32_gradients_of_values_that_are_not_finite(D, value):
    """One value of one key's V or K, one row's dO or Q, in tiles that a document's edge crosses, in either half of the columns: who
    sees it has it, nobody else does."""
    q, k, v, d_o, bounds = _packed(19, torch.float32, D=D)
    spans = st.st_mask_spans(bounds, q.shape[1], 0, False)
    clean = _all(q, k, v, d_o, 0, 0, 0.1, dict(spans=spans))
    at = 120                                         # of entry 0: in the document 101 .. 259
    seen = (spans[0, :, 0] <= at) & (at < spans[0, :, 1])
    for column in (3, D - 2):
        for what in "vkdq":
            x = dict(q=q.clone(), k=k.clone(), v=v.clone(), d=d_o.clone())
            x[what][0, at, 1, column] = value       # (KV head 1: query heads 3, 4, 5; query head 1: KV head 0)
            o, lse, dq, dk, dv = _all(x["q"], x["k"], x["v"], x["d"], 0, 0, 0.1, dict(spans=spans))
            for a, b, name in zip((o, dq, dk, dv), (clean[0],) + clean[2:], ("o", "dq", "dk", "dv")):
                assert torch.equal(a[1], b[1]) and torch.equal(a[0, ~seen], b[0, ~seen]), f"{what}, {column}: {name} of those that see nothing of it"
            fine = torch.isfinite
            rest = torch.arange(D, device="cuda") != column
            if what == "d":                          # P is what it was: dV has the value where its row looks, in its column
                assert not fine(dv[0, seen, 0, column]).any() and torch.equal(dv[0, :, 0, rest], clean[4][0, :, 0, rest])
                assert dv[0, seen, 0, column].isnan().all() if math.isnan(value) else (dv[0, seen, 0, column] == value).all()
                assert not fine(dq[0, at, 1]).any() and not fine(dk[0, seen, 0]).any() and torch.equal(o, clean[0])
                assert torch.equal(dv[0, :, 1], clean[4][0, :, 1]) and torch.equal(dk[0, :, 1], clean[3][0, :, 1])
            elif what == "v":                        # O has it in its column, Delta and the rows' dS everywhere
                assert not fine(o[0, seen][:, 3:, column]).any() and torch.equal(o[0][:, 3:, rest], clean[0][0][:, 3:, rest])
                assert not fine(dq[0, seen][:, 3:]).any() and not fine(dk[0, seen, 1]).any() and torch.equal(dv, clean[4])
                assert torch.equal(dq[0][:, :3], clean[2][0][:, :3])
            elif what == "q":
                assert not fine(dq[0, at, 1]).any() and not fine(dk[0, seen, 0]).any() and torch.equal(dk[0, :, 1], clean[3][0, :, 1])
            elif math.isnan(value):
                assert not fine(o[0, seen][:, 3:]).any() and not fine(dq[0, seen][:, 3:]).any() and not fine(dk[0, seen, 1]).any()
                assert torch.equal(dq[0][:, :3], clean[2][0][:, :3])
