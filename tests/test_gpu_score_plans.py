"""Paths of the backward of modified scores that hang on how a launch is planned, each with the plan it needs asserted from the size
of the workspace, and its results in the storage type where a row sees few keys.  Tolerances: those of test_gpu_score.py."""
import pytest
import torch

import paper_2407_00611_amd as st
from oracle import score as so
from test_gpu_score import STEP, _positions, _run
from test_score_plan_constants import constant

pytestmark = pytest.mark.gpu

LIST = constant("kBlockList")                        # row blocks that a key tile's workgroup looks through at a time


@pytest.mark.parametrize("how", [dict(), dict(spans="random"), dict(where=8000, causal=True)], ids=["whole", "edges", "causal"])
def test_row_blocks_beyond_one_list(how):
    """Key tiles in one share each, so that a workgroup goes through its list twice: 520 row blocks of 32."""
    B, Hq, Hkv, D, Sq, Sk = 4, 16, 1, 64, 1040, 17300
    blocks = Sq * (Hq // Hkv) // 32
    assert blocks > LIST
    q, k = (torch.empty((B, S, h, D), dtype=torch.bfloat16, device="cuda") for S, h in ((Sq, Hq), (Sk, Hkv)))
    need = st.st_attn_score_workspace_bytes(q, k, k, 0, 0, how.get("causal", False), 0.1, backward=True)
    assert need == B * Hkv * blocks * (16 + 1024)          # the rows' statistics and what blocks see: no partial gradients
    del q, k
    _run("bf16", B, Hq, Hkv, D, Sq, Sk, **how)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 40), ("f32", 256)])
@pytest.mark.parametrize("case", [dict(Sq=1, Sk=1), dict(Sq=40, Sk=1), dict(Sq=33, Sk=70, spans=1), dict(Sq=33, Sk=70, spans=2), dict(Sq=1, Sk=3),
                                  dict(Sq=130, Sk=130, spans=1, Hq=40, Hkv=2)], ids=str)
def test_gradients_of_rows_that_see_a_key_or_two(dtype, D, case):
    """dQ and dK of a row with one key are rounding of terms that cancel: within the bound of those terms, and finite, in the
    accumulators and in the storage type, both of one call and of a call without accumulators."""
    c = dict(B=2, Hq=4, Hkv=2, spans=0, cap=5.0)
    c.update(case)
    t, one = (torch.bfloat16, STEP) if dtype == "bf16" else (torch.float32, 1e-5)
    g = torch.Generator().manual_seed(c["Sk"] + D)
    q, k, v, d_o = (torch.randn((c["B"], S, h, D), generator=g).to(t).cuda() for S, h in
                    ((c["Sq"], c["Hq"]), (c["Sk"], c["Hkv"]), (c["Sk"], c["Hkv"]), (c["Sq"], c["Hq"])))
    spans = None
    if c["spans"]:
        first = torch.randint(0, c["Sk"] - c["spans"] + 1, (c["B"], c["Sq"], 1), generator=g)
        spans = torch.cat([first, first + c["spans"]], -1).cuda()
    pos, kpos = _positions(0, c["Sq"]), _positions(0, c["Sk"])
    mods, ref = dict(softcap=c["cap"], spans=spans), dict(cap=c["cap"], span=spans)
    o, lse = st.st_attn_score_fwd(q, k, v, 0, 0, False, 0.2, **mods)
    o_ref, lse_ref = so.forward(q, k, v, pos, kpos, False, 0.2, **ref)
    delta = st.st_attn_delta(d_o, o)
    want = so.backward(q, k, v, d_o, lse_ref, so.delta(d_o, o_ref), pos, kpos, False, 0.2, **ref)
    sizes = so.magnitudes(q, k, v, d_o, lse_ref, pos, kpos, False, 0.2, **ref)[1:]
    acc = [torch.empty(x.shape, device="cuda") for x in (q, k, v)]
    low = [torch.empty_like(x) for x in (q, k, v)]
    st.st_attn_score_bwd(q, k, v, d_o, lse, delta, 0, 0, False, 0.2, dq_acc=acc[0], dk_acc=acc[1], dv_acc=acc[2], assign=True,
                         dq_lowp=low[0], dk_lowp=low[1], dv_lowp=low[2], **mods)
    alone = st.st_attn_score_bwd(q, k, v, d_o, lse, delta, 0, 0, False, 0.2, **mods)
    for a, l, b, y, size, n, name in zip(acc, low, alone, want, sizes, (3, 3, 2), ("dq", "dk", "dv")):
        # terms: P of one rounding (none in fp32 beside the sums'), dU of another; the exponent's error is lse's half step and the cap's
        bound = n * one * (1 if dtype == "bf16" else 4) + 2.0 ** -22 * c["cap"]
        assert torch.isfinite(a).all() and torch.isfinite(l).all(), name
        assert ((a.double() - y).abs() <= bound * (size + y.abs()) + 1e-6).all(), name
        assert torch.equal(l, a.to(t)) and torch.equal(l, b), f"{name} in the storage type"
