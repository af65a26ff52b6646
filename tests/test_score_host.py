"""Refusals of the entry points for modified scores, spans, norms and rotations: on the host, before anything is launched (CPU)."""
import ctypes as C

import pytest
import torch

import paper_2407_00611_amd as st
from paper_2407_00611_amd import api

lib = api._lib
PTR = 0x10000                                        # never read: every call here ends before a launch


def _desc(**kw):
    x = dict(dtype=1, B=1, Hq=4, Hkv=2, D=128, Sq=8, Sk=8, q_offset=0, k_offset=0, causal=0, scale=0.1, q_seg=0, q_offset2=0)
    x.update(kw)
    return api.st_block_desc(*[x[n] for n, _ in api.st_block_desc._fields_])


def _view(ptr=PTR, s=512, h=128, b=4096):
    return api.st_tensor(ptr, b, s, h)


def _fwd(d=None, m=None, q=None, k=None, v=None, o=PTR, lse=PTR, low=None, ws=None, size=0):
    d, q, k, v = d or _desc(), q or _view(), k or _view(), v or _view()
    return lib.st_attn_score_fwd(C.byref(d), C.byref(m) if m else None, C.byref(q), C.byref(k), C.byref(v), o, lse, low, ws, size, None)


def _bwd(d=None, m=None, flags=0, acc=(PTR, 2 * PTR, 3 * PTR), low=(None, None, None), ws=None, size=0, lse=PTR, q=None):
    d, q, x = d or _desc(), q or _view(), _view()
    return lib.st_attn_score_bwd(C.byref(d), C.byref(m) if m else None, C.byref(q), C.byref(x), C.byref(x), C.byref(x), lse, PTR, flags, *acc, *low,
                                 ws, size, None)


def test_score_shapes_and_modifications():
    for call in (_fwd, _bwd):
        assert call(_desc(dtype=5)) == 1 and call(_desc(Hq=3)) == 1 and call(_desc(Sq=-1)) == 1
        assert call(_desc(D=80)) == 2 and call(_desc(dtype=0, D=260)) == 2 and call(_desc(dtype=0, D=12)) == 2
        assert call(_desc(scale=0.0)) == 1 and call(_desc(q_seg=8, q_offset2=100)) == 1
        assert call(_desc(Sq=1 << 30, B=64)) == 2 and call(_desc(Sq=1 << 30, Hq=64)) == 2
        for cap in (-1.0, float("nan"), float("inf"), 3.4e38, 1e-40):
            assert call(m=api.st_score(cap, None, None)) == 1, cap
        assert call(_desc(Sk=(1 << 24) + 1), m=api.st_score(0.0, PTR, None)) == 2
        assert call(m=api.st_score(1025.0, None, None)) == 2                 # the hardware's exponential is not exact enough
        assert call(m=api.st_score(0.0, PTR + 2, None)) == 3 and call(m=api.st_score(0.0, None, PTR + 8)) == 3
        assert call(q=_view(PTR + 8)) == 3 and call(q=_view(s=513)) == 3 and call(q=_view(None)) == 1 and call(q=_view(b=-4096)) == 1


def test_forward_outputs():
    assert _fwd(o=None, low=None) == 1 and _fwd(o=PTR, low=PTR) == 1
    assert _fwd(o=PTR + 4) == 3 and _fwd(o=None, low=PTR + 8) == 3 and _fwd(lse=None) == 1 and _fwd(lse=PTR + 4) == 3
    assert _fwd(_desc(Sq=0), o=None, lse=None) == 0 and _fwd(_desc(B=0), o=None, lse=None) == 0     # nothing to do


def test_backward_outputs():
    assert _bwd(flags=2) == 1 and _bwd(lse=None) == 1
    assert _bwd(acc=(None, 2 * PTR, 3 * PTR), low=(PTR, None, None)) == 1        # nothing to add to
    assert _bwd(flags=1, acc=(PTR, None, 3 * PTR)) == 1 and _bwd(flags=1, low=(None, 2 * PTR, None)) == 1
    assert _bwd(acc=(PTR, PTR, 3 * PTR)) == 1 and _bwd(low=(None, 3 * PTR, None)) == 1 and _bwd(low=(None, 5 * PTR, 5 * PTR)) == 1   # shared memory
    assert _bwd(acc=(PTR, PTR + 8, 3 * PTR)) == 3 and _bwd(low=(0x20008, None, None)) == 3


def test_workspaces():
    few = _desc(Sq=1, Sk=100000)
    m = api.st_score(0.0, None, PTR)
    assert lib.st_attn_score_workspace_bytes(C.byref(few), None, 0) > 0
    assert _fwd(few) == 5 and _fwd(few, ws=PTR, size=1000) == 5 and _fwd(few, ws=PTR + 128, size=1 << 30) == 3
    assert _bwd(m=m) == 5                                                # the statistics of the rows
    assert lib.st_attn_score_workspace_bytes(C.byref(_desc(Sq=0)), None, 1) == 0
    assert lib.st_attn_score_workspace_bytes(C.byref(_desc(D=80)), None, 1) == 0
    # enough places for every tile: nothing is split
    assert lib.st_attn_score_workspace_bytes(C.byref(_desc(B=8, Hq=32, Hkv=8, Sq=4096, Sk=4096)), None, 0) == 0


def test_mask_spans():
    call = lambda B=1, Sq=4, off=0, seg=0, off2=0, bounds=PTR, n=1, prefix=None, spans=PTR: lib.st_mask_spans(B, Sq, off, seg, off2, 1, bounds, n, prefix, spans, None)
    assert call(B=-1) == 1 and call(n=-1) == 1 and call(bounds=None) == 1 and call(spans=None) == 1 and call(seg=4, off2=9) == 1
    assert call(bounds=PTR + 4) == 3 and call(spans=PTR + 8) == 3 and call(prefix=PTR + 4) == 3
    assert call(Sq=0, bounds=None, spans=None) == 0


def _rope(**kw):
    x = dict(dtype=1, B=1, S=4, Hq=4, Hkv=2, D=128, rot=128, pairing=0, norm=1, eps=1e-6, n_axes=1, axis_pairs=(64,), offset=0, seg=0, offset2=0)
    x.update(kw)
    x["axis_pairs"] = (C.c_int32 * 4)(*x["axis_pairs"])
    return api.st_rope_desc(*[x[n] for n, _ in api.st_rope_desc._fields_])


def _rope_fwd(d=None, wq=None, wk=None, freq=PTR, pos=None, q=None, out=None):
    d, x = d or _rope(), _view()
    return lib.st_qk_rope_fwd(C.byref(d), C.byref(q or x), C.byref(x), wq, wk, freq, pos, C.byref(out or x), C.byref(x), None)


def _rope_bwd(d=None, dd=0, flags=0, wq=None, dwq=None, dwk=None, ws=None, size=0, freq=PTR, pos=None, q=None):
    d, x = d or _rope(), _view()
    return lib.st_qk_rope_bwd(C.byref(d), C.byref(q or x), C.byref(x), C.byref(x), C.byref(x), dd, wq, None, freq, pos, flags, C.byref(x), C.byref(x),
                              dwq, dwk, ws, size, None)


def test_rope_descriptors():
    for call in (_rope_fwd, _rope_bwd):
        for bad in (dict(dtype=3), dict(S=-1), dict(Hq=0), dict(Hkv=-1), dict(rot=3), dict(rot=130), dict(rot=-2), dict(pairing=2), dict(norm=2),
                    dict(eps=-1.0), dict(eps=float("nan")), dict(n_axes=0), dict(n_axes=5), dict(axis_pairs=(63,)), dict(axis_pairs=(65, -1), n_axes=2),
                    dict(axis_pairs=(32, 32), n_axes=2), dict(seg=4, offset2=9), dict(seg=2, offset2=1)):
            assert call(_rope(**bad)) == 1, bad
        assert call(_rope(D=260, rot=64, axis_pairs=(32,))) == 2 and call(_rope(D=12, rot=0, axis_pairs=(0,))) == 2
        assert call(_rope(S=1 << 26)) == 2 and call(_rope(Hq=70000)) == 2 and call(_rope(Hq=16000, Hkv=400)) == 2
        assert call(freq=None) == 1 and call(freq=PTR + 4) == 3 and call(pos=PTR + 2) == 3 and call(wq=PTR + 4) == 3
        assert call(_rope(seg=2, offset2=9), pos=PTR) == 1
        assert call(_rope(norm=0), wq=PTR) == 1
        assert call(q=_view(PTR + 8)) == 3 and call(q=_view(None)) == 1
    assert _rope_fwd(out=_view(PTR + 8)) == 3
    assert _rope_fwd(_rope(S=0)) == 0 and _rope_bwd(_rope(S=0)) == 0


def test_rope_gradients():
    assert _rope_bwd(dd=7) == 1 and _rope_bwd(_rope(dtype=0), dd=1) == 1 and _rope_bwd(flags=2) == 1
    assert _rope_bwd(dwq=PTR) == 5 and _rope_bwd(dwq=PTR, ws=PTR, size=16) == 5 and _rope_bwd(dwq=PTR, ws=PTR + 64, size=1 << 20) == 3
    assert _rope_bwd(dwq=PTR, dwk=PTR, ws=PTR, size=1 << 20) == 1 and _rope_bwd(dwq=PTR + 4) == 3 and _rope_bwd(_rope(norm=0), dwk=PTR) == 1
    assert lib.st_qk_rope_bwd_workspace_bytes(C.byref(_rope(S=0))) == 0 and lib.st_qk_rope_bwd_workspace_bytes(C.byref(_rope(norm=0))) == 0


def test_the_wrappers_refuse_what_the_calls_cannot_see():
    x = torch.zeros((1, 8, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on a GPU"):
        st.st_attn_score_fwd(x, x, x, 0, 0, True, 0.1)
    with pytest.raises(ValueError, match="on a GPU"):
        st.st_mask_spans(torch.zeros((1, 2), dtype=torch.int64), 8, 0, True)
    with pytest.raises(ValueError, match="on a GPU"):
        st.st_qk_rope_fwd(x, x, torch.zeros(32, dtype=torch.float64))
    for bad in (dict(k=x[:, :, :, :32]), dict(v=x[:, :4]), dict(k=x.float()), dict(slopes=torch.zeros(3)), dict(slopes=torch.zeros(4).double()),
                dict(spans=torch.zeros((1, 8), dtype=torch.int64)), dict(spans=torch.zeros((1, 8, 2), dtype=torch.int32))):
        args = dict(q=x, k=x, v=x, slopes=None, spans=None)
        args.update(bad)
        with pytest.raises(ValueError):
            api._score_desc(args["q"], args["k"], args["v"], 0, 0, True, 0.1, 0.0, args["slopes"], args["spans"])
    f = torch.zeros(32, dtype=torch.float64)
    for bad in (dict(pairs="odd"), dict(axes=[16, 15]), dict(axes=[8] * 5), dict(freq=f.float()), dict(positions=torch.zeros((2, 1, 8), dtype=torch.int32)),
                dict(positions=torch.zeros((1, 1, 8), dtype=torch.int64)), dict(k=x.float()), dict(k=x[:, :4]), dict(q_weight=torch.ones(32))):
        args = dict(q=x, k=x, freq=f, offset=0, positions=None, axes=None, pairs="halves", norm=True, eps=1e-6, q_weight=None, k_weight=None)
        args.update(bad)
        with pytest.raises(ValueError):
            api._rope_desc(**args)
