"""Refusals of the cache's entry points: on the host, before anything is launched (CPU)."""
import ctypes as C

import pytest
import torch

import paper_2407_00611_amd as st
from paper_2407_00611_amd import api

lib = api._lib
PTR = 0x10000                                        # never read: every call here ends before a launch


def _view(ptr=PTR, b=1 << 16, s=512, h=128):
    return api.st_tensor(ptr, b, s, h)


def _cache(**kw):
    x = dict(dtype=1, n_pages=4, page=16, Hkv=2, D=128, B=1, width=3, k=_view(), v=_view(2 * PTR), k_scale=None, v_scale=None, table=PTR, lens=PTR)
    x.update(kw)
    return api.st_cache(*[x[n] for n, _ in api.st_cache._fields_])


def _rows(**kw):
    x = dict(dtype=1, T=1, Hq=4, max_rows=1, causal=1, window=0, scale=0.1, softcap=0.0, slopes=None)
    x.update(kw)
    return api.st_cache_rows(*[x[n] for n, _ in api.st_cache_rows._fields_])


def _rope(**kw):
    x = dict(dtype=1, B=1, S=4, Hq=4, Hkv=2, D=128, rot=128, pairing=0, norm=0, eps=1e-6, n_axes=1, axis_pairs=(C.c_int32 * 4)(64), offset=0, seg=0, offset2=0)
    x.update(kw)
    return api.st_rope_desc(*[x[n] for n, _ in api.st_rope_desc._fields_])


def _attn(r=None, c=None, starts=PTR, first=None, q=None, o=PTR, lse=PTR, low=None, ws=None, size=0):
    r, c, q = r or _rows(), c or _cache(), q or _view()
    return lib.st_attn_cache(C.byref(r), C.byref(c), starts, first, C.byref(q), o, lse, low, ws, size, None)


def _append(d=None, c=None, starts=PTR, q=None, k=None, v=None, qw=None, kw=None, freq=PTR, positions=None, out=None):
    d, c, q, k, v, out = d or _rope(), c or _cache(), q or _view(), k or _view(), v or _view(), out or _view()
    return lib.st_cache_append(C.byref(d), C.byref(c), starts, C.byref(q), C.byref(k), C.byref(v), qw, kw, freq, positions, C.byref(out), None)


def _read(c=None, first=None, count=4, dtype=1, k=None, v=None):
    c, k, v = c or _cache(), k or _view(), v or _view(2 * PTR)
    return lib.st_cache_read(C.byref(c), first, count, dtype, C.byref(k), C.byref(v), None)


BAD_CACHES = [(dict(dtype=3), 1), (dict(n_pages=-1), 1), (dict(B=-1), 1), (dict(width=-1), 1), (dict(Hkv=0), 1), (dict(D=0), 1),
              (dict(page=8), 2), (dict(page=48), 2), (dict(page=512), 2), (dict(page=0), 2), (dict(D=264), 2), (dict(D=12), 2),
              (dict(Hkv=20000), 2), (dict(B=65536), 2), (dict(width=1 << 27), 2), (dict(k=_view(None)), 1), (dict(v=_view(PTR + 8)), 3),
              (dict(k=_view(s=516)), 3), (dict(v=_view(s=1 << 20)), 2), (dict(v=_view(h=-128)), 1), (dict(k_scale=PTR), 1), (dict(dtype=2), 1), (dict(dtype=2, k_scale=PTR), 1),
              (dict(dtype=2, k_scale=PTR, v_scale=PTR, k=_view(s=520)), 3), (dict(lens=None), 1), (dict(table=None), 1), (dict(table=PTR + 2), 3),
              (dict(lens=PTR + 1), 3)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_caches(bad, status):
    for call in (_attn, _append, _read):
        assert call(c=_cache(**bad)) == status, (call, bad)
    r, c = _rows(), _cache(**bad)
    assert lib.st_attn_cache_workspace_bytes(C.byref(r), C.byref(c)) == 0


def test_pages_in_8_bits_have_heads_of_whole_loads():
    assert _read(c=_cache(dtype=2, D=72, k_scale=PTR, v_scale=PTR)) == 2


def test_attention():
    for bad, status in ((dict(dtype=2), 1), (dict(dtype=5), 1), (dict(dtype=0), 2), (dict(T=-1), 1), (dict(max_rows=-1), 1), (dict(window=-1), 1),
                        (dict(Hq=3), 1), (dict(Hq=0), 1), (dict(Hq=65536), 2), (dict(T=(1 << 25) + 1), 2), (dict(T=1 << 25, Hq=256), 2), (dict(scale=0.0), 1),
                        (dict(scale=float("nan")), 1), (dict(softcap=-1.0), 1), (dict(softcap=float("inf")), 1), (dict(softcap=1025.0), 2),
                        (dict(softcap=1e-40), 1), (dict(slopes=PTR + 2), 3)):
        assert _attn(_rows(**bad)) == status, bad
        r, c = _rows(**bad), _cache()
        assert lib.st_attn_cache_workspace_bytes(C.byref(r), C.byref(c)) == 0
    assert _attn(c=_cache(D=80)) == 2                                            # bf16: 64 or 128
    assert _attn(_rows(slopes=PTR), _cache(width=(1 << 20) + 1)) == 2            # distances that fp32 does not hold
    assert _attn(starts=None) == 1 and _attn(starts=PTR + 2) == 3 and _attn(first=PTR + 4) == 3
    assert _attn(q=_view(PTR + 8)) == 3 and _attn(q=_view(None)) == 1 and _attn(q=_view(s=513)) == 3
    assert _attn(o=None) == 1 and _attn(low=PTR) == 1 and _attn(o=PTR + 4) == 3 and _attn(o=None, low=PTR + 8) == 3
    assert _attn(lse=None) == 1 and _attn(lse=PTR + 4) == 3
    for nothing in (dict(r=_rows(T=0)), dict(c=_cache(B=0)), dict(r=_rows(max_rows=0))):
        assert _attn(**nothing, o=None, lse=None) == 0
    assert lib.st_attn_cache(None, None, None, None, None, None, None, None, None, 0, None) == 1


@pytest.mark.parametrize("dtype,Hq,Hkv,B,T", [(1, 32, 8, 1, 1), (1, 32, 8, 8, 8), (1, 32, 8, 16, 80), (1, 24, 24, 64, 64), (1, 8, 2, 64, 700), (0, 8, 2, 16, 16), (0, 8, 8, 3, 400)])
def test_a_window_needs_no_more_room_than_none(dtype, Hq, Hkv, B, T):
    """A workspace for rows without a window is enough for every window, and one for a longer table for every shorter one."""
    need = lambda width, window, causal=1: lib.st_attn_cache_workspace_bytes(C.byref(_rows(dtype=dtype, T=T, Hq=Hq, max_rows=T, window=window, causal=causal)),
                                                                             C.byref(_cache(dtype=dtype, Hkv=Hkv, B=B, width=width)))
    last = 0
    for width in list(range(1, 260, 3)) + [500, 1000, 8192]:
        most = need(width, 0)
        assert need(width, 0, 0) == most and need(width, 64, 0) == most
        assert max(need(width, w) for w in (1, 17, 300, 700, 1000, 1500, 2000, 2950, 3000, 4000, 10 ** 6)) <= most, width
        assert most >= last, width
        last = most


def test_appending():
    for bad, status in ((dict(dtype=2), 1), (dict(B=2), 1), (dict(B=0), 1), (dict(seg=2, offset2=9), 1), (dict(Hkv=1), 1), (dict(D=64, rot=64, axis_pairs=(C.c_int32 * 4)(32)), 1),
                        (dict(Hq=-1), 1), (dict(dtype=0), 2), (dict(S=-1), 1), (dict(S=(1 << 25) + 1), 2), (dict(rot=130), 1), (dict(rot=64), 1), (dict(pairing=2), 1),
                        (dict(norm=2), 1), (dict(norm=1, eps=-1.0), 1), (dict(n_axes=2), 1), (dict(Hq=16384), 2)):
        assert _append(_rope(**bad)) == status, bad
    assert _append(starts=None) == 1 and _append(starts=PTR + 1) == 3 and _append(freq=None) == 1 and _append(freq=PTR + 4) == 3
    for name in "qkv":
        assert _append(**{name: _view(None)}) == 1 and _append(**{name: _view(PTR + 2)}) == 3
    assert _append(out=_view(None)) == 1 and _append(qw=PTR) == 1 and _append(_rope(norm=1), kw=PTR + 4) == 3
    assert _append(_rope(S=0)) == 0 and _append(c=_cache(B=0)) == 0


def test_reading():
    assert _read(dtype=2) == 1 and _read(dtype=0) == 2 and _read(count=-1) == 1 and _read(first=PTR + 2) == 3
    assert _read(k=_view(None)) == 1 and _read(v=_view(PTR + 4)) == 3 and _read(v=_view()) == 1 and _read(count=0x7fffffff, c=_cache(Hkv=64)) == 2
    assert _read(count=0) == 0 and _read(c=_cache(B=0)) == 0
    c = _cache()
    assert lib.st_cache_read(C.byref(c), None, 4, 1, None, None, None) == 1


def test_the_wrapper_refuses_what_does_not_fit_together():
    k = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
    table, lens, starts = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    good = st.KVCache(k, k, table, lens)
    assert api._cache_desc(good).width == 3 and api._cache_desc(good).page == 16
    e = k.to(torch.float8_e4m3fn)
    s = torch.ones((4, 2), dtype=torch.uint8)
    assert api._cache_desc(st.KVCache(e, e, table, lens, s, s)).dtype == st.ST_E4M3
    for bad in (good._replace(k_scale=s), st.KVCache(e, e, table, lens), st.KVCache(e, e, table, lens, s, s[:3]), good._replace(lens=lens.long()),
                good._replace(table=table[0]), good._replace(v=k[:3]), good._replace(lens=torch.zeros(2, dtype=torch.int32)), good._replace(table=table.t())):
        if bad.table is not good.table and bad.table.dim() == 2 and bad.table.shape == (3, 1):
            bad = bad._replace(lens=torch.zeros(3, dtype=torch.int32), table=torch.zeros((3, 2), dtype=torch.int32)[:, :1])
        with pytest.raises(ValueError):
            api._cache_desc(bad)
    with pytest.raises(TypeError):
        api._cache_desc(good._replace(k=k.half(), v=k.half()))
    q = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16)
    for call in (lambda: st.st_attn_cache(q, starts, good, True, 0.1), lambda: st.st_cache_read(good, None, 4),
                 lambda: st.st_cache_append(q, q[:, :, :2], q[:, :, :2], starts, good, torch.zeros(32, dtype=torch.float64))):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
