"""Refusals of the paged cache's calls: nothing here launches anything (no GPU needed)."""

import ctypes

import pytest

from paper_2506_02850_b200 import binding as B
from paper_2506_02850_b200 import build as builder

from .test_abi import device_pointers


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return B.lib()


def cache(**kw):
    p0, _, p1 = device_pointers()
    c = dict(k_pool=p0, v_pool=p1, block_table=p0 + (2 << 20), kv_len=p0 + (3 << 20), n_pages=8, Hkv=2, page_size=16, dh=64, n_seqs=3,
             max_pages=2)
    c.update(kw)
    return B.PagedCache(**c)


def launches(lib, fn, *args):
    assert lib.metok_profile_begin() == 0
    rc = fn(*args)
    return rc, lib.metok_profile_end(None, 0)


BAD_CACHES = [(dict(n_pages=0), -1), (dict(Hkv=0), -1), (dict(n_seqs=0), -1), (dict(max_pages=0), -1), (dict(page_size=0), -1), (dict(dh=0), -1),
              (dict(block_table=None), -1), (dict(kv_len=None), -1), (dict(page_size=24), -2), (dict(page_size=8), -2), (dict(page_size=512), -2),
              (dict(dh=96), -2), (dict(n_pages=1 << 30), -2), (dict(max_pages=(1 << 20) + 1), -2)]


def test_append_refuses(lib):
    p0, odd, p1 = device_pointers()
    fn = lib.metok_paged_append
    names = ["dtype", "c", "k_new", "v_new", "k_head", "k_row", "v_head", "v_row", "n_new", "off", "pos", "pos_new", "mass", "mass_new", "new_len",
             "status", "stream"]

    def call(c=None, **kw):
        a = dict(dtype=B.BF16, c=ctypes.byref(c or cache()), k_new=p0, v_new=p1, k_head=3 * 64, k_row=64, v_head=192, v_row=64, n_new=3, off=None,
                 pos=p0, pos_new=p0, mass=p0, mass_new=p0, new_len=p1, status=p0, stream=None)
        a.update(kw)
        return launches(lib, fn, *[a[n] for n in names])

    for kw, rc in BAD_CACHES + [(dict(k_pool=None), -1), (dict(v_pool=p0 + 4), -1)]:
        assert call(cache(**kw)) == (rc, 0), kw
    for kw in [dict(dtype=5), dict(k_new=None), dict(v_new=odd), dict(n_new=-1), dict(n_new=2), dict(pos=None), dict(mass=None), dict(k_row=60), dict(k_row=32),
               dict(v_head=-8), dict(v_row=68), dict(new_len=None), dict(status=None), dict(off=p0 + 2), dict(new_len=p0 + (3 << 20) + 8)]:
        assert call(**kw) == (-1, 0), kw


def test_attention_refuses(lib):
    p0, odd, p1 = device_pointers()
    fn = lib.metok_paged_attention
    names = ["dtype", "c", "q", "q_seq", "q_head", "Hq", "scale", "cap", "slopes", "pos", "mass", "out", "out_seq", "out_head", "lse", "status", "ws",
             "ws_bytes", "stream"]

    def call(c=None, **kw):
        a = dict(dtype=B.BF16, c=ctypes.byref(c or cache()), q=p0, q_seq=256, q_head=64, Hq=4, scale=0.1, cap=0.0, slopes=p0, pos=p0, mass=p1, out=p1,
                 out_seq=256, out_head=64, lse=p0, status=p0, ws=p0, ws_bytes=1 << 24, stream=None)
        a.update(kw)
        return launches(lib, fn, *[a[n] for n in names])

    for kw, rc in BAD_CACHES + [(dict(k_pool=None), -1), (dict(v_pool=p0 + 4), -1)]:
        assert call(cache(**kw)) == (rc, 0), kw
    for kw in [dict(dtype=-1), dict(q=None), dict(out=odd), dict(Hq=0), dict(Hq=3), dict(q_head=60), dict(out_head=32), dict(out_seq=0), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")),
               dict(status=None), dict(slopes=p0 + 1), dict(mass=p0 + 2)]:
        assert call(**kw) == (-1, 0), kw
    assert call(Hq=2050) == (-2, 0)
    assert call(ws=None) == (-3, 0) and call(ws_bytes=64) == (-3, 0)
    c = cache()
    size = lambda hq, mass: lib.metok_paged_attention_workspace_bytes(B.BF16, ctypes.byref(c), hq, mass)
    assert 0 < size(4, 0) < size(4, 1) and size(3, 0) == 0
    assert call(ws_bytes=size(4, 1) - 1) == (-3, 0)


def test_evict_refuses(lib):
    p0, odd, p1 = device_pointers()
    fn = lib.metok_paged_evict
    names = ["dtype", "c", "ks", "vs", "L", "budget", "sink", "recent", "pos", "mass", "keep", "new_len", "status", "ws", "ws_bytes", "stream"]
    at = lambda *p: (ctypes.c_void_p * len(p))(*p)
    ks, vs = at(p0, p1), at(p0 + (4 << 20), p0 + (5 << 20))

    def call(c=None, **kw):
        a = dict(dtype=B.F32, c=ctypes.byref(c or cache()), ks=ks, vs=vs, L=2, budget=20, sink=2, recent=4, pos=p0, mass=p0, keep=p0, new_len=p1,
                 status=p0, ws=p0, ws_bytes=1 << 24, stream=None)
        a.update(kw)
        return launches(lib, fn, *[a[n] for n in names])

    for kw, rc in BAD_CACHES:
        assert call(cache(**kw)) == (rc, 0), kw
    for kw in [dict(dtype=2), dict(ks=None), dict(ks=at(p0, None)), dict(vs=at(p0 + (4 << 20), odd)), dict(L=0), dict(budget=0), dict(budget=33),
               dict(sink=-1), dict(recent=0), dict(pos=None), dict(mass=None), dict(keep=None), dict(status=p0 + 1), dict(new_len=p0 + (3 << 20) + 4),
               dict(ks=at(p0, p0)), dict(vs=at(p1, p0 + (5 << 20))), dict(vs=at(p0, p0 + (5 << 20)))]:
        assert call(**kw) == (-1, 0), kw
    assert call(cache(n_seqs=40000)) == (-2, 0)                           # 80 000 problems
    assert call(L=1025, ks=at(*[p0] * 1025), vs=at(*[p1] * 1025)) == (-2, 0)
    assert call(ws=None) == (-3, 0) and call(ws_bytes=16) == (-3, 0)
