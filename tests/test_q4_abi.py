"""Refusals of the calls on heads and on a cache held in 4 bits: nothing here launches anything (no GPU needed)."""

import ctypes

import pytest

from paper_2506_02850_b200 import binding as B
from paper_2506_02850_b200 import build as builder

from .test_abi import device_pointers
from .test_paged_abi import BAD_CACHES, cache, launches


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return B.lib()


def test_rotate_refuses(lib):
    p0, odd, p1 = device_pointers()
    M = 1 << 20

    def call(dtype=B.BF16, axis=None, **kw):
        a = dict(q=p0, k=p0 + M, q_out=p0 + 2 * M, k_out=p0 + 3 * M, q_head=64, q_row=320, k_head=64, k_row=320, qo_head=192, qo_row=64, ko_head=192, ko_row=64,
                 Hq=4, Hkv=1, dh=64, n=3, rotary_dim=64, interleaved=0, n_axes=1, norm=1, q_weight=p0, k_weight=p0, inv_freq=p0, positions=p0,
                 pair_axis=None, eps=1e-6)
        a.update(kw)
        if axis is not None:
            a["pair_axis"] = (ctypes.c_int32 * 64)(*axis)
        p = B.RotateParams(**a)
        return launches(lib, lib.metok_rotate_heads, dtype, ctypes.byref(p), None)

    assert launches(lib, lib.metok_rotate_heads, B.BF16, None, None) == (-1, 0)
    assert call(n=0) == (0, 0) and call()[0] in (0, -4)                  # sound arguments: launched, or there is no GPU
    for kw in [dict(dtype=3), dict(dtype=B.Q4), dict(q=None), dict(k=None), dict(q_out=odd), dict(k_out=odd), dict(q=odd), dict(Hq=0), dict(Hkv=-1), dict(n=-1),
               dict(dh=0), dict(rotary_dim=-16), dict(rotary_dim=72), dict(rotary_dim=80), dict(n_axes=0), dict(n_axes=5), dict(n_axes=2, positions=None),
               dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(inv_freq=None), dict(inv_freq=p0 + 2), dict(positions=p0 + 1),
               dict(q_weight=p0 + 2), dict(k_weight=p0 + 3), dict(q_head=60), dict(q_row=32), dict(k_row=-320), dict(qo_row=32), dict(qo_head=64, qo_row=64),
               dict(ko_row=60), dict(axis=[0] * 31 + [1] + [0] * 32), dict(axis=[-1] + [0] * 63), dict(n_axes=3, axis=[3] + [0] * 63),
               # outputs over inputs and over one another
               dict(q_out=p0, qo_head=192, qo_row=64), dict(q_out=p0 + M, qo_head=64, qo_row=320), dict(k_out=p0 + 2 * M), dict(k_out=p0, ko_head=64, ko_row=320),
               dict(k_out=p0 + 2 * M + 3 * 128, ko_head=64, ko_row=320, qo_head=64, qo_row=320)]:
        assert call(**kw) == (-1, 0), kw
    # in place, and side by side in one buffer
    assert call(q_out=p0, qo_head=64, qo_row=320, k=p0 + 512, k_out=p0 + 512, ko_head=64, ko_row=320)[0] in (0, -4)
    assert call(qo_head=64, qo_row=320, k_out=p0 + 2 * M + 512, ko_head=64, ko_row=320)[0] in (0, -4)
    assert call(dh=96) == (-2, 0) and call(dh=256) == (-2, 0)


def append_args(c, p0, p1, kw):
    a = dict(dtype=B.BF16, c=ctypes.byref(c), k_new=p0, v_new=p1, k_head=3 * 64, k_row=64, v_head=192, v_row=64, n_new=3, off=None,
             pos=p0, pos_new=p0, mass=p0, mass_new=p0, new_len=p1, status=p0, stream=None)
    a.update(kw)
    return list(a.values())


def test_append_refuses(lib):
    p0, odd, p1 = device_pointers()
    call = lambda c=None, **kw: launches(lib, lib.metok_paged_append_q4, *append_args(c or cache(), p0, p1, kw))
    for kw, rc in BAD_CACHES + [(dict(k_pool=None), -1), (dict(v_pool=p0 + 4), -1)]:
        assert call(cache(**kw)) == (rc, 0), kw
    for kw in [dict(dtype=5), dict(dtype=B.Q4), dict(k_new=None), dict(v_new=odd), dict(n_new=-1), dict(n_new=2), dict(pos=None), dict(mass=None), dict(k_row=60),
               dict(k_row=32), dict(v_head=-8), dict(v_row=68), dict(new_len=None), dict(status=None), dict(off=p0 + 2), dict(new_len=p0 + (3 << 20) + 8)]:
        assert call(**kw) == (-1, 0), kw
    # the other append takes no such cache
    assert launches(lib, lib.metok_paged_append, *append_args(cache(), p0, p1, dict(dtype=B.Q4))) == (-1, 0)


def test_read_refuses(lib):
    p0, odd, p1 = device_pointers()

    def call(c=None, **kw):
        a = dict(dtype=B.BF16, c=ctypes.byref(c or cache()), off=p0, first=p0, n=3, k=p0, v=p1, k_head=192, k_row=64, v_head=192, v_row=64, pos=p0,
                 pos_out=p0, status=p0, stream=None)
        a.update(kw)
        return launches(lib, lib.metok_paged_read_q4, *a.values())

    for kw, rc in BAD_CACHES + [(dict(k_pool=None), -1), (dict(v_pool=p0 + 4), -1)]:
        assert call(cache(**kw)) == (rc, 0), kw
    for kw in [dict(dtype=5), dict(dtype=B.Q4), dict(k=None), dict(v=odd), dict(n=-1), dict(off=None), dict(off=p0 + 2), dict(first=p0 + 1), dict(pos=None),
               dict(pos_out=p0 + 2), dict(status=None), dict(k_row=60), dict(k_row=32), dict(v_head=-8), dict(v_row=68), dict(k_head=64), dict(v=p0 + 64)]:
        assert call(**kw) == (-1, 0), kw


def test_attention_refuses(lib):
    p0, odd, p1 = device_pointers()

    def call(c=None, **kw):
        a = dict(dtype=B.BF16, c=ctypes.byref(c or cache()), q=p0, q_seq=256, q_head=64, Hq=4, scale=0.1, cap=0.0, slopes=p0, pos=p0, mass=p1, out=p1,
                 out_seq=256, out_head=64, lse=p0, status=p0, ws=p0, ws_bytes=1 << 24, stream=None)
        a.update(kw)
        return launches(lib, lib.metok_paged_attention_q4, *a.values())

    for kw, rc in BAD_CACHES + [(dict(k_pool=None), -1), (dict(v_pool=p0 + 4), -1)]:
        assert call(cache(**kw)) == (rc, 0), kw
    for kw in [dict(dtype=-1), dict(dtype=B.Q4), dict(q=None), dict(out=odd), dict(Hq=0), dict(Hq=3), dict(q_head=60), dict(out_head=32), dict(out_seq=0), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")),
               dict(status=None), dict(slopes=p0 + 1), dict(mass=p0 + 2)]:
        assert call(**kw) == (-1, 0), kw
    assert call(Hq=2050) == (-2, 0)
    assert call(ws=None) == (-3, 0) and call(ws_bytes=64) == (-3, 0)
    c = cache()
    size = lambda hq, mass: lib.metok_paged_attention_q4_workspace_bytes(B.BF16, ctypes.byref(c), hq, mass)
    assert 0 < size(4, 0) < size(4, 1) and size(3, 0) == 0 and lib.metok_paged_attention_q4_workspace_bytes(B.Q4, ctypes.byref(c), 4, 0) == 0
    assert call(ws_bytes=size(4, 1) - 1) == (-3, 0)


def test_evict_refuses_pools_that_overlap(lib):
    p0, odd, p1 = device_pointers()
    at = lambda *p: (ctypes.c_void_p * len(p))(*p)
    pool = 8 * 2 * 9 * 64                                               # bytes of one

    def call(ks, vs, c=None, **kw):
        a = dict(dtype=B.Q4, c=ctypes.byref(c or cache()), ks=at(*ks), vs=at(*vs), L=1, budget=20, sink=2, recent=4, pos=p0, mass=p0, keep=p0, new_len=p1,
                 status=p0, ws=None, ws_bytes=0, stream=None)
        a.update(kw)
        return launches(lib, lib.metok_paged_evict, *a.values())

    assert call([p0], [p0 + pool]) == (-3, 0)                           # next to one another: only the workspace is missing
    assert call([p0], [p0 + pool - 16]) == (-1, 0) and call([p0], [p0]) == (-1, 0) and call([odd], [p1]) == (-1, 0)
    for kw, rc in BAD_CACHES:
        assert call([p0], [p1], cache(**kw)) == (rc, 0), kw


def test_pool_sizes():
    assert B.q4_pool(3, 2, 32, 64, device="cpu").shape == (3, 2, 2, 576)
    with pytest.raises(ValueError):
        B.q4_pool(3, 2, 24, 64, device="cpu")
