"""Refusals of metok_prefill_attention: nothing here launches anything (no GPU needed)."""

import ctypes

import pytest

from paper_2506_02850_b200 import binding as B
from paper_2506_02850_b200 import build as builder

from .test_abi import device_pointers


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return B.lib()


def params(**kw):
    p0, _, p1 = device_pointers()
    p = dict(q=p0, k=p1, v=p0 + (2 << 20), out=p0 + (3 << 20), lse=p0 + (4 << 20), q_head=10 * 64, q_row=64, k_head=20 * 64, k_row=64, v_head=20 * 64, v_row=64,
             out_head=10 * 64, out_row=64, Hq=4, Hkv=2, dh=64, n_q=10, n_k=20, n_seq=2, seq_q=p0, seq_k=p0, prefix_len=p0, positions=p0, slopes=p0,
             softmax_scale=0.125, softcap=0.0, causal=1)
    p.update(kw)
    return B.AttentionParams(**p)


def test_refusals(lib):
    p0, odd, _ = device_pointers()

    def call(dtype=B.BF16, status=p0, ws=p0, ws_bytes=1 << 26, **kw):
        assert lib.metok_profile_begin() == 0
        rc = lib.metok_prefill_attention(dtype, ctypes.byref(params(**kw)), status, ws, ws_bytes, None)
        return rc, lib.metok_profile_end(None, 0)

    for kw in [dict(dtype=9), dict(status=None), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=odd), dict(out=odd), dict(Hq=3), dict(Hq=0), dict(Hkv=0),
               dict(dh=0), dict(n_q=-1), dict(n_k=-1), dict(n_seq=0), dict(seq_q=None), dict(seq_k=None), dict(seq_q=None, seq_k=None), dict(q_row=56), dict(k_row=0),
               dict(v_row=68), dict(out_row=32), dict(out_head=32), dict(k_head=-64), dict(q_head=4), dict(softmax_scale=0.0), dict(softmax_scale=-1.0),
               dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(softcap=-2.0), dict(softcap=float("inf")), dict(softcap=float("nan")),
               dict(seq_q=p0 + 2), dict(positions=p0 + 1), dict(slopes=p0 + 3), dict(lse=p0 + 2), dict(prefix_len=p0 + 1)]:
        assert call(**kw) == (-1, 0), kw
    for kw in [dict(dh=96), dict(dh=256), dict(n_q=(1 << 24) + 1), dict(n_k=(1 << 24) + 1), dict(n_seq=8193), dict(Hq=65536, Hkv=1)]:
        assert call(**kw) == (-2, 0), kw
    # few rows over many keys are split, which takes a workspace
    few = dict(n_k=20000, seq_q=None, seq_k=None, n_seq=1)
    need = lib.metok_prefill_attention_workspace_bytes(B.BF16, ctypes.byref(params(**few)))
    assert need > 0
    assert call(ws=None, **few) == (-3, 0) and call(ws_bytes=need - 1, **few) == (-3, 0)
    assert lib.metok_prefill_attention_workspace_bytes(B.BF16, ctypes.byref(params(dh=32))) == 0
