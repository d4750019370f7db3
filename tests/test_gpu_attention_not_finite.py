"""Logits that are no finite numbers, where rows see them: a NaN or +infinity makes the row's out and lse NaN, -infinity is a weight
of 0, and no other row changes.  Wherever the keys are cut among processors, and on either pipe that makes weights.

Tolerances as in test_gpu_prompt_attention.py and test_gpu_paged.py."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

from . import test_gpu_paged as P
from . import test_gpu_prompt_attention as Q

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]
INF = float("inf")

# query heads, K/V heads, queries, keys: one tile; several whole pairs; keys cut among processors (both types), with parts of one
# tile and of more
SHAPES = [(2, 1, 50, 60), (4, 2, 300, 300), (4, 2, 5, 3000), (14, 2, 33, 9000)]


def call(q, k, v, scale, **kw):
    got = B.metok_prefill_attention(q, k, v, scale, with_lse=True, **kw)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    return Q.num(got["out"]), Q.num(got["lse"])


def tolerance(want, dtype):
    return want["out_err"] + Q.HALF[dtype] * np.abs(want["out"]) + (2.0 ** -8 * want["absv"] if dtype == torch.bfloat16 else 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n_q,n_k", SHAPES)
@pytest.mark.parametrize("softcap,bias", [(0.0, False), (4.0, True)])
def test_a_nan_in_k_reaches_the_rows_that_see_it(dtype, dh, Hq, Hkv, n_q, n_k, softcap, bias):
    g = Q.gen(n_k + dh)
    # (logits of deviation 3 go beyond a cap of 4 in every tile)
    q, k, v = Q.rows(g, Hq, n_q, dh, dtype, 3.0), Q.rows(g, Hkv, n_k, dh, dtype), Q.rows(g, Hkv, n_k, dh, dtype)
    slopes = torch.linspace(0.0, 0.01, Hq, device="cuda") if bias else None
    kw = dict(softcap=softcap, slopes=slopes)
    want = A.prompt_attention(Q.num(q), Q.num(k), Q.num(v), dh ** -0.5, softcap=softcap, slopes=Q.num(slopes))
    tol = tolerance(want, dtype)
    first = n_k - n_q
    at = sorted({0, 6, 7, n_k // 2, n_k // 2 + 3, n_k - 65, n_k - 64, n_k - 11, n_k - 2, n_k - 1} & set(range(n_k)))
    for j in at:
        bad = k.clone()
        bad[0, j, 5] = float("nan")
        out, lse = call(q, bad, v, dh ** -0.5, **kw)
        sees = np.zeros((Hq, n_q), bool)
        sees[:Hq // Hkv] = first + np.arange(n_q) >= j
        assert np.isnan(lse[sees]).all() and np.isnan(out[sees]).all(), j
        assert (np.abs(out - want["out"]) <= tol)[~sees].all(), j
        assert (np.abs(lse - want["lse"]) <= want["lse_err"] + 2.0 ** -23 * np.abs(want["lse"]))[~sees].all(), j
    # a block of them: whole groups of keys without a number
    bad = k.clone()
    bad[0, n_k // 3:] = float("nan")
    out, lse = call(q, bad, v, dh ** -0.5, **kw)
    sees = np.zeros((Hq, n_q), bool)
    sees[:Hq // Hkv] = first + np.arange(n_q) >= n_k // 3
    assert np.isnan(lse[sees]).all() and np.isnan(out[sees]).all()
    assert (np.abs(out - want["out"]) <= tol)[~sees].all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,n_q,n_k", SHAPES)
@pytest.mark.parametrize("softcap", [0.0, 4.0])
def test_a_query_of_nan_or_infinity(dtype, Hq, Hkv, n_q, n_k, softcap):
    g = Q.gen(n_k)
    q, k, v = Q.rows(g, Hq, n_q, 64, dtype, 3.0), Q.rows(g, Hkv, n_k, 64, dtype), Q.rows(g, Hkv, n_k, 64, dtype)
    want = A.prompt_attention(Q.num(q), Q.num(k), Q.num(v), 0.125, softcap=softcap)
    tol = tolerance(want, dtype)
    for value in (float("nan"), INF, -INF):
        bad = q.clone()
        row = n_q - 2 if n_q > 2 else 0
        bad[1, row, 9] = value
        out, lse = call(bad, k, v, 0.125, softcap=softcap)
        other = np.ones((Hq, n_q), bool)
        other[1, row] = False
        assert (np.abs(out - want["out"]) <= tol)[other].all()
        if softcap and not np.isnan(value):            # +-cap everywhere: two weights, e^2cap apart
            continue
        assert np.isnan(lse[1, row]) and np.isnan(out[1, row]).all(), value


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,n_q,n_k", SHAPES)
def test_infinite_logits(dtype, Hq, Hkv, n_q, n_k):
    """K of +infinity in one element: +infinity for rows whose q is positive there, -infinity for the others."""
    g = Q.gen(n_k + 1)
    q, k, v = Q.rows(g, Hq, n_q, 64, dtype, 3.0), Q.rows(g, Hkv, n_k, 64, dtype), Q.rows(g, Hkv, n_k, 64, dtype)
    q[:, :, 0] = torch.where(torch.arange(n_q, device="cuda") % 3 == 0, 1.0, -1.0).to(dtype)
    up = np.broadcast_to(np.arange(n_q) % 3 == 0, (Hq, n_q))
    for j in (0, 7, n_k // 2, n_k - 7):
        bad = k.clone()
        bad[:, j, 0] = INF
        there = [i for i in range(n_k) if i != j]
        for softcap in (0.0, 4.0):
            out, lse = call(q, bad, v, 0.125, causal=False, softcap=softcap)
            if softcap:                                # +-cap: one logit known to the last bits of the cap
                for h in range(Hq):
                    hk = h // (Hq // Hkv)
                    x, err = A.logits(Q.num(q)[h], Q.num(k)[hk], 0.125, softcap)
                    x[:, j] = np.where(up[h], softcap, -softcap)
                    err[:, j] = 16 * A.STEP * softcap
                    want, _, p, out_err, _, _ = A.weigh(x, err, np.ones(x.shape, bool), Q.num(v)[hk])
                    tol = out_err + Q.HALF[dtype] * np.abs(want) + (2.0 ** -8 * (p @ np.abs(Q.num(v)[hk])) if dtype == torch.bfloat16 else 0)
                    assert (np.abs(out[h] - want) <= tol).all(), (j, h)
                continue
            want = A.prompt_attention(Q.num(q), Q.num(k)[:, there], Q.num(v)[:, there], 0.125, causal=False)
            assert np.isnan(out[up]).all() and np.isnan(lse[up]).all(), j
            assert (np.abs(out - want["out"]) <= tolerance(want, dtype))[~up].all(), j
            assert (np.abs(lse - want["lse"]) <= want["lse_err"] + 2.0 ** -23 * np.abs(want["lse"]))[~up].all(), j


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq", [2, 6])
def test_one_token_over_a_cache(dtype, Hq):
    c = P.Cache([700, 3000, 40], 2, 64, 16, dtype, seed=5)
    g = Q.gen(6)
    q = Q.rows(g, 3, Hq, 64, dtype, 2.0)
    q[:, :, 0] = 1.0
    q[1, 1, 0] = -1.0
    want = P.A.paged_attention(P.num(q), P.num(c.k[0]), P.num(c.v[0]), c.table_np, c.lens, 0.125)
    tol = want["out_err"] + P.HALF[dtype] * np.abs(want["out"]) + 2.0 ** -16 * want["absv"]
    for j in (0, 7, 1500, 2999):
        for value in (float("nan"), INF):
            k = c.k[0].clone()
            k[int(c.table_np[1, j // 16]), 0, j % 16, 0] = value
            got = B.metok_paged_attention(q, k, c.v[0], c.block_table, c.kv_len, 0.125, with_lse=True)
            torch.cuda.synchronize()
            out, lse = P.num(got["out"]), P.num(got["lse"])
            hit = np.zeros((3, Hq), bool)
            hit[1, :Hq // 2] = True
            if value == INF and Hq > 2:
                hit[1, 1] = False                      # -infinity there: a weight of 0
            assert np.isnan(out[hit]).all() and np.isnan(lse[hit]).all()
            hit[1, :Hq // 2] = True
            assert (np.abs(out - want["out"]) <= tol)[~hit].all()


@pytest.mark.parametrize("dtype", TYPES)
def test_nothing_but_minus_infinity(dtype):
    """A row all of whose logits are -infinity is as one that sees no key."""
    g = Q.gen(8)
    for n_k in (60, 3000):
        q, k, v = Q.rows(g, 2, 5, 64, dtype), Q.rows(g, 1, n_k, 64, dtype), Q.rows(g, 1, n_k, 64, dtype)
        k[:, :, 3] = INF
        q[0, :, 3], q[1, :, 3] = -1.0, 1.0
        out, lse = call(q, k, v, 0.125)
        assert (out[0] == 0).all() and (lse[0] == -INF).all() and np.isnan(out[1]).all() and np.isnan(lse[1]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_cache_of_nothing_but_minus_infinity(dtype):
    """A token all of whose logits are -infinity is as one of an empty cache; the other sequences are served."""
    c = P.Cache([700, 33], 1, 64, 16, dtype, seed=5)
    g = Q.gen(9)
    q = Q.rows(g, 2, 4, 64, dtype)
    q[0, :, 3] = -1.0
    q[1, :, 3] = 0.0
    k = c.k[0].clone()
    k[[int(p) for p in c.table_np[0] if p < c.n_pages], :, :, 3] = INF
    mass = c.mass[0].clone()
    got = B.metok_paged_attention(q, k, c.v[0], c.block_table, c.kv_len, 0.125, mass=mass, with_lse=True)
    torch.cuda.synchronize()
    assert (got["out"][0] == 0).all() and (got["lse"][0] == -INF).all() and torch.equal(mass[0], c.mass[0, 0])
    assert torch.isfinite(got["out"][1].float()).all() and torch.isfinite(got["lse"][1]).all() and (mass[1, :33] > c.mass[0, 1, :33]).any()
