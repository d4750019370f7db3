"""Pins of oracle/attention_oracle.py: closed forms, brute force over tiny inputs, and invariants.  CPU only."""

import itertools
import math

import numpy as np
import pytest

from oracle import attention_oracle as A


def brute(q, k, v, scale, seen, softcap=0.0, slope=0.0, far=None):
    """Sums over the keys in plain loops."""
    out, lse = np.zeros((len(q), v.shape[1])), np.full(len(q), -math.inf)
    for i in range(len(q)):
        xs = []
        for j in range(len(k)):
            x = scale * sum(float(a) * float(b) for a, b in zip(q[i], k[j]))
            if softcap:
                x = softcap * math.tanh(x / softcap)
            if far is not None:
                x -= slope * far[i][j]
            xs.append(x if seen[i][j] else None)
        total = sum(math.exp(x) for x in xs if x is not None)
        if total:
            lse[i] = math.log(total)
            for j, x in enumerate(xs):
                if x is not None:
                    out[i] += math.exp(x) / total * v[j]
    return out, lse


@pytest.mark.parametrize("causal,prefix,softcap,bias", [(True, 0, 0.0, False), (True, 3, 5.0, True), (False, 0, 2.0, False), (True, 9, 0.0, True)])
def test_prompt_attention_against_plain_loops(causal, prefix, softcap, bias):
    rng = np.random.default_rng(1)
    lq, lk = [3, 0, 4], [5, 2, 3]                              # the last document has a query that sees no key
    q, k, v = rng.standard_normal((4, 7, 6)), rng.standard_normal((2, 10, 6)), rng.standard_normal((2, 10, 6))
    sq, sk = np.concatenate([[0], np.cumsum(lq)]), np.concatenate([[0], np.cumsum(lk)])
    pos = np.sort(rng.choice(60, 10, replace=False))
    slopes = np.array([0.5, 0.25, 0.1, 0.0]) if bias else None
    got = A.prompt_attention(q, k, v, 0.7, sq, sk, [prefix] * 3, causal, softcap, slopes, pos if bias else None)
    for d, h in itertools.product(range(3), range(4)):
        Q, K, V = q[h, sq[d]:sq[d + 1]], k[h // 2, sk[d]:sk[d + 1]], v[h // 2, sk[d]:sk[d + 1]]
        at = [lk[d] - lq[d] + i for i in range(lq[d])]
        seen = [[not causal or j <= c or j < prefix for j in range(lk[d])] for c in at]
        P = pos[sk[d]:sk[d + 1]]
        far = [[abs(P[max(c, 0)] - P[j]) for j in range(lk[d])] for c in at] if bias else None
        out, lse = brute(Q, K, V, 0.7, seen, softcap, 0.0 if slopes is None else slopes[h], far)
        np.testing.assert_allclose(got["out"][h, sq[d]:sq[d + 1]], out, atol=1e-12)
        np.testing.assert_allclose(got["lse"][h, sq[d]:sq[d + 1]], lse, atol=1e-12)


def test_paged_attention_is_prompt_attention_of_one_row():
    rng = np.random.default_rng(2)
    Hq, Hkv, dh, page, n = 6, 2, 8, 4, 11
    pool_k, pool_v = rng.standard_normal((7, Hkv, page, dh)), rng.standard_normal((7, Hkv, page, dh))
    table = np.array([[5, 0, 3, 6], [1, 2, 4, 0]])
    q = rng.standard_normal((2, Hq, dh))
    pos = rng.permutation(40)[:32].reshape(2, 16)
    slopes = rng.random(Hq)
    got = A.paged_attention(q, pool_k, pool_v, table, [n, 0], 0.4, 3.0, slopes, pos)
    k, v = A.cache_rows(pool_k, table[0], n), A.cache_rows(pool_v, table[0], n)
    assert np.array_equal(k[1, 9], pool_k[3, 1, 1])
    want = A.prompt_attention(q[0][:, None], k, v, 0.4, softcap=3.0, slopes=slopes, positions=pos[0, :n])
    np.testing.assert_allclose(got["out"][0], want["out"][:, 0], atol=1e-13)
    np.testing.assert_allclose(got["lse"][0], want["lse"][:, 0], atol=1e-13)
    assert np.all(got["out"][1] == 0) and np.all(got["lse"][1] == -np.inf)
    np.testing.assert_allclose(got["p"][0].sum(1), 1.0, atol=1e-12)


def test_visible_rows():
    assert A.visible(2, 4).tolist() == [[True, True, True, False], [True] * 4]
    assert A.visible(3, 2).tolist() == [[False, False], [True, False], [True, True]]
    assert A.visible(2, 4, prefix=4).all() and A.visible(2, 4, causal=False).all()
    assert A.visible(3, 3, prefix=2).tolist() == [[True, True, False], [True, True, False], [True, True, True]]


def test_evicted_rows():
    mass = np.array([5.0, 1.0, 9.0, 0.0, 7.0, 2.0, 3.0, 0.0])
    pos = np.arange(8)
    # the newest row is safe; of the others 9, 7 and 5 stay: row 4 goes to 1's place, row 7 to 3's
    assert A.evict_rows(mass, pos, 8, 4, 0, 1).tolist() == [0, 4, 2, 7]
    assert A.evict_rows(mass, pos, 8, 4, 2, 1).tolist() == [0, 1, 2, 7]
    assert A.evict_rows(mass, pos, 4, 4, 0, 1).tolist() == [0, 1, 2, 3]
    assert A.evict_rows(mass, pos, 8, 2, 3, 8).tolist() == [0, 1]            # more protected than room: lower rows first
    ties = np.zeros(8)
    assert A.evict_rows(ties, pos, 8, 5, 0, 2).tolist() == [0, 1, 2, 6, 7]
    nan = np.array([0.0, np.nan, 1.0, np.inf, 2.0])
    assert A.evict_rows(nan, np.arange(5), 5, 2, 0, 1).tolist() == [4, 1]


def test_error_bounds_hold_for_fp32_arithmetic():
    rng = np.random.default_rng(3)
    q, k, v = (rng.standard_normal((2, n, 64)).astype(np.float32) for n in (40, 90, 90))
    want = A.prompt_attention(q, k, v, 0.125, softcap=4.0)
    for h in range(2):
        x = np.float32(4.0) * np.tanh(np.float32(0.125) * (q[h] @ k[h].T) / np.float32(4.0))
        seen = A.visible(40, 90)
        e = np.where(seen, np.exp(x - x.max()), np.float32(0))
        out = (e @ v[h]) / e.sum(1, keepdims=True)
        assert (np.abs(out - want["out"][h]) <= want["out_err"][h] + 2.0 ** -24 * np.abs(want["out"][h])).all()
        assert (np.abs(np.log(e.sum(1)) + x.max() - want["lse"][h]) <= want["lse_err"][h]).all()
    assert want["out_err"].max() < 1e-3
