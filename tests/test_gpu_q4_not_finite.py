"""Attention over a cache held in 4 bits: infinite logits, with a cap, a bias and weights, and what is no number beside them."""

import math

import numpy as np
import pytest
import torch

from paper_2506_02850_b200 import binding as B

from .test_gpu_q4 import HALF, Cache, num

pytestmark = pytest.mark.gpu

CAP = 2.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,dh", [(4, 64), (7, 128), (12, 128)])
@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("bent", ["", "cap", "bias", "cap bias"])
def test_infinite_elements_of_q(dtype, Hq, dh, mass, bent):
    """K's rows are 1 or -1 in the place of Q's infinity: logits of both signs, of one, or (under a cap) the cap's."""
    lens, page = [150, 33, 200], 16
    n, n_seqs = sum(lens), len(lens)
    g = torch.Generator(device="cuda").manual_seed(Hq)
    used = [(m + page - 1) // page for m in lens]
    n_pages, S_cap = sum(used), max(used) * page
    table = torch.full((n_seqs, max(used)), 2 ** 30, dtype=torch.int32, device="cuda")
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    for b, u in enumerate(used):
        table[b, :u] = order[sum(used[:b]):sum(used[:b + 1])]
    K, V = B.q4_pool(n_pages, 1, page, dh), B.q4_pool(n_pages, 1, page, dh)
    off = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    k, v = (torch.randn((1, n, dh), generator=g, device="cuda") for _ in range(2))
    k[0, :, 5] = 1.0
    k[0, lens[0]:lens[0] + 11, 5] = -1.0                             # sequence 1: eleven rows of 33
    length = B.metok_paged_append_q4(k, v, K, V, table, torch.zeros(n_seqs, dtype=torch.int32, device="cuda"), off)["new_len"]
    q = torch.randn((n_seqs, Hq, dh), generator=g, device="cuda").to(dtype)
    slopes = torch.zeros(Hq, device="cuda") if "bias" in bent else None
    cap = CAP if "cap" in bent else 0.0
    call = lambda q, m: B.metok_paged_attention_q4(q, K, V, table, length, 0.125, softcap=cap, slopes=slopes, mass=m, with_lse=True)
    m0, m1 = (torch.zeros((n_seqs, S_cap), device="cuda") if mass else None for _ in range(2))
    clean = call(q, m0)
    Q = q.clone()
    Q[0, 1, 5], Q[1, 2, 5], Q[2, 0, 5] = -math.inf, math.inf, math.inf
    got = call(Q, m1)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    out, lse, was = num(got["out"]), num(got["lse"]), num(clean["out"])
    values = num(B.metok_paged_read_q4(K, V, table, length, off, n, dtype=torch.float32)["v"])[0]
    close = lambda x, y: (np.abs(x - y) <= 2 * HALF[dtype] * np.abs(y) + 2.0 ** -18 * np.abs(values).max()).all()
    # the other heads: as they were, up to the arithmetic's roundings
    for b, h in ((0, 1), (1, 2), (2, 0)):
        rest = [i for i in range(Hq) if i != h]
        assert close(out[b, rest], was[b, rest]) and np.allclose(lse[b, rest], num(clean["lse"])[b, rest], rtol=1e-5, atol=1e-5)
    if cap:                                                          # logits of CAP or -CAP: weights of rows of two kinds
        for (b, h), x in {(0, 1): np.full(150, -CAP), (1, 2): np.where(np.arange(33) < 11, -CAP, CAP), (2, 0): np.full(200, CAP)}.items():
            p = np.exp(x) / np.exp(x).sum()
            assert close(out[b, h], p @ values[sum(lens[:b]):sum(lens[:b + 1])]) and np.isclose(lse[b, h], np.log(np.exp(x).sum()), rtol=1e-5)
            if mass:
                assert torch.isfinite(m1[b]).all() and not m1[b, lens[b]:].any()
    else:
        assert (out[0, 1] == 0).all() and lse[0, 1] == -math.inf     # every logit -infinity: no weight
        for b, h in ((1, 2), (2, 0)):
            assert np.isnan(out[b, h]).all() and np.isnan(lse[b, h])
        if mass:
            assert np.allclose(num(m1)[0, :150].sum(), (Hq - 1) / Hq, rtol=1e-4)
            for b in (1, 2):
                assert torch.isnan(m1[b, :lens[b]]).all() and not m1[b, lens[b]:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh", [(4, 2, 64), (14, 2, 128), (24, 2, 64)])
@pytest.mark.parametrize("bent,size", [("", 1.0), ("cap", 0.2), ("cap", 20.0), ("bias", 1.0), ("cap bias", 20.0)])
def test_what_is_no_number_under_caps_and_biases(dtype, Hq, Hkv, dh, bent, size):
    """Logits below the cap and far above it; in a first tile and in later ones."""
    lens = [300, 140, 290]
    c = Cache(lens, Hkv, dh, 32, seed=6)
    G = Hq // Hkv
    q = (torch.randn((3, Hq, dh), generator=c.g, device="cuda") * size).to(dtype)
    slopes = torch.rand(Hq, generator=c.g, device="cuda") * 0.01 if "bias" in bent else None
    pos = c.positions[0].contiguous() if "bias" in bent else None
    call = lambda q, K, V, m: B.metok_paged_attention_q4(q, K, V, c.block_table, c.kv_len, 0.125, softcap=CAP if "cap" in bent else 0.0, slopes=slopes,
                                                         positions=pos, mass=m, with_lse=True)
    m0, m1 = c.mass[0].clone(), c.mass[0].clone()
    clean = call(q, c.k[0], c.v[0], m0)
    K, V, Q = c.k[0].clone(), c.v[0].clone(), q.clone()
    place = lambda r: (r // 32, r % 32 // 16, r % 16)                # page of the sequence, piece, row of it
    for pool, b, head, r, block in ((K, 0, 1, 267, 3), (V, 1, 0, 133, 2)):
        page, piece, row = place(r)
        pool[int(c.table_np[b, page]), head, piece, 8 * dh + row * (dh // 16) + block] = 0x7F
    Q[2, Hq - 1, 7] = float("nan")
    got = call(Q, K, V, m1)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    out, lse, was = num(got["out"]), num(got["lse"]), num(clean["out"])
    most = 5.0                                                       # |V| of normal numbers
    close = lambda x, y: (np.abs(x - y) <= 2 * HALF[dtype] * np.abs(y) + 2.0 ** -16 * most).all()
    assert np.isnan(out[0, G:]).all() and np.isnan(lse[0, G:]).all() and close(out[0, :G], was[0, :G])
    assert np.isnan(out[1, :G, 32:48]).all() and close(out[1, :G, :32], was[1, :G, :32]) and close(out[1, :G, 48:], was[1, :G, 48:])
    assert close(out[1, G:], was[1, G:]) and np.allclose(lse[1], num(clean["lse"])[1], rtol=1e-5, atol=1e-5)
    assert np.isnan(out[2, -1]).all() and np.isnan(lse[2, -1]) and close(out[2, :-1], was[2, :-1])
    for b in (0, 2):
        assert torch.isnan(m1[b, :lens[b]]).all() and torch.equal(m1[b, lens[b]:], c.mass[0, b, lens[b]:])
    assert torch.allclose(m1[1], m0[1], rtol=1e-5, atol=1e-6)
