"""Rows into and out of a cache held in 4 bits at each number of rows a CTA takes (1, 2, 4 .. 32: by how many there are), around the numbers of
sequences that a warp holds, and evictions of many layers and sequences.  Codes, scales and values are exact."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

from .test_gpu_q4 import elements, num

pytestmark = pytest.mark.gpu


def stand_for(pool, table, n, page):
    """Values of the first n rows of a sequence, [Hkv, n, dh], fp32 on the GPU."""
    dh, Hkv = pool.shape[-1] // 9, pool.shape[1]
    raw = pool[table[:(n + page - 1) // page].long()].transpose(0, 1)
    codes = raw[..., :8 * dh].reshape(Hkv, -1, dh // 2)[:, :n].int()
    e = torch.tensor(np.append(A.E5M2, np.full(256 - len(A.E5M2), np.nan)), device="cuda").float()[raw[..., 8 * dh:].reshape(Hkv, -1, dh // 16)[:, :n].long()]
    return (torch.stack([codes & 15, codes >> 4], -1).flatten(-2) - 8) * torch.repeat_interleave(16 * e, 16, -1)


def same(x, y):
    return torch.equal(torch.nan_to_num(x.float(), 1e30), torch.nan_to_num(y.float(), 1e30)) and torch.equal(x.isnan(), y.isnan())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("total", [601, 1300, 2600, 5003, 9800, 19007])
@pytest.mark.parametrize("Hkv,dh,n_seqs", [(1, 128, 5), (2, 64, 32), (3, 128, 33), (5, 64, 1), (9, 128, 2)])
def test_every_number_of_rows_of_a_cta(dtype, total, Hkv, dh, n_seqs):
    page = 32
    rng = np.random.default_rng(total)
    g = torch.Generator(device="cuda").manual_seed(total)
    cuts = np.sort(rng.integers(0, total + 1, n_seqs - 1))
    off = np.concatenate([[0], cuts, [total]]).astype(np.int32)
    old = rng.integers(0, 50, n_seqs)
    max_pages = int(max(old + off[1:] - off[:-1]) + page - 1) // page
    table = torch.randperm(n_seqs * max_pages, generator=g, device="cuda").to(torch.int32).view(n_seqs, max_pages)
    K, V = B.q4_pool(n_seqs * max_pages, Hkv, page, dh), B.q4_pool(n_seqs * max_pages, Hkv, page, dh)
    K.fill_(255), V.fill_(255)
    new = [elements((total, Hkv, dh), dtype, g).transpose(0, 1) for _ in range(2)]
    kv_len, offsets = torch.tensor(old, dtype=torch.int32, device="cuda"), torch.from_numpy(off).cuda()
    got = B.metok_paged_append_q4(*new, K, V, table, kv_len, offsets)
    back = [B.metok_paged_read_q4(K, V, table, got["new_len"], offsets, total, first_row=kv_len, dtype=t) for t in (torch.bfloat16, torch.float32)]
    torch.cuda.synchronize()
    assert int(got["status"]) == 0 and all(int(r["status"]) == 0 for r in back)
    for pool, x, name in ((K, new[0], "k"), (V, new[1], "v")):
        want = torch.from_numpy(A.q4_values(*A.q4_hold(num(x)))).float().cuda()
        assert all(same(r[name], want) for r in back)
        for b in range(n_seqs):
            n = int(old[b]) + int(off[b + 1] - off[b])
            rows = stand_for(pool, table[b], n, page)
            assert same(rows[:, int(old[b]):], want[:, off[b]:off[b + 1]]) and rows[:, :int(old[b])].isnan().all()
    written = (K[..., 8 * dh:] != 255).any(-1).sum()                 # rows of no sequence are as they were: at most two pieces of a run are not all new
    assert int(written) <= Hkv * (total // 16 + 2 * n_seqs)


@pytest.mark.parametrize("n_seqs,layers,budget", [(300, 3, 40), (70, 28, 100), (2, 40, 700)])
def test_evictions_of_many_layers_and_sequences(n_seqs, layers, budget):
    Hkv, dh, page = 2, 64, 16
    rng = np.random.default_rng(n_seqs)
    g = torch.Generator(device="cuda").manual_seed(n_seqs)
    lens = rng.integers(0, 3 * budget, n_seqs)
    lens[:2] = 3 * budget, budget
    max_pages = 3 * budget // page + 1
    n_pages = n_seqs * max_pages
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).view(n_seqs, max_pages)
    pools = [[torch.randint(0, 256, (n_pages, Hkv, page // 16, 9 * dh), generator=g, device="cuda", dtype=torch.uint8) for _ in range(layers)] for _ in range(2)]
    S_cap = max_pages * page
    mass = torch.rand((layers, n_seqs, S_cap), generator=g, device="cuda")
    pos = torch.arange(S_cap, dtype=torch.int32, device="cuda").repeat(layers, n_seqs, 1)
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def raw(pool, b, rows):
        """Codes and scales of rows of a sequence: [Hkv, rows, 9 dh / 16]."""
        x = pool[table[b].long()].transpose(0, 1)
        x = torch.cat([x[..., :8 * dh].reshape(Hkv, S_cap, dh // 2), x[..., 8 * dh:].reshape(Hkv, S_cap, dh // 16)], -1)
        return x[:, rows]

    some = [(l, b) for l in {0, layers // 2, layers - 1} for b in {0, 1, 2 % n_seqs, n_seqs // 2, n_seqs - 1}]
    want = {}
    for l, b in some:
        rows = A.evict_rows(num(mass[l, b]), pos[l, b].cpu().numpy(), int(lens[b]), budget, 3, 8)
        want[l, b] = rows, [raw(p[l], b, torch.from_numpy(rows).cuda()) for p in pools]
    got = B.metok_paged_evict(*pools, table, kv_len, mass, pos, budget, 3, 8)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0 and got["new_len"].tolist() == np.minimum(lens, budget).tolist()
    for (l, b), (rows, held) in want.items():
        n = len(rows)
        assert got["keep_idx"][l, b].tolist() == rows.tolist() + [-1] * (budget - n)
        assert all(torch.equal(raw(p[l], b, torch.arange(n, device="cuda")), x) for p, x in zip(pools, held))
