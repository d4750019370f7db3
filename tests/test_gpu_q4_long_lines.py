"""Attention over a cache held in 4 bits where a piece of the line has many tiles of one unit (rings that wrap, softmaxes carried from tile to
tile, references taken anew), where both of a CTA's groups have work, and for batches around the numbers of sequences that warps hold.

The reference is the definition in 64 bits on the GPU (its own check: test_the_reference).  Bounds: a logit's as the oracle's (a chain of dh
steps of 2^-23 of the sum of the products' absolute values, and some of |x|, cap and bias); weights 2^-21 beside that; a sum over all rows is a chain of a lane's rows
of a piece (four a tile, fewer than 25 tiles), trees over lanes and warps, and a chain of pieces of a few steps: 150 steps of 2^-23; weights as two 11-bit numbers
2^-22, and 2^-37 of |v| for those below fp16's normal numbers; half a step of the output's type."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

from .test_gpu_q4 import HALF, num

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23


class Codes:
    """Pools of random codes and scales; `growth`: scales of K go up so many powers of two over a sequence's rows.  Places of no row hold ones in all bits, the table
    indices far out of range."""

    def __init__(self, lens, Hkv, dh, page, seed, growth=0, room=1):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.Hkv, self.dh, self.page = list(lens), Hkv, dh, page
        used = [(n + page - 1) // page for n in lens]
        self.max_pages, self.n_pages = max(used) + room, sum(used) + 2
        table = np.full((len(lens), self.max_pages), 2 ** 30, np.int32)
        order = np.random.default_rng(seed).permutation(self.n_pages)[:sum(used)]
        for b, u in enumerate(used):
            table[b, :u] = order[sum(used[:b]):sum(used[:b + 1])]
        self.block_table, self.S_cap = torch.from_numpy(table).cuda(), self.max_pages * page
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.k, self.v = (torch.full((self.n_pages, Hkv, page // 16, 9 * dh), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
        randint = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=self.g, device="cuda")
        for b, n in enumerate(lens):
            if not n:
                continue
            m, pages = used[b] * page, self.block_table[b, :used[b]].long()
            there = (torch.arange(m, device="cuda") < n)[None, :, None]
            for pool, up in ((self.k, growth), (self.v, 0)):
                codes = randint(1, 16, Hkv, m, dh // 2) | randint(1, 16, Hkv, m, dh // 2) << 4
                scales = randint(34, 37, Hkv, m, dh // 16) + (4 * up * torch.arange(m, device="cuda") // max(n, 1))[None, :, None]
                codes, scales = (torch.where(there, x, 255).to(torch.uint8).view(Hkv, used[b], page // 16, -1).transpose(0, 1) for x in (codes, scales))
                pool[pages] = torch.cat([codes, scales], -1)
        self.positions = torch.stack([torch.sort(randint(0, 4 * self.S_cap, self.S_cap)).values for _ in lens]).to(torch.int32)
        self.mass = torch.rand((len(lens), self.S_cap), generator=self.g, device="cuda")

    def rows(self, pool, b):
        """Values of sequence b's rows, [Hkv, n, dh] in 64 bits."""
        n, dh = self.lens[b], self.dh
        raw = pool[self.block_table[b, :(n + self.page - 1) // self.page].long()].transpose(0, 1)
        codes = raw[..., :8 * dh].reshape(self.Hkv, -1, dh // 2)[:, :n].long()
        e = torch.tensor(np.append(A.E5M2, np.full(256 - len(A.E5M2), np.nan)), device="cuda")[raw[..., 8 * dh:].reshape(self.Hkv, -1, dh // 16)[:, :n].long()]
        return (torch.stack([codes & 15, codes >> 4], -1).flatten(-2) - 8).double() * torch.repeat_interleave(16 * e, 16, -1)


def reference(c, q, scale, cap, slopes, pos, b):
    """out, lse, weights of sequence b, and how far fp32 arithmetic may be off: (values, bounds), a triple each."""
    Hq = q.shape[1]
    k, v = (c.rows(p, b).repeat_interleave(Hq // c.Hkv, 0) for p in (c.k, c.v))
    x = scale * torch.einsum("hd,hnd->hn", q[b].double(), k)
    err = scale * torch.einsum("hd,hnd->hn", q[b].double().abs(), k.abs()) * (c.dh * STEP)
    if cap:
        x = cap * torch.tanh(x / cap)
        err = err + 8 * STEP * cap
    err = err + 8 * STEP * x.abs()
    if slopes is not None:
        far = (pos[b, c.lens[b] - 1] - pos[b, :c.lens[b]]).abs().double()[None] * slopes.double()[:, None]
        x = x - far
        err = err + 8 * STEP * far + 2 * STEP * x.abs()
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[:, None])
    rel = torch.expm1(err) + 4 * STEP
    norm = (p * rel).sum(-1) + 150 * STEP
    out, absv = torch.einsum("hn,hnd->hd", p, v), torch.einsum("hn,hnd->hd", p, v.abs())
    out_err = torch.einsum("hn,hnd->hd", p * rel, v.abs()) + (norm + 150 * STEP)[:, None] * absv
    return (out, lse, p), (out_err, norm + 4 * STEP * torch.maximum(lse.abs(), x.abs().amax(-1)).clamp(min=1), p * (rel + norm[:, None])), absv, v.abs().max()


def check(c, Hq, dtype, bent, mass, size=1.0, bad=None):
    scale, cap = c.dh ** -0.5, 6.0 if bent else 0.0
    q = (torch.randn((len(c.lens), Hq, c.dh), generator=c.g, device="cuda") * size).to(dtype)
    slopes = torch.rand(Hq, generator=c.g, device="cuda") * 1e-4 if bent else None
    pos, m = c.positions if bent else None, c.mass.clone() if mass else None
    call = lambda table, m: B.metok_paged_attention_q4(q, c.k, c.v, table, c.kv_len, scale, softcap=cap, slopes=slopes, positions=pos, mass=m, with_lse=True)
    got = call(c.block_table, m)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    for b, n in enumerate(c.lens):
        if n == 0:
            assert not got["out"][b].any() and (got["lse"][b] == -np.inf).all()
        else:
            (out, lse, p), (out_err, lse_err, p_err), absv, most = reference(c, q, scale, cap, slopes, pos, b)
            tol = out_err + HALF[dtype] * out.abs() + 2.0 ** -22 * absv + 2.0 ** -37 * n * most
            assert bool(((got["out"][b].double() - out).abs() <= tol).all()), (b, float(((got["out"][b].double() - out).abs() / tol).max()))
            assert bool(((got["lse"][b].double() - lse).abs() <= lse_err + STEP * lse.abs()).all()), b
            if mass:
                inc, err, new = p.mean(0), p_err.mean(0), m[b, :n].double()
                assert bool(((new - c.mass[b, :n] - inc).abs() <= err + 2.0 ** -20 * inc + STEP * new.abs()).all()), b
        if mass:
            assert torch.equal(m[b, n:], c.mass[b, n:])
    # again, and with a bad page far behind the first rows of one sequence
    again = call(c.block_table, c.mass.clone() if mass else None)
    assert torch.equal(again["out"], got["out"]) and torch.equal(again["lse"], got["lse"])
    if bad is not None:
        table, m2 = c.block_table.clone(), c.mass.clone() if mass else None
        table[bad, (c.lens[bad] * 2 // 3) // c.page] = c.n_pages
        out = torch.full_like(q, 3.0)
        marked = B.metok_paged_attention_q4(q, c.k, c.v, table, c.kv_len, scale, softcap=cap, slopes=slopes, positions=pos, mass=m2, with_lse=True, out=out)
        torch.cuda.synchronize()
        others = [b for b in range(len(c.lens)) if b != bad]
        assert int(marked["status"]) == -1 and (out[bad] == 3).all()
        assert torch.equal(out[others], got["out"][others]) and torch.equal(marked["lse"][others], got["lse"][others])
        if mass:
            assert torch.equal(m2[bad], c.mass[bad]) and torch.equal(m2[others], m[others])


def test_the_reference():
    c = Codes([70, 0, 33], 2, 64, 16, seed=1, growth=2)
    q = torch.randn((3, 6, 64), generator=c.g, device="cuda")
    slopes = torch.rand(6, generator=c.g, device="cuda") * 0.01
    want = A.paged_attention(num(q), *(np.nan_to_num(A.q4_pool_values(p.cpu().numpy())) for p in (c.k, c.v)), c.block_table.cpu().numpy(), c.lens, 0.1, 5.0, num(slopes),
                             num(c.positions))
    for b in (0, 2):
        (out, lse, p), _, absv, _ = reference(c, q, 0.1, 5.0, slopes, c.positions, b)
        assert np.allclose(num(out), want["out"][b], rtol=1e-12, atol=1e-12) and np.allclose(num(lse), want["lse"][b], rtol=1e-12)
        assert np.allclose(num(p), want["p"][b], rtol=1e-11) and np.allclose(num(absv), want["absv"][b], rtol=1e-12)


# tiles of a unit in a piece (444 pieces, or 296 of units of more than eight heads): about eight
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh,page", [(16, 8, 128, 64), (16, 8, 64, 128), (8, 8, 128, 16), (36, 4, 128, 256), (64, 4, 64, 32), (60, 3, 128, 64)])
@pytest.mark.parametrize("bent", [False, True])
@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("growth", [0, 3])
def test_many_tiles_of_a_unit_in_a_piece(dtype, Hq, Hkv, dh, page, bent, mass, growth):
    c = Codes([20001, 17, 19000, 18944], Hkv, dh, page, seed=Hq, growth=growth)
    check(c, Hq, dtype, bent, mass, size=0.5 if growth else 1.0, bad=2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh", [(9, 1, 64), (20, 1, 128), (16, 1, 128)])
def test_one_unit_of_many_heads_over_a_long_sequence(dtype, Hq, Hkv, dh):
    """Pieces of one or of two tiles: the joins of a head's partials, and of a unit's."""
    for n in (30000, 60000, 300):
        check(Codes([n], Hkv, dh, 64, seed=n, growth=2), Hq, dtype, n == 60000, True, size=0.5)


@pytest.mark.parametrize("n_seqs", [32, 33, 64, 255, 256, 257])
@pytest.mark.parametrize("dtype,Hq,Hkv,dh", [(torch.bfloat16, 28, 4, 64), (torch.float32, 6, 3, 128), (torch.bfloat16, 24, 2, 128)])
def test_batches(n_seqs, dtype, Hq, Hkv, dh):
    """Sequences of mixed lengths, some of them empty, with more tiles than there are pieces; the last one empty, or the only long one."""
    lens = np.random.default_rng(n_seqs).integers(0, 90000 // n_seqs, n_seqs)
    lens[::7] = 0
    lens[5] = 2500
    for last in (0, 4001):
        lens[-1] = last
        check(Codes(lens.tolist(), Hkv, dh, 32, seed=n_seqs), Hq, dtype, last > 0, True, bad=5)
