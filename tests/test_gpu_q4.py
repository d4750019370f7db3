"""A paged cache held in 4 bits: append and read back, attention of one token, eviction, against oracle/attention_oracle.py.

Codes, scales and values are exact.  Tolerances of the attention: the oracle's bounds on fp32 arithmetic; half a step of the output's type
(2^-8 of a bf16 value, 2^-24 of an fp32 one); weights as one (two) 11-bit numbers, the largest at 2^12 at least: 2^-12 (2^-23) of the sum of
weight * |v|, and 2^-25 / 2^12 = 2^-37 of |v| for each weight that is below fp16's normal numbers."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
WEIGHT = {torch.bfloat16: 2.0 ** -12, torch.float32: 2.0 ** -23}


def num(t):
    return t.detach().cpu().double().numpy()


class Cache:
    """A cache whose unused places hold ones in all bits (a scale of NaN), and whose table behind the sequences' pages holds indices far out of
    range."""

    def __init__(self, lens, Hkv, dh, page, seed, room=1, layers=1, spare=2, size=1.0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        n_seqs = len(lens)
        self.max_pages = max((n + room + page - 1) // page for n in lens) + 1
        used = [(n + room + page - 1) // page for n in lens]
        self.n_pages = sum(used) + spare
        order = rng.permutation(self.n_pages)[:sum(used)]
        self.table_np = np.full((n_seqs, self.max_pages), 2 ** 30, np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table_np[b, :u] = order[at:at + u]
            at += u
        self.block_table = torch.from_numpy(self.table_np).cuda()
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.lens, self.page, self.Hkv, self.dh, self.S_cap = list(lens), page, Hkv, dh, self.max_pages * page
        pools = []
        for _ in range(2):
            pool = np.full((layers, self.n_pages, Hkv, page // 16, 9 * dh), 255, np.uint8)
            codes, scales = A.q4_parts(pool.reshape(-1, Hkv, page // 16, 9 * dh))
            codes, scales = (np.ascontiguousarray(x).reshape(layers, self.n_pages, Hkv, page, -1) for x in (codes, scales))
            for b, n in enumerate(lens):
                c, e = A.q4_hold(rng.standard_normal((layers, Hkv, n, dh)) * size)
                for p in range(0, n, page):
                    m = min(page, n - p)
                    codes[:, self.table_np[b, p // page], :, :m], scales[:, self.table_np[b, p // page], :, :m] = c[:, :, p:p + m], e[:, :, p:p + m]
            pool[..., :8 * dh] = codes.reshape(*pool.shape[:-1], 8 * dh)
            pool[..., 8 * dh:] = scales.reshape(*pool.shape[:-1], dh)
            pools.append(torch.from_numpy(pool).cuda())
        self.k, self.v = pools
        pos = [[np.sort(rng.choice(4 * self.S_cap, self.S_cap, replace=False)) for _ in range(n_seqs)] for _ in range(layers)]
        self.positions = torch.from_numpy(np.array(pos).astype(np.int32)).cuda()
        self.mass = torch.rand((layers, n_seqs, self.S_cap), generator=self.g, device="cuda")

    def rows(self, pool, b, n):
        """Values of the first n rows of sequence b, [Hkv, n, dh]."""
        return A.cache_rows(A.q4_pool_values(pool.cpu().numpy()), self.table_np[b], n)


# ---- append and read ---------------------------------------------------------------------------------------------------


def elements(shape, dtype, g):
    """Blocks of many sizes, with elements on the borders between two codes and two scales, zeros and what is no number."""
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp2(torch.randint(-17, 13, shape[:2] + (1,), generator=g, device="cuda").float())
    flat = x.view(-1, 16)
    n = flat.shape[0]
    flat[1::7, 0] = 7.5 * 16 * 2.0 ** torch.randint(-10, 2, (len(flat[1::7]),), generator=g, device="cuda")     # the largest that a scale takes
    flat[2::7] = torch.randint(-15, 16, flat[2::7].shape, generator=g, device="cuda") * 0.5                       # halves of a step
    flat[2::7, 3] = 7.5
    flat[3::11] = 0
    if n > 40:
        flat[5, 3], flat[16, 15], flat[27, 0], flat[38, 2] = float("nan"), float("inf"), -float("inf"), 2e4
    return x.to(dtype)


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32 if t.dtype == torch.float32 else t.dtype)


def expected(c, layer, kn, vn, off, lens):
    """The pools after an append, from the oracle."""
    res = []
    for pool, new in ((c.k, kn), (c.v, vn)):
        pool = pool[layer].cpu().numpy().copy()
        codes, scales = A.q4_parts(pool)
        codes, scales = codes.copy(), scales.copy()
        cc, ee = A.q4_hold(num(new))
        for b, n in enumerate(lens):
            for i in range(off[b], off[b + 1]):
                r = n + i - off[b]
                pg, at = c.table_np[b, r // c.page], r % c.page
                codes[pg, :, at // 16, at % 16], scales[pg, :, at // 16, at % 16] = cc[:, i], ee[:, i]
        pool[..., :8 * c.dh], pool[..., 8 * c.dh:] = codes.reshape(*pool.shape[:-1], -1), scales.reshape(*pool.shape[:-1], -1)
        res.append(torch.from_numpy(pool).cuda())
    return res


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hkv,dh,page", [(1, 64, 16), (4, 128, 64), (40, 128, 16), (3, 64, 256)])
@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [0, 37, 5, 0], [16, 0, 1, 130], [0, 0, 0, 0]])
def test_append_and_read(dtype, Hkv, dh, page, counts):
    lens = [0, 15, 33, 64]
    c = Cache(lens, Hkv, dh, page, seed=1, room=max(counts) + 1)
    n = sum(counts)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    off_t = torch.from_numpy(off).cuda()
    kn = elements((n, Hkv, dh), dtype, c.g).transpose(0, 1)
    base = torch.randn((n, Hkv + 1, dh + 16), generator=c.g, device="cuda").to(dtype)
    vn = base[:, :Hkv, :dh].transpose(0, 1)                          # rows and heads further apart than dense
    k, v = expected(c, 0, kn, vn, off, lens)
    K, V, P, M = c.k[0].clone(), c.v[0].clone(), c.positions[0].clone(), c.mass[0].clone()
    pos_new = torch.randint(0, 1 << 20, (n,), generator=c.g, device="cuda", dtype=torch.int32)
    mass_new = torch.rand(n, generator=c.g, device="cuda")
    got = B.metok_paged_append_q4(kn, vn, K, V, c.block_table, c.kv_len, None if counts == [1] * 4 else off_t, P, pos_new, M, mass_new)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    assert got["new_len"].tolist() == [a + b for a, b in zip(lens, counts)]
    assert torch.equal(K, k) and torch.equal(V, v)
    for b, (o, m) in enumerate(zip(lens, counts)):
        assert torch.equal(P[b, o:o + m], pos_new[off[b]:off[b + 1]]) and torch.equal(M[b, o:o + m], mass_new[off[b]:off[b + 1]])
    # the new rows back, in both types
    for out in (torch.bfloat16, torch.float32):
        back = B.metok_paged_read_q4(K, V, c.block_table, got["new_len"], off_t, n, first_row=c.kv_len, positions=P, dtype=out)
        torch.cuda.synchronize()
        assert int(back["status"]) == 0 and torch.equal(back["positions"], pos_new)
        for name, new in (("k", kn), ("v", vn)):
            want = A.q4_values(*A.q4_hold(num(new)))
            assert back[name].dtype == out and np.array_equal(num(back[name]), want, equal_nan=True)


@pytest.mark.parametrize("dh", [64, 128])
def test_read_whole_sequences_into_rows_with_room(dh):
    lens = [70, 0, 33, 200, 1]
    c = Cache(lens, 3, dh, 32, seed=2)
    off = np.concatenate([[2], 2 + np.cumsum(lens)]).astype(np.int32)     # two rows before the first sequence's, three behind the last one's
    n = int(off[-1]) + 3
    whole = torch.full((n, 7, dh + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    k_out, v_out = whole[:, :3, :dh].transpose(0, 1), whole[:, 4:, :dh].transpose(0, 1)
    got = B.metok_paged_read_q4(c.k[0], c.v[0], c.block_table, c.kv_len, torch.from_numpy(off).cuda(), n, k_out=k_out, v_out=v_out)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0 and "positions" not in got
    for b, m in enumerate(lens):
        assert np.array_equal(num(k_out[:, off[b]:off[b + 1]]), c.rows(c.k[0], b, m)) and np.array_equal(num(v_out[:, off[b]:off[b + 1]]), c.rows(c.v[0], b, m))
    assert (whole[:2] == 5).all() and (whole[-3:] == 5).all() and (whole[:, 3] == 5).all() and (whole[..., dh:] == 5).all()


def test_many_sequences():
    rng = np.random.default_rng(3)
    lens, counts = rng.integers(0, 50, 150).tolist(), rng.integers(0, 40, 150).tolist()
    c = Cache(lens, 2, 64, 16, seed=3, room=41)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n = int(off[-1])
    kn, vn = (elements((n, 2, 64), torch.bfloat16, c.g).transpose(0, 1) for _ in range(2))
    k, v = expected(c, 0, kn, vn, off, lens)
    got = B.metok_paged_append_q4(kn, vn, c.k[0], c.v[0], c.block_table, c.kv_len, torch.from_numpy(off).cuda())
    back = B.metok_paged_read_q4(c.k[0], c.v[0], c.block_table, got["new_len"], torch.from_numpy(off).cuda(), n, first_row=c.kv_len)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0 and int(back["status"]) == 0 and torch.equal(c.k[0], k) and torch.equal(c.v[0], v)
    assert np.array_equal(num(back["v"]), A.q4_values(*A.q4_hold(num(vn))), equal_nan=True)


def test_unsound_sequences_are_reported():
    c = Cache([20, 30, 40, 10, 50], 2, 64, 16, seed=4, room=16)
    off = torch.tensor([0, 4, 8, 12, 16, 20], dtype=torch.int32, device="cuda")
    kn, vn = (torch.randn((2, 20, 64), generator=c.g, device="cuda") for _ in range(2))
    want = expected(c, 0, kn, vn, off.tolist(), c.lens)
    table, lens = c.block_table.clone(), c.kv_len.clone()
    table[0, 1] = -3                                                 # its rows 20 .. 23
    lens[2] = c.S_cap - 3                                            # no room for four
    lens[3] = -1
    K, V = c.k[0].clone(), c.v[0].clone()
    got = B.metok_paged_append_q4(kn, vn, K, V, table, lens, off)
    assert int(got["status"]) == -1 and got["new_len"].tolist() == [20, 34, c.S_cap - 3, -1, 54]
    for b in (1, 4):
        pages = [int(p) for p in c.table_np[b] if p < c.n_pages]
        assert torch.equal(K[pages], want[0][pages]) and torch.equal(V[pages], want[1][pages])
    # reading: rows that are not there, a bad page, a bad length; the others are served
    first = torch.tensor([18, 28, 39, 0, 46], dtype=torch.int32, device="cuda")
    lens = torch.tensor([20, 30, 40, 10, 50], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 2, 4, 6, 8, 10], dtype=torch.int32, device="cuda")
    table = c.block_table.clone()
    table[3, 0] = c.n_pages
    got = B.metok_paged_read_q4(c.k[0], c.v[0], table, lens, off, 10, first_row=first, dtype=torch.float32)
    assert int(got["status"]) == -1                                  # sequence 2 has one row from 39 on, sequence 3 a bad page
    for b, f in ((0, 18), (1, 28), (4, 46)):
        assert np.array_equal(num(got["k"][:, 2 * b:2 * b + 2]), c.rows(c.k[0], b, f + 2)[:, f:])
    for bad in ([0, 4, 2, 6, 8, 10], [0, 2, 4, 6, 8, 11], [-1, 2, 4, 6, 8, 10]):
        got = B.metok_paged_read_q4(c.k[0], c.v[0], c.block_table, lens, torch.tensor(bad, dtype=torch.int32, device="cuda"), 10)
        assert int(got["status"]) == -1
    out = torch.full((2, 10, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    B.metok_paged_read_q4(c.k[0], c.v[0], c.block_table, lens, torch.tensor([0, 4, 2, 6, 8, 10], dtype=torch.int32, device="cuda"), 10, k_out=out)
    torch.cuda.synchronize()
    assert (out == 3).all()
    for bad in (torch.tensor([-1] * 5, dtype=torch.int32), torch.tensor([2 ** 31 - 1] * 5, dtype=torch.int32)):
        assert int(B.metok_paged_read_q4(c.k[0], c.v[0], c.block_table, lens, off, 10, first_row=bad.cuda())["status"]) == -1


# ---- attention ---------------------------------------------------------------------------------------------------------


def check_attention(c, Hq, dtype, cap=0.0, bias=False, mass=True, q=None, scale=None, layer=0):
    scale = c.dh ** -0.5 if scale is None else scale
    if q is None:
        q = (torch.randn((len(c.lens), Hq, c.dh), generator=c.g, device="cuda") * (5 if cap else 1.5)).to(dtype)
    slopes = torch.rand(Hq, generator=c.g, device="cuda") * 0.2 if bias else None
    pos = c.positions[layer].contiguous() if bias else None
    m = c.mass[layer].clone() if mass else None
    got = B.metok_paged_attention_q4(q, c.k[layer], c.v[layer], c.block_table, c.kv_len, scale, softcap=cap, slopes=slopes, positions=pos, mass=m, with_lse=True)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    vk, vv = (A.q4_pool_values(p[layer].cpu().numpy()) for p in (c.k, c.v))
    want = A.paged_attention(num(q), vk, vv, c.table_np, c.lens, scale, cap, None if slopes is None else num(slopes), None if pos is None else num(pos))
    most = np.nanmax(np.abs(vv), initial=0.0)
    tol = want["out_err"] + HALF[dtype] * np.abs(want["out"]) + WEIGHT[dtype] * want["absv"] + 2.0 ** -37 * most * np.array(c.lens)[:, None, None]
    out = num(got["out"])
    assert np.isfinite(out).all()
    worst = float(np.max(np.abs(out - want["out"]) / np.maximum(tol, 1e-30)))
    assert worst <= 1, worst
    lse = num(got["lse"])
    for b, n in enumerate(c.lens):
        if n == 0:
            assert np.all(lse[b] == -np.inf) and np.all(out[b] == 0)
        else:
            assert (np.abs(lse[b] - want["lse"][b]) <= want["lse_err"][b] + 2.0 ** -23 * np.abs(want["lse"][b])).all()
    if mass:
        new, old = num(m), num(c.mass[layer])
        for b, n in enumerate(c.lens):
            inc, err = want["p"][b].mean(0), want["p_err"][b].mean(0)
            assert (np.abs(new[b, :n] - old[b, :n] - inc) <= err + 2.0 ** -20 * inc + 2.0 ** -23 * np.abs(new[b, :n])).all()
            assert np.array_equal(new[b, n:], old[b, n:])
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh", [(1, 1, 64), (14, 2, 64), (28, 4, 128), (5, 5, 128), (6, 3, 64), (12, 3, 128), (16, 1, 64), (40, 2, 64), (33, 1, 128)])
def test_attention_heads_and_lengths(dtype, Hq, Hkv, dh):
    c = Cache([1, 0, 63, 64, 65, 200, 17, 31, 33], Hkv, dh, 16, seed=Hq)
    check_attention(c, Hq, dtype)
    check_attention(c, Hq, dtype, cap=4.0, bias=True, mass=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attention_page_sizes_cap_bias(dtype, page):
    c = Cache([3 * page + 5, 2 * page, 1, page - 1, page + 1], 2, 64, page, seed=page)
    check_attention(c, 14, dtype, cap=8.0, bias=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_one_long_sequence_is_split(dtype):
    check_attention(Cache([2500], 2, 128, 64, seed=9), 14, dtype)
    check_attention(Cache([2500, 3, 0, 700], 1, 64, 32, seed=10), 7, dtype, bias=True)


def test_attention_many_sequences():
    lens = np.random.default_rng(4).integers(0, 40, 333).tolist()
    check_attention(Cache(lens, 1, 64, 16, seed=11), 3, torch.bfloat16, cap=3.0)
    check_attention(Cache([0] * 7, 1, 64, 16, seed=12), 3, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [1e-3, 900.0])
def test_attention_of_small_and_large_numbers(dtype, size):
    c = Cache([90, 130], 2, 64, 16, seed=5, size=size)
    for scale_q in (1e-30, 1.0, 1e25):
        q = (torch.randn((2, 4, 64), generator=c.g, device="cuda") * scale_q).to(dtype)
        q[0, 0, ::2] *= 2.0 ** -12                                     # a head's elements differ in size
        check_attention(c, 4, dtype, q=q, scale=0.2 / size / scale_q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cap", [1e6, 1e20, 1e30, 1e38])
def test_attention_under_a_cap_that_is_far_away(dtype, cap):
    """A cap that no logit comes near changes next to nothing: cap tanh(x / cap) is x up to fp32's roundings.  At 1e38 the scale over the cap is 1e-39,
    where numbers are 2^-149 apart: it is off by 7e-7 of itself, and logits (below 16 here) by 1.1e-5."""
    c = Cache([300, 65], 2, 128, 32, seed=31)
    q = torch.randn((2, 8, 128), generator=c.g, device="cuda").to(dtype)
    call = lambda x: B.metok_paged_attention_q4(q, c.k[0], c.v[0], c.block_table, c.kv_len, 0.1, softcap=x, with_lse=True)
    plain, capped = call(0.0), call(cap)
    torch.cuda.synchronize()
    assert torch.allclose(capped["lse"], plain["lse"], rtol=0, atol=2e-5)
    assert torch.allclose(capped["out"].float(), plain["out"].float(), rtol=2 * HALF[dtype], atol=1e-4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_equal_weights_and_large_logits(dtype):
    c = Cache([90, 130], 2, 64, 16, seed=5)
    check_attention(c, 4, dtype, q=torch.zeros((2, 4, 64), dtype=dtype, device="cuda"))
    big = (torch.randn((2, 4, 64), generator=c.g, device="cuda") * 60).to(dtype)
    check_attention(c, 4, dtype, q=big, scale=1.0)


def test_attention_what_is_no_number():
    for dtype in (torch.bfloat16, torch.float32):
        c = Cache([70, 40, 90], 2, 64, 16, seed=6)
        q = torch.randn((3, 4, 64), generator=c.g, device="cuda").to(dtype)
        clean = B.metok_paged_attention_q4(q, c.k[0], c.v[0], c.block_table, c.kv_len, 0.125, with_lse=True)
        K, V, Q = c.k[0].clone(), c.v[0].clone(), q.clone()
        K[int(c.table_np[0, 2]), 1, 0, 8 * 64 + 4 * 3] = 0x7F             # a block of row 35 of sequence 0, head 1
        V[int(c.table_np[1, 0]), 0, 0, 8 * 64 + 4 * 5 + 2] = 0x7F         # elements 32 .. 47 of row 5 of sequence 1, head 0
        Q[2, 3, 7] = float("nan")
        got = B.metok_paged_attention_q4(Q, K, V, c.block_table, c.kv_len, 0.125, with_lse=True)
        torch.cuda.synchronize()
        out, lse, want = got["out"].float(), got["lse"], clean["out"].float()
        assert torch.isnan(out[0, 2:]).all() and torch.isnan(lse[0, 2:]).all() and torch.equal(out[0, :2], want[0, :2])
        assert torch.isnan(out[1, :2, 32:48]).all() and torch.equal(out[1, :2, :32], want[1, :2, :32]) and torch.equal(out[1, :2, 48:], want[1, :2, 48:])
        assert torch.equal(out[1, 2:], want[1, 2:]) and torch.equal(lse[1], clean["lse"][1])
        assert torch.isnan(out[2, 3]).all() and torch.equal(out[2, :3], want[2, :3])


def test_attention_strides_outputs_and_repeats():
    c = Cache([77, 200, 5], 2, 64, 32, seed=6)
    q = torch.randn((4, 3, 128), generator=c.g, device="cuda").to(torch.bfloat16)
    view = q[:, :, 32:96].transpose(0, 1)                           # [3, 4, 64], heads further apart than sequences
    whole = torch.full((3, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[:, :, 64:]
    first = check_attention(c, 4, torch.bfloat16, q=view.contiguous())
    for _ in range(20):
        got = B.metok_paged_attention_q4(view, c.k[0], c.v[0], c.block_table, c.kv_len, c.dh ** -0.5, out=out, with_lse=True)
        torch.cuda.synchronize()
        assert got["out"].data_ptr() == out.data_ptr()
        assert torch.equal(out, first["out"]) and torch.equal(got["lse"], first["lse"])
        assert (whole[:, :, :64] == 7).all()


def test_attention_bad_pages_and_lengths_leave_the_sequence_alone():
    c = Cache([70, 40, 90, 20], 2, 64, 16, seed=7)
    q = torch.randn((4, 4, 64), generator=c.g, device="cuda").to(torch.bfloat16)
    good = B.metok_paged_attention_q4(q, c.k[0], c.v[0], c.block_table, c.kv_len, 0.125, mass=c.mass[0].clone())
    table, lens = c.block_table.clone(), c.kv_len.clone()
    table[0, 2] = c.n_pages
    table[2, 5] = -1
    lens[3] = c.S_cap + 1
    mass = c.mass[0].clone()
    out = torch.full((4, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    got = B.metok_paged_attention_q4(q, c.k[0], c.v[0], table, lens, 0.125, mass=mass, out=out, with_lse=True)
    torch.cuda.synchronize()
    assert int(got["status"]) == -1
    for b in (0, 2, 3):
        assert (out[b] == 3.0).all() and torch.equal(mass[b], c.mass[0, b])
    assert torch.allclose(out[1].float(), good["out"][1].float(), rtol=0.02, atol=0.02)


@pytest.mark.parametrize("mass", [False, True])
def test_attention_a_bad_page_among_many_sequences(mass):
    lens = np.random.default_rng(5).integers(1, 90, 300).tolist()
    lens[7] = 80
    c = Cache(lens, 2, 64, 16, seed=13)
    q = torch.randn((300, 6, 64), generator=c.g, device="cuda").to(torch.bfloat16)
    call = lambda table, m, out: B.metok_paged_attention_q4(q, c.k[0], c.v[0], table, c.kv_len, 0.125, mass=m, out=out, with_lse=True)
    m0, m1 = (c.mass[0].clone() if mass else None for _ in range(2))
    good, out = torch.empty_like(q), torch.full_like(q, 3.0)
    want = call(c.block_table, m0, good)
    table = c.block_table.clone()
    table[7, 4] = -5
    got = call(table, m1, out)
    torch.cuda.synchronize()
    assert int(want["status"]) == 0 and int(got["status"]) == -1
    others = [b for b in range(300) if b != 7]
    assert (out[7] == 3).all() and torch.equal(out[others], good[others]) and torch.equal(got["lse"][others], want["lse"][others])
    if mass:
        assert torch.equal(m1[7], c.mass[0, 7]) and torch.equal(m1[others], m0[others])


def test_attention_captured_with_lengths_that_change():
    c = Cache([100, 37], 2, 128, 16, seed=8, room=40)
    q = torch.randn((2, 8, 128), generator=c.g, device="cuda").to(torch.bfloat16)
    new = [(torch.randn((2, 2, 128), generator=c.g, device="cuda") * 2).to(torch.bfloat16) for _ in range(2)]
    length = c.kv_len.clone()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            new_len = B.metok_paged_append_q4(new[0], new[1], c.k[0], c.v[0], c.block_table, length)["new_len"]
            got = B.metok_paged_attention_q4(q, c.k[0], c.v[0], c.block_table, new_len, 0.1, with_lse=True)
            length.copy_(new_len)
    for _ in range(20):
        graph.replay()
    torch.cuda.synchronize()
    assert length.tolist() == [120, 57]
    c.kv_len, c.lens = length, [120, 57]
    want = check_attention(c, 8, torch.bfloat16, q=q, scale=0.1, mass=False)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    assert np.array_equal(c.rows(c.v[0], 1, 57)[:, 37:], np.repeat(A.q4_values(*A.q4_hold(num(new[1])))[:, 1:], 20, axis=1))


# ---- eviction ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("Hkv,dh,page", [(1, 64, 16), (4, 128, 64), (5, 128, 16), (9, 64, 32)])
@pytest.mark.parametrize("budget", [1, 40, 128])
def test_evict(Hkv, dh, page, budget):
    lens = [200, 40, 0, 129, 333]
    c = Cache(lens, Hkv, dh, page, seed=budget, layers=3)
    before = [[(c.rows(c.k[l], b, n), c.rows(c.v[l], b, n)) for b, n in enumerate(lens)] for l in range(3)]
    pos, mass = c.positions.clone(), c.mass.clone()
    untouched = [c.k.clone(), c.v.clone()]
    got = B.metok_paged_evict(list(c.k), list(c.v), c.block_table, c.kv_len, mass, pos, budget, 2, 5)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0 and got["new_len"].tolist() == [min(n, budget) for n in lens]
    for l in range(3):
        for b, n in enumerate(lens):
            rows = A.evict_rows(num(c.mass[l, b]), c.positions[l, b].cpu().numpy(), n, budget, 2, 5)
            assert got["keep_idx"][l, b].tolist() == rows.tolist() + [-1] * (budget - len(rows))
            assert np.array_equal(c.rows(c.k[l], b, len(rows)), before[l][b][0][:, rows]) and np.array_equal(c.rows(c.v[l], b, len(rows)), before[l][b][1][:, rows])
    # what no row of the new length has is as it was
    for pool, old in zip((c.k, c.v), untouched):
        mine = A.q4_parts(pool.cpu().numpy())
        was = A.q4_parts(old.cpu().numpy())
        for x, y in zip(mine, was):
            x, y = x.reshape(3, c.n_pages, Hkv, page, -1).copy(), y.reshape(3, c.n_pages, Hkv, page, -1).copy()
            for b, n in enumerate(lens):
                for r in range(min(n, budget)):
                    x[:, c.table_np[b, r // page], :, r % page] = y[:, c.table_np[b, r // page], :, r % page] = 0
            assert np.array_equal(x, y)


# ---- a run of the calls, as an answer uses them ------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_from_projections_to_an_answer(dtype):
    """A pruned prompt's heads are turned and go into the cache, its attention reads them back; then tokens, an eviction, and more tokens."""
    n, Hq, Hkv, dh, page = 150, 6, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(21)
    keep = torch.sort(torch.randperm(400, generator=g, device="cuda")[:n]).values
    pos3 = torch.stack([keep // 100, keep % 100 // 10, keep % 10]).to(torch.int32)     # frame, row and column of the kept rows
    axis = [i % 3 for i in range(dh // 2)]
    freq = (1e4 ** (-torch.arange(0, dh, 2, dtype=torch.float64) / dh)).float().cuda()
    w = 1 + 0.1 * torch.randn(dh, generator=g, device="cuda")
    table = torch.randperm(12, generator=g, device="cuda")[None].to(torch.int32)
    K, V = B.q4_pool(12, Hkv, page, dh), B.q4_pool(12, Hkv, page, dh)
    cap = 12 * page
    mass, positions = torch.zeros((1, cap), device="cuda"), torch.zeros((1, cap), dtype=torch.int32, device="cuda")
    length = torch.zeros(1, dtype=torch.int32, device="cuda")

    def layer(rows, pos, seed):
        x = torch.randn((rows, Hq + 2 * Hkv, dh), generator=g, device="cuda").to(dtype)
        q, k, v = x[:, :Hq].transpose(0, 1), x[:, Hq:Hq + Hkv].transpose(0, 1), x[:, Hq + Hkv:].transpose(0, 1)
        r = B.metok_rotate_heads(q, k, freq, pos, pair_axis=axis, eps=1e-6, q_weight=w, k_weight=w)
        ang = np.stack([num(pos[a]) * f for a, f in zip(axis, num(freq))], 1)
        assert (np.abs(num(r["k"]) - A.rotate(num(k), ang, False, 1e-6, num(w))[0]) <= 2.0 ** -7 * 8).all()
        return r["q"], r["k"], v

    q, k, v = layer(n, pos3, 0)
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    length = B.metok_paged_append_q4(k, v, K, V, table, length, offsets, positions, keep.to(torch.int32), mass)["new_len"]
    back = B.metok_paged_read_q4(K, V, table, length, offsets, n, positions=positions, dtype=dtype)
    assert torch.equal(back["positions"], keep.to(torch.int32))
    hk, hv = A.q4_values(*A.q4_hold(num(k))), A.q4_values(*A.q4_hold(num(v)))
    assert np.array_equal(num(back["k"]), hk) and np.array_equal(num(back["v"]), hv)
    got = B.metok_prefill_attention(q, back["k"], back["v"], 0.125)
    want = A.prompt_attention(num(q), hk, hv, 0.125)
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    assert (np.abs(num(got["out"]) - want["out"]) <= want["out_err"] + HALF[dtype] * np.abs(want["out"]) + rounding * want["absv"]).all()
    account = np.zeros(n)

    def token(at):
        nonlocal length, hk, hv, account
        pos = torch.full((3, 1), at, dtype=torch.int32, device="cuda")
        q1, k1, v1 = layer(1, pos, at)
        length = B.metok_paged_append_q4(k1, v1, K, V, table, length, positions=positions, pos_new=pos[0].contiguous(), mass=mass)["new_len"]
        hk, hv = (np.concatenate([h, A.q4_values(*A.q4_hold(num(x)))], 1) for h, x in ((hk, k1), (hv, v1)))
        o = B.metok_paged_attention_q4(q1.transpose(0, 1), K, V, table, length, 0.125, mass=mass)
        assert int(o["status"]) == 0
        e = A.prompt_attention(num(q1), hk, hv, 0.125)
        assert (np.abs(num(o["out"])[0] - e["out"][:, 0]) <= e["out_err"][:, 0] + HALF[dtype] * np.abs(e["out"][:, 0]) + WEIGHT[dtype] * e["absv"][:, 0] + 1e-9).all()
        x = np.einsum("hd,hnd->hn", num(q1)[:, 0], np.repeat(hk, Hq // Hkv, 0)) * 0.125
        p = np.exp(x - x.max(1, keepdims=True))
        account = np.append(account, 0.0) + (p / p.sum(1, keepdims=True)).mean(0)
        assert np.allclose(num(mass)[0, :len(account)], account, rtol=1e-4, atol=1e-6)

    for i in range(4):
        token(400 + i)
    rows = A.evict_rows(num(mass)[0], positions[0].cpu().numpy(), n + 4, 100, 3, 10)
    ev = B.metok_paged_evict([K], [V], table, length, mass[None], positions[None], 100, 3, 10)
    assert int(ev["status"]) == 0 and ev["keep_idx"][0, 0].tolist() == rows.tolist()
    length, hk, hv, account = ev["new_len"], hk[:, rows], hv[:, rows], account[rows]
    for i in range(3):
        token(404 + i)
