"""Attention and the paged cache at the ends of their ranges: large values in places that do not count, thousands of documents, groups
of many heads, hundreds of sequences, pools of more than 2^32 elements, two streams at once.  Tolerances as in
test_gpu_prompt_attention.py and test_gpu_paged.py, whose checks are used."""

import numpy as np
import pytest
import torch

from paper_2506_02850_b200 import binding as B

from . import test_gpu_paged as P
from . import test_gpu_prompt_attention as Q

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("softcap,bias", [(0.0, False), (6.0, True)])
def test_values_that_a_row_does_not_see_may_be_large(dtype, dh, softcap, bias):
    """Row i does not see key i + 1, whose V is up to 2^99: its weight has to be 0, not merely small.  K there may hold anything."""
    g = Q.gen(21)
    n = 300
    q, k, v = Q.rows(g, 4, n, dh, dtype, 1.5), Q.rows(g, 2, n, dh, dtype), Q.rows(g, 2, n, dh, dtype)
    for j in (17, 100, 128, 200, 255, 256, 299):
        v[:, j] = 6.0e29 * (-1) ** j
        k[:, j] *= 40
    slopes = torch.tensor([0.4, 0.01, 0.0, 0.1], device="cuda") if bias else None
    Q.check(q, k, v, dh ** -0.5, softcap=softcap, slopes=slopes)
    Q.check(q[:, 120:], k, v, dh ** -0.5, softcap=softcap, slopes=slopes, prefix_len=torch.tensor([90], dtype=torch.int32, device="cuda"))
    # the last row alone sees the last key (with a cap its logits decide how a tile's tanh are computed)
    k, v = Q.rows(g, 2, n, dh, dtype), Q.rows(g, 2, n, dh, dtype)
    k2, v2 = k.clone(), v.clone()
    k2[:, -1] = float("nan")
    v2[:, -1] = 1.0e30
    a = B.metok_prefill_attention(q, k, v, dh ** -0.5, softcap=softcap, slopes=slopes)["out"]
    b = B.metok_prefill_attention(q, k2, v2, dh ** -0.5, softcap=softcap, slopes=slopes)["out"]
    torch.cuda.synchronize()
    assert torch.isfinite(b[:, :-1]).all()
    assert torch.allclose(a[:, :-1], b[:, :-1], rtol=2.0 ** -7, atol=2.0 ** -7) if softcap else torch.equal(a[:, :-1], b[:, :-1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rise", [3.0, 14.0, 60.0, 900.0])
def test_logits_that_rise_towards_the_first_keys(dtype, rise):
    """Logits of 64 keys after 64 keys lie `rise` above the ones before, in the order that the kernel takes them and against it."""
    n = 640
    for order in (1, -1):
        k = torch.zeros((1, n, 64), device="cuda")
        k[0, :, 0] = (torch.arange(n, device="cuda") // 64).float() if order == 1 else (n // 64 - 1 - torch.arange(n, device="cuda") // 64).float()
        k[0, :, 1:] = torch.randn((n, 63), generator=Q.gen(2), device="cuda") * 0.1
        q = torch.randn((1, 200, 64), generator=Q.gen(3), device="cuda") * 0.1
        q[:, :, 0] = rise
        v = torch.randn((1, n, 64), generator=Q.gen(4), device="cuda")
        Q.check(q.to(dtype), k.to(dtype), v.to(dtype), 1.0)
        Q.check(q.to(dtype), k.to(dtype), v.to(dtype), 1.0, causal=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_thousands_of_documents(dtype):
    rng = np.random.default_rng(1)
    lq = rng.integers(0, 5, 8192)
    lk = lq + rng.integers(0, 6, 8192)
    lq[5000:6000] = 0
    g = Q.gen(6)
    Q.check(Q.rows(g, 2, int(lq.sum()), 64, dtype), Q.rows(g, 1, int(lk.sum()), 64, dtype), Q.rows(g, 1, int(lk.sum()), 64, dtype), 0.125, Q.offsets(lq), Q.offsets(lk))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,dh", [(40, 1, 64), (130, 1, 64), (260, 2, 128), (128, 1, 128), (65, 1, 64)])
def test_many_heads_on_one(dtype, Hq, Hkv, dh):
    g = Q.gen(Hq)
    slopes = torch.rand(Hq, generator=g, device="cuda") * 0.1
    Q.check(Q.rows(g, Hq, 7, dh, dtype, 1.5), Q.rows(g, Hkv, 200, dh, dtype), Q.rows(g, Hkv, 200, dh, dtype), dh ** -0.5, slopes=slopes)
    Q.check(Q.rows(g, Hq, 9, dh, dtype, 1.5), Q.rows(g, Hkv, 40, dh, dtype), Q.rows(g, Hkv, 40, dh, dtype), dh ** -0.5, Q.offsets([4, 0, 5]), Q.offsets([4, 3, 33]),
            softcap=4.0)
    c = P.Cache([100, 0, 37], Hkv, dh, 16, dtype, seed=Hq)
    P.check_attention(c, Hq, bias=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_k", [40, 300])
def test_documents_without_keys_have_no_positions_to_read(dtype, n_k):
    g = Q.gen(9)
    q, k, v = Q.rows(g, 2, 30, 64, dtype), Q.rows(g, 1, n_k, 64, dtype), Q.rows(g, 1, n_k, 64, dtype)
    pos = torch.arange(n_k, device="cuda", dtype=torch.int32) * 3
    slopes = torch.tensor([0.1, 0.2], device="cuda")
    for lq, lk in (([10, 20], [n_k, 0]), ([10, 20], [0, n_k]), ([10, 0, 20], [n_k, 0, 0])):
        Q.check(q, k, v, 0.125, Q.offsets(lq), Q.offsets(lk), slopes=slopes, positions=pos, prefix_len=torch.full((len(lq),), 4, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
def test_two_streams_at_once(dtype):
    """Calls of every kind on two streams, each with tensors of its own: the results are those of one after the other."""
    def build(seed):
        c = P.Cache([900 + seed, 50, 333], 2, 64, 16, dtype, seed=seed)
        g = Q.gen(seed)
        return c, Q.rows(g, 14, 700, 64, dtype), Q.rows(g, 2, 700, 64, dtype), Q.rows(g, 2, 700, 64, dtype), torch.randn((3, 14, 64), generator=g, device="cuda").to(dtype)

    def run(args):
        c, q, k, v, one = args
        mass, pos, K, V = c.mass[0].clone(), c.positions[0].clone(), c.k[0].clone(), c.v[0].clone()
        a = B.metok_prefill_attention(q, k, v, 0.125)["out"]
        length = B.metok_paged_append(k[:, :3], v[:, :3], K, V, c.block_table, c.kv_len - 1, positions=pos, mass=mass)["new_len"]
        d = B.metok_paged_attention(one, K, V, c.block_table, length, 0.125, mass=mass)["out"]
        e = B.metok_paged_evict([K], [V], c.block_table, length, mass, pos, 40, 2, 3)["keep_idx"]
        return a, d, e, mass, pos

    sets = [build(1), build(2)]
    want = [run(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(run(sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            for x, y in zip(r, want[i]):
                assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", TYPES)
def test_two_thousand_heads_with_weights(dtype):
    P.check_attention(P.Cache([5, 40], 2048, 64, 16, dtype, seed=2), 2048)


def test_evict_of_hundreds_of_sequences():
    """More sequences than look through each other's pages: the pages are claimed."""
    rng = np.random.default_rng(5)
    c = P.Cache(rng.integers(0, 60, 300).tolist(), 1, 64, 16, torch.bfloat16, seed=7, layers=2)
    P.check_evict(c, 20, 2, 5)
    table, lens = c.block_table.clone(), c.kv_len.clone()
    full = [b for b, n in enumerate(c.lens) if n > 32]
    x, y, z, w = full[:4]
    table[x, 1] = table[y, 2]
    table[z, 0] = table[z, 1]
    table[w, 0] = -1
    lens[full[4]] = c.S_cap + 1
    bad = set(full[:5])
    K, V, Pos, M = c.k.clone(), c.v.clone(), c.positions.clone(), c.mass.clone()
    got = B.metok_paged_evict(list(K.unbind(0)), list(V.unbind(0)), table, lens, M, Pos, 20, 2, 5)
    torch.cuda.synchronize()
    assert int(got["status"]) == -1
    for b, n in enumerate(c.lens):
        if b in bad:
            assert (got["keep_idx"][:, b] == -1).all() and int(got["new_len"][b]) == int(lens[b])
            assert torch.equal(M[:, b], c.mass[:, b]) and torch.equal(Pos[:, b], c.positions[:, b])
        else:
            assert int(got["new_len"][b]) == min(n, 20)
            used = table[b, :(n + 15) // 16].long()
            if n <= 20:
                assert P.same(K[:, used], c.k[:, used])


def test_evict_of_sequences_too_long_for_shared_memory():
    """More keys than a select's shared memory holds, with many equal weights at the threshold."""
    c = P.Cache([50001, 100], 1, 64, 256, torch.bfloat16, seed=9)
    P.check_evict(c, 20000, 16, 128)
    c.mass = torch.round(c.mass * 3) / 3
    P.check_evict(c, 30000, 16, 128)


def big_pool(n_pages, Hkv, page, dh):
    """Two pools, of which only the pages that are used get values."""
    return [torch.empty((n_pages, Hkv, page, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def test_pools_of_more_than_2_32_elements():
    """The same rows in a small cache and at both ends of pools of 8.6 GB each give the same results."""
    Hkv, page, dh, n_pages = 2, 256, 64, (1 << 17) + 8
    c = P.Cache([600, 300, 700], Hkv, dh, page, torch.bfloat16, seed=3, room=2)
    K, V = big_pool(n_pages, Hkv, page, dh)
    far = torch.cat([torch.arange(3), n_pages - 1 - torch.arange(c.n_pages)]).cuda()[torch.randperm(c.n_pages + 3, generator=torch.Generator().manual_seed(1))]
    used = c.block_table < c.n_pages
    table = torch.where(used, far[c.block_table.clamp(0, c.n_pages - 1).long()].int(), c.block_table)
    place = far[:c.n_pages]
    K[place], V[place] = c.k[0], c.v[0]
    k, v = c.k[0].clone(), c.v[0].clone()
    g = Q.gen(4)
    new = [Q.rows(g, Hkv, 3, dh, torch.bfloat16) for _ in range(2)]
    q = torch.randn((3, 14, dh), generator=g, device="cuda").bfloat16()
    res = []
    for a, b, t in ((k, v, c.block_table), (K, V, table)):
        mass, pos = c.mass[0].clone(), c.positions[0].clone()
        length = B.metok_paged_append(*new, a, b, t, c.kv_len, positions=pos, mass=mass)["new_len"]
        out = B.metok_paged_attention(q, a, b, t, length, 0.125, mass=mass, with_lse=True)
        ev = B.metok_paged_evict([a], [b], t, length, mass, pos, 100, 4, 8)
        torch.cuda.synchronize()
        assert int(out["status"]) == 0 and int(ev["status"]) == 0
        res.append((out["out"], out["lse"], mass, pos, ev["keep_idx"], ev["new_len"]))
    for x, y in zip(*res):
        assert P.same(x, y)
    assert P.same(K[place], k) and P.same(V[place], v)


def test_pools_of_more_pages_than_a_sequence_can_mark():
    """More than 2^18 pages: an eviction claims them in global memory."""
    Hkv, page, dh, n_pages = 1, 16, 64, (1 << 18) + 40
    c = P.Cache([90, 10, 200], Hkv, dh, page, torch.bfloat16, seed=6)
    K, V = big_pool(n_pages, Hkv, page, dh)
    place = n_pages - 1 - torch.arange(c.n_pages, device="cuda")
    K[place], V[place] = c.k[0], c.v[0]
    table = torch.where(c.block_table < c.n_pages, place[c.block_table.clamp(0, c.n_pages - 1).long()].int(), c.block_table)
    res = []
    for a, b, t in ((c.k[0].clone(), c.v[0].clone(), c.block_table), (K, V, table)):
        mass, pos = c.mass[0].clone(), c.positions[0].clone()
        ev = B.metok_paged_evict([a], [b], t, c.kv_len, mass, pos, 50, 4, 8)
        torch.cuda.synchronize()
        assert int(ev["status"]) == 0
        res.append((ev["keep_idx"], mass, pos, a if a is not K else K[place], b if b is not V else V[place]))
    for x, y in zip(*res):
        assert P.same(x, y)


@pytest.mark.parametrize("dtype", TYPES)
def test_sequences_may_share_the_pages_of_a_common_prompt(dtype):
    c = P.Cache([64 + 20, 64 + 7, 64], 2, 64, 32, dtype, seed=13)
    c.block_table[1:, :2] = c.block_table[0, :2]
    c.table_np[1:, :2] = c.table_np[0, :2]
    P.check_attention(c, 14, bias=True)


def test_rows_of_the_output_that_would_overlap_are_refused():
    q, k = torch.randn((4, 10, 64), device="cuda"), torch.randn((2, 10, 64), device="cuda")
    room = torch.zeros(64 * 200, device="cuda")
    for strides in ((64, 64, 1), (128, 64, 1), (64, 192, 1)):
        with pytest.raises(B.MetokError):
            B.metok_prefill_attention(q, k, k, 0.1, out=room.as_strided((4, 10, 64), strides))
    for strides in ((640, 64, 1), (64, 256, 1), (704, 64, 1), (68, 272, 1)):
        Q.check(q, k, k, 0.1, out=room.as_strided((4, 10, 64), strides))
    for cap in (1e-40, 2e38):
        with pytest.raises(B.MetokError):
            B.metok_prefill_attention(q, k, k, 0.1, softcap=cap)
    c = P.Cache([20, 30], 2, 64, 16, torch.float32, seed=1)
    one = torch.randn((2, 4, 64), device="cuda")
    for strides in ((64, 64, 1), (128, 64, 1), (64, 64, 1)):
        with pytest.raises(B.MetokError):
            B.metok_paged_attention(one, c.k[0], c.v[0], c.block_table, c.kv_len, 0.1, out=room.as_strided((2, 4, 64), strides))
    for cap in (1e-40, 2e38):
        with pytest.raises(B.MetokError):
            B.metok_paged_attention(one, c.k[0], c.v[0], c.block_table, c.kv_len, 0.1, softcap=cap)
    pool = torch.zeros(9 * 2 * 16 * 64, device="cuda")
    a, b = pool[:8 * 2 * 16 * 64].view(8, 2, 16, 64), pool[2 * 16 * 64:].view(8, 2, 16, 64)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8)
    with pytest.raises(B.MetokError):
        B.metok_paged_evict([a], [b], table, torch.tensor([100], dtype=torch.int32, device="cuda"), torch.zeros((1, 128), device="cuda"),
                            torch.zeros((1, 128), dtype=torch.int32, device="cuda"), 50, 1, 1)


@pytest.mark.parametrize("softcap", [0.0, 6.0])
@pytest.mark.parametrize("lens", [[1000], [500, 1, 130, 0, 369], [128] * 7 + [104], [30, 900, 70], [40] * 25])
def test_more_pairs_of_tiles_than_processors(softcap, lens):
    """Every processor has several pairs of tiles, cut where it suits the others."""
    g = Q.gen(31)
    q, k, v = Q.rows(g, 40, 1000, 64, torch.bfloat16, 1.5), Q.rows(g, 40, 1000, 64, torch.bfloat16), Q.rows(g, 40, 1000, 64, torch.bfloat16)
    i = Q.offsets(lens)
    Q.check(q, k, v, 0.125, i, i, softcap=softcap)
    Q.check(q[:, :700], k, v, 0.125, Q.offsets([300, 0, 400]), Q.offsets([310, 90, 600]), softcap=softcap)
    # most rows are in no document: less work than their number says
    Q.check(q, k, v, 0.125, Q.offsets([5, 0, 90], 17), Q.offsets([5, 300, 90], 200), softcap=softcap)
    Q.check(q, k, v, 0.125, Q.offsets([3], 900), Q.offsets([1], 900), softcap=softcap)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hkv,dh", [(5, 64), (40, 64), (9, 128), (4, 64)])
def test_evict_of_many_heads(dtype, Hkv, dh):
    c = P.Cache([100, 31, 77, 500], Hkv, dh, 16, dtype, seed=Hkv, layers=2)
    P.check_evict(c, 30, 2, 5)
    P.check_evict(c, 90, 0, 40)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("softcap", [0.0, 6.0])
def test_slopes_of_either_sign_and_any_size(dtype, softcap):
    g = Q.gen(41)
    n = 500
    q, k, v = Q.rows(g, 4, n, 64, dtype), Q.rows(g, 2, n, 64, dtype), Q.rows(g, 2, n, 64, dtype)
    slopes = torch.tensor([-0.3, 1000.0, -2.0, 1e-6], device="cuda")
    for kw in (dict(), dict(causal=False), dict(prefix_len=torch.tensor([333], dtype=torch.int32, device="cuda"))):
        Q.check(q, k, v, 0.125, softcap=softcap, slopes=slopes, **kw)
    c = P.Cache([300, 17], 2, 64, 32, dtype, seed=1)
    one = torch.randn((2, 4, 64), generator=g, device="cuda").to(dtype)
    got = B.metok_paged_attention(one, c.k[0], c.v[0], c.block_table, c.kv_len, 0.125, softcap=softcap, slopes=slopes)
    torch.cuda.synchronize()
    want = P.A.paged_attention(P.num(one), P.num(c.k[0]), P.num(c.v[0]), c.table_np, c.lens, 0.125, softcap, P.num(slopes))
    assert (np.abs(P.num(got["out"]) - want["out"]) <= want["out_err"] + P.HALF[dtype] * np.abs(want["out"]) + 2.0 ** -16 * want["absv"]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_more_than_2_32_elements_apart(dtype):
    """Every tensor of a call is a slice of one buffer whose rows lie 2^26 elements apart."""
    n, far = 80, 1 << 26
    room = torch.empty(n * far, dtype=dtype, device="cuda")
    at = lambda col, heads: room[col:].as_strided((heads, n, 64), (64, far, 1))
    g = Q.gen(51)
    dense = [Q.rows(g, 4, n, 64, dtype), Q.rows(g, 2, n, 64, dtype), Q.rows(g, 2, n, 64, dtype)]
    q, k, v, out = at(0, 4), at(512, 2), at(1024, 2), at(2048, 4)
    for x, y in zip((q, k, v), dense):
        x.copy_(y)
    want = B.metok_prefill_attention(*dense, 0.125)["out"]
    B.metok_prefill_attention(q, k, v, 0.125, out=out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    # heads far apart, in the appended rows too
    wide = lambda col: room[col:].as_strided((2, 70, 64), (20 * far, 128, 1))
    kn, vn = wide(4096), wide(20480)
    kd, vd = dense[1][:, :70].contiguous(), dense[2][:, :70].contiguous()
    kn.copy_(kd)
    vn.copy_(vd)
    table = torch.arange(5, dtype=torch.int32, device="cuda").view(1, 5)
    off, length = torch.tensor([0, 70], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    pools = [[torch.zeros((5, 2, 16, 64), dtype=dtype, device="cuda") for _ in range(2)] for _ in range(2)]
    for (a, b), (x, y) in zip(pools, ((kn, vn), (kd, vd))):
        assert int(B.metok_paged_append(x, y, a, b, table, length, off)["new_len"]) == 70
    assert torch.equal(pools[0][0], pools[1][0]) and torch.equal(pools[0][1], pools[1][1])


def test_more_sequences_than_one_look():
    """Hundreds of sequences of every length, with weights and a bias: where each lies in the line comes from the first kernel."""
    lens = np.random.default_rng(8).integers(0, 200, 40).tolist() + [0, 900, 1, 0]
    c = P.Cache(lens, 2, 64, 32, torch.bfloat16, seed=14)
    P.check_attention(c, 6, bias=True)
    c.kv_len[3] = -1
    c.lens = list(c.lens)
    out = torch.full((len(lens), 6, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    got = B.metok_paged_attention(torch.randn((len(lens), 6, 64), generator=c.g, device="cuda").bfloat16(), c.k[0], c.v[0], c.block_table, c.kv_len, 0.125, out=out)
    torch.cuda.synchronize()
    assert int(got["status"]) == -1 and (out[3] == 3).all() and torch.isfinite(out.float()).all()
