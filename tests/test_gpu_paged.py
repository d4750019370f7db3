"""The paged cache: append, attention of one token, eviction, against oracle/attention_oracle.py and exact copies.

Tolerances: the oracle's bounds on fp32 arithmetic; half a step of the output's type (2^-8 of a bf16 value, 2^-24 of an fp32 one);
for bf16 2^-16 of the sum of weight * |v| for the weights' two-part rounding."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def num(t):
    return t.detach().cpu().double().numpy()


class Cache:
    """A cache whose unused places hold NaN, and whose table behind the sequences' pages holds indices far out of range."""

    def __init__(self, lens, Hkv, dh, page, dtype, seed, room=1, layers=1, spare=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        B_ = len(lens)
        self.max_pages = max((n + room + page - 1) // page for n in lens) + 1
        used = [(n + room + page - 1) // page for n in lens]
        self.n_pages = sum(used) + spare
        order = rng.permutation(self.n_pages)[:sum(used)]
        table = np.full((B_, self.max_pages), 2 ** 30, np.int32)
        at = 0
        for b, u in enumerate(used):
            table[b, :u] = order[at:at + u]
            at += u
        self.table_np = table
        self.block_table = torch.from_numpy(table).cuda()
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.lens, self.page, self.dtype, self.Hkv, self.dh, self.S_cap = list(lens), page, dtype, Hkv, dh, self.max_pages * page
        shape = (layers, self.n_pages, Hkv, page, dh)
        self.k = torch.full(shape, float("nan"), dtype=dtype, device="cuda")
        self.v = torch.full(shape, float("nan"), dtype=dtype, device="cuda")
        for b, n in enumerate(lens):
            r = torch.arange(n, device="cuda")
            pg = self.block_table[b].long()[r // page]
            for pool in (self.k, self.v):
                pool[:, pg, :, r % page] = torch.randn((n, layers, Hkv, dh), generator=g, device="cuda").to(dtype)
        pos = [[np.sort(rng.choice(4 * self.S_cap, self.S_cap, replace=False)) for _ in range(B_)] for _ in range(layers)]
        self.positions = torch.from_numpy(np.array(pos).astype(np.int32)).cuda()
        self.mass = torch.rand((layers, B_, self.S_cap), generator=g, device="cuda")
        self.g = g


def check_attention(c, Hq, cap=0.0, bias=False, mass=True, q=None, scale=None, layer=0):
    scale = c.dh ** -0.5 if scale is None else scale
    if q is None:
        q = (torch.randn((len(c.lens), Hq, c.dh), generator=c.g, device="cuda") * (5 if cap else 1.5)).to(c.dtype)
    slopes = torch.rand(Hq, generator=c.g, device="cuda") * 0.2 if bias else None
    pos = c.positions[layer].contiguous() if bias else None
    m = c.mass[layer].clone() if mass else None
    got = B.metok_paged_attention(q, c.k[layer], c.v[layer], c.block_table, c.kv_len, scale, softcap=cap, slopes=slopes, positions=pos, mass=m, with_lse=True)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    want = A.paged_attention(num(q), num(c.k[layer]), num(c.v[layer]), c.table_np, c.lens, scale, cap, None if slopes is None else num(slopes),
                             None if pos is None else num(pos))
    tol = want["out_err"] + HALF[c.dtype] * np.abs(want["out"]) + (2.0 ** -16 * want["absv"] if c.dtype == torch.bfloat16 else 0)
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
    c = Cache([1, 0, 63, 64, 65, 200, 17, 31, 33], Hkv, dh, 16, dtype, seed=Hq)
    check_attention(c, Hq)
    check_attention(c, Hq, cap=4.0, bias=True, mass=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attention_page_sizes_cap_bias(dtype, page):
    c = Cache([3 * page + 5, 2 * page, 1, page - 1, page + 1], 2, 64, page, dtype, seed=page)
    check_attention(c, 14, cap=8.0, bias=True)


@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 2500), (torch.float32, 1300)])
def test_attention_one_long_sequence_is_split(dtype, n):
    check_attention(Cache([n], 2, 128, 64, dtype, seed=9), 14)
    check_attention(Cache([n, 3, 0, 700], 1, 64, 32, dtype, seed=10), 7, bias=True)


def test_attention_many_sequences():
    lens = np.random.default_rng(4).integers(0, 40, 333).tolist()
    check_attention(Cache(lens, 1, 64, 16, torch.bfloat16, seed=11), 3, cap=3.0)
    check_attention(Cache([0] * 7, 1, 64, 16, torch.bfloat16, seed=12), 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_weights_that_are_all_one_rows_and_large_logits(dtype):
    c = Cache([90, 130], 2, 64, 16, dtype, seed=5)
    q = torch.zeros((2, 4, 64), dtype=dtype, device="cuda")
    check_attention(c, 4, q=q)                                       # equal weights
    big = (torch.randn((2, 4, 64), generator=c.g, device="cuda") * 60).to(dtype)
    got = B.metok_paged_attention(big, c.k[0], c.v[0], c.block_table, c.kv_len, 1.0, with_lse=True)   # one row has almost all
    torch.cuda.synchronize()
    assert torch.isfinite(got["out"].float()).all() and torch.isfinite(got["lse"]).all()
    want = A.paged_attention(num(big), num(c.k[0]), num(c.v[0]), c.table_np, c.lens, 1.0)
    assert (np.abs(num(got["lse"]) - want["lse"]) <= want["lse_err"] + 2.0 ** -23 * np.abs(want["lse"])).all()


def test_attention_strides_outputs_and_repeats():
    c = Cache([77, 200, 5], 2, 64, 32, torch.bfloat16, seed=6)
    q = torch.randn((4, 3, 128), generator=c.g, device="cuda").to(torch.bfloat16)
    view = q[:, :, 32:96].transpose(0, 1)                           # [3, 4, 64], heads further apart than sequences
    whole = torch.full((3, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[:, :, 64:]
    first = check_attention(c, 4, q=view.contiguous())
    for _ in range(20):
        got = B.metok_paged_attention(view, c.k[0], c.v[0], c.block_table, c.kv_len, c.dh ** -0.5, out=out, with_lse=True)
        torch.cuda.synchronize()
        assert got["out"].data_ptr() == out.data_ptr()
        assert torch.equal(out, first["out"]) and torch.equal(got["lse"], first["lse"])
        assert (whole[:, :, :64] == 7).all()


def test_bad_pages_and_lengths_leave_the_sequence_alone():
    for dtype in (torch.bfloat16, torch.float32):
        c = Cache([70, 40, 90, 20], 2, 64, 16, dtype, seed=7)
        q = torch.randn((4, 4, 64), generator=c.g, device="cuda").to(dtype)
        good = B.metok_paged_attention(q, c.k[0], c.v[0], c.block_table, c.kv_len, 0.125, mass=c.mass[0].clone())
        table, lens = c.block_table.clone(), c.kv_len.clone()
        table[0, 2] = c.n_pages
        table[2, 5] = -1
        lens[3] = c.S_cap + 1
        mass = c.mass[0].clone()
        out = torch.full((4, 4, 64), 3.0, dtype=dtype, device="cuda")
        got = B.metok_paged_attention(q, c.k[0], c.v[0], table, lens, 0.125, mass=mass, out=out, with_lse=True)
        torch.cuda.synchronize()
        assert int(got["status"]) == -1
        for b in (0, 2, 3):
            assert (out[b] == 3.0).all() and torch.equal(mass[b], c.mass[0, b])
        lens[3] = -5
        B.metok_paged_attention(q, c.k[0], c.v[0], table, lens, 0.125, out=out)
        torch.cuda.synchronize()
        assert (out[3] == 3.0).all()
        # the other one is served; where it is cut differs with the others' lengths
        assert torch.allclose(out[1].float(), good["out"][1].float(), rtol=0.02, atol=0.02)


def append_expected(c, layer, kn, vn, off, pos_new, mass_new):
    k, v, pos, mass = c.k[layer].clone(), c.v[layer].clone(), c.positions[layer].clone(), c.mass[layer].clone()
    for b, n in enumerate(c.lens):
        for i in range(off[b], off[b + 1]):
            r = n + i - off[b]
            pg = int(c.table_np[b, r // c.page])
            k[pg, :, r % c.page], v[pg, :, r % c.page] = kn[:, i], vn[:, i]
            pos[b, r] = int(pos_new[i]) if pos_new is not None else (int(c.positions[layer, b, n - 1]) + 1 if n else 0) + i - off[b]
            mass[b, r] = float(mass_new[i]) if mass_new is not None else 0.0
    return k, v, pos, mass


def same(x, y):
    return torch.equal(x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32), y.view(torch.int16 if y.dtype == torch.bfloat16 else torch.int32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hkv,dh,page", [(1, 64, 16), (4, 128, 64), (40, 128, 16), (3, 64, 256)])
@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [0, 37, 5, 0], [16, 0, 1, 130], [0, 0, 0, 0]])
def test_append(dtype, Hkv, dh, page, counts):
    lens = [0, 15, 33, 64]
    c = Cache(lens, Hkv, dh, page, dtype, seed=1, room=max(counts) + 1)
    n = sum(counts)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    base = torch.randn((n, Hkv + 1, dh + 16), generator=c.g, device="cuda").to(dtype)
    kn = base[:, :Hkv, :dh].transpose(0, 1)                         # token by token, rows further apart than dense
    vn = torch.randn((Hkv, n, dh), generator=c.g, device="cuda").to(dtype)
    for given in (True, False):
        pos_new = torch.randint(0, 1 << 20, (n,), generator=c.g, device="cuda", dtype=torch.int32) if given else None
        mass_new = torch.rand(n, generator=c.g, device="cuda") if given else None
        k, v, pos, mass = append_expected(c, 0, kn, vn, off, pos_new, mass_new)
        K, V, P, M = c.k[0].clone(), c.v[0].clone(), c.positions[0].clone(), c.mass[0].clone()
        got = B.metok_paged_append(kn, vn, K, V, c.block_table, c.kv_len, None if counts == [1] * 4 else torch.from_numpy(off).cuda(), P, pos_new, M, mass_new)
        torch.cuda.synchronize()
        assert int(got["status"]) == 0
        assert got["new_len"].tolist() == [a + b for a, b in zip(lens, counts)]
        assert same(K, k) and same(V, v) and torch.equal(P, pos) and torch.equal(M, mass)
        assert c.kv_len.tolist() == lens
    K = c.k[0].clone()
    B.metok_paged_append(kn, vn, K, V, c.block_table, c.kv_len, torch.from_numpy(off).cuda())    # no arrays beside the pools
    torch.cuda.synchronize()
    assert same(K, k)


def test_append_reports_sequences_that_it_cannot_serve():
    c = Cache([20, 30, 40, 10, 50], 2, 64, 16, torch.float32, seed=2, room=16)
    off = torch.tensor([0, 4, 8, 12, 16, 20], dtype=torch.int32, device="cuda")
    kn, vn = (torch.randn((2, 20, 64), generator=c.g, device="cuda") for _ in range(2))
    want = append_expected(c, 0, kn, vn, off.tolist(), None, None)
    table, lens = c.block_table.clone(), c.kv_len.clone()
    table[0, 1] = -3                                                 # its rows 20 .. 23
    lens[2] = c.S_cap - 3                                            # no room for four
    lens[3] = -1
    K, V = c.k[0].clone(), c.v[0].clone()
    got = B.metok_paged_append(kn, vn, K, V, table, lens, off)
    torch.cuda.synchronize()
    assert int(got["status"]) == -1
    assert got["new_len"].tolist() == [20, 34, c.S_cap - 3, -1, 54]
    for b in (1, 4):
        pages = [int(p) for p in c.table_np[b] if p < c.n_pages]
        assert same(K[pages].contiguous(), want[0][pages].contiguous()) and same(V[pages].contiguous(), want[1][pages].contiguous())
    for bad in ([0, 4, 2, 12, 16, 20], [0, 4, 8, 12, 16, 21], [-1, 4, 8, 12, 16, 20]):
        K = c.k[0].clone()
        got = B.metok_paged_append(kn, vn, K, V, c.block_table, c.kv_len, torch.tensor(bad, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert int(got["status"]) == -1


def check_evict(c, budget, sink, recent):
    L, Bn = c.mass.shape[:2]
    K, V, P, M = c.k.clone(), c.v.clone(), c.positions.clone(), c.mass.clone()
    got = B.metok_paged_evict(list(K.unbind(0)), list(V.unbind(0)), c.block_table, c.kv_len, M, P, budget, sink, recent)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    k, v, p, m = c.k.clone(), c.v.clone(), c.positions.clone(), c.mass.clone()
    keep = torch.full((L, Bn, budget), -1, dtype=torch.int32)
    for l in range(L):
        for b, n in enumerate(c.lens):
            if n == 0:
                continue
            rows = A.evict_rows(num(c.mass[l, b]), num(c.positions[l, b]), n, budget, sink, recent)
            keep[l, b, :len(rows)] = torch.from_numpy(rows.astype(np.int32))
            if n <= budget:
                continue
            src, dst = torch.from_numpy(rows).cuda(), torch.arange(len(rows), device="cuda")
            t = c.block_table[b].long()
            for new, old in ((k, c.k), (v, c.v)):
                new[l, t[dst // c.page], :, dst % c.page] = old[l, t[src // c.page], :, src % c.page]
            m[l, b, :n] = 0
            m[l, b, :len(rows)] = c.mass[l, b][src]
            p[l, b, :len(rows)] = c.positions[l, b][src]
    assert torch.equal(got["keep_idx"].cpu(), keep)
    assert got["new_len"].tolist() == [min(n, budget) for n in c.lens]
    assert same(K, k) and same(V, v) and torch.equal(P, p) and same(M, m)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hkv,dh,page,budget,sink,recent", [(1, 64, 16, 1, 0, 1), (4, 128, 64, 30, 4, 8), (2, 64, 32, 100, 0, 1), (3, 64, 16, 63, 100, 20),
                                                            (2, 128, 256, 199, 1000000, 1), (2, 64, 16, 200, 2, 3), (1, 64, 16, 10, 0, 2 ** 31 - 1)])
def test_evict(dtype, Hkv, dh, page, budget, sink, recent):
    c = Cache([0, 1, 29, 30, 31, 200, 64, 63, 150], Hkv, dh, page, dtype, seed=budget, layers=3)
    check_evict(c, budget, sink, recent)


def test_evict_ties_nans_and_order():
    c = Cache([500, 300, 77], 1, 64, 16, torch.bfloat16, seed=3, layers=2)
    c.mass = torch.round(c.mass * 4) / 4                             # many equal weights
    c.mass[0, 0, 5:60:7] = float("nan")
    c.mass[0, 1, 3:50:11] = float("inf")
    c.mass[1, 0, 3:50:11] = -0.0
    c.mass[1, 1] = 0.0
    c.mass[1, 2] = -float("inf")
    perm = torch.from_numpy(np.random.default_rng(0).permutation(77)).cuda()
    c.positions[0, 2, :77] = c.positions[0, 2, :77][perm]
    for budget in (20, 76, 299):
        check_evict(c, budget, 40, 13)


def test_evict_of_long_sequences():
    check_evict(Cache([5000, 9001], 1, 64, 128, torch.bfloat16, seed=8), 1263, 16, 128)
    check_evict(Cache([1200, 1111], 1, 64, 128, torch.bfloat16, seed=8, layers=70), 1100, 16, 128)


def test_evict_leaves_bad_and_shared_sequences_alone():
    c = Cache([60, 60, 60, 60, 60, 60], 2, 64, 16, torch.float32, seed=4, layers=2)
    table, lens = c.block_table.clone(), c.kv_len.clone()
    table[0, 1] = table[1, 2]                                        # two sequences share a page
    table[2, 3] = c.n_pages + 5
    lens[3] = -2
    table[4, 0] = table[4, 3]                                        # one twice in a sequence
    K, V, P, M = c.k.clone(), c.v.clone(), c.positions.clone(), c.mass.clone()
    got = B.metok_paged_evict(list(K.unbind(0)), list(V.unbind(0)), table, lens, M, P, 20, 2, 2)
    torch.cuda.synchronize()
    assert int(got["status"]) == -1
    assert got["new_len"].tolist() == [60, 60, 60, -2, 60, 20]
    assert torch.equal(P[:, :5], c.positions[:, :5]) and torch.equal(M[:, :5], c.mass[:, :5])
    own = [int(p) for p in c.table_np[5] if p < c.n_pages]
    others = [p for p in range(c.n_pages) if p not in own]
    assert same(K[:, others].contiguous(), c.k[:, others].contiguous()) and same(V[:, others].contiguous(), c.v[:, others].contiguous())
    assert (got["keep_idx"][:, :5] == -1).all() and (got["keep_idx"][:, 5] >= 0).all()
    M2 = c.mass.clone()
    got = B.metok_paged_evict(list(c.k.clone().unbind(0)), list(c.v.clone().unbind(0)), c.block_table, c.kv_len, M2, c.positions.clone(), 20, 2, 2)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0 and got["new_len"].tolist() == [20] * 6


def test_a_conversation_in_a_captured_graph():
    """Append, attention and eviction as a decoding loop uses them, once eagerly and once as a replayed graph."""
    def make():
        return Cache([100, 40], 2, 64, 16, torch.bfloat16, seed=21, room=40)

    def steps(c, kn, vn, q, lens):
        outs = []
        for t in range(6):
            new = B.metok_paged_append(kn[t], vn[t], c.k[0], c.v[0], c.block_table, lens[t], positions=c.positions[0], mass=c.mass[0], new_len=lens[t + 1])
            r = B.metok_paged_attention(q[t], c.k[0], c.v[0], c.block_table, new["new_len"], 0.125, positions=c.positions[0], mass=c.mass[0],
                                        slopes=torch.full((4,), 0.01, device="cuda"))
            outs.append(r["out"])
            if t == 3:
                B.metok_paged_evict([c.k[0]], [c.v[0]], c.block_table, lens[4], c.mass, c.positions, 50, 4, 8, new_len=lens[7])
                lens[4].copy_(lens[7])
        return outs

    g = torch.Generator(device="cuda").manual_seed(5)
    kn, vn = (torch.randn((6, 2, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((6, 2, 4, 64), generator=g, device="cuda").bfloat16()
    a = make()
    la = [torch.tensor([100, 40], dtype=torch.int32, device="cuda")] + [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(7)]
    eager = [o.clone() for o in steps(a, kn, vn, q, la)]
    torch.cuda.synchronize()
    assert la[6].tolist() == [52, 46]
    b = make()
    lb = [t.clone() for t in [torch.tensor([100, 40], dtype=torch.int32, device="cuda")] + la[1:]]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        warm = make()
        steps(warm, kn, vn, q, [t.clone() for t in lb])
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            outs = steps(b, kn, vn, q, lb)
    fresh = make()
    for name in ("k", "v", "positions", "mass"):
        getattr(b, name).copy_(getattr(fresh, name))
    lb[0].copy_(torch.tensor([100, 40]))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert [t.tolist() for t in lb] == [t.tolist() for t in la]
    for x, y in zip(outs, eager):
        assert torch.equal(x, y)
    assert same(a.k, b.k) and same(a.v, b.v) and torch.equal(a.positions, b.positions) and torch.equal(a.mass, b.mass)


def test_binding_refuses():
    c = Cache([20, 30], 2, 64, 16, torch.bfloat16, seed=2)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    ok = dict(q=q, k_pool=c.k[0], v_pool=c.v[0], block_table=c.block_table, kv_len=c.kv_len, softmax_scale=0.1)
    for kw, err in [(dict(q=q.float()), TypeError), (dict(q=q.cpu()), ValueError), (dict(q=q[:1]), ValueError), (dict(q=q[:, :3]), B.MetokError),
                    (dict(k_pool=c.k[0].half(), v_pool=c.v[0].half(), q=q.half()), TypeError), (dict(v_pool=c.v[0][:1]), ValueError),
                    (dict(block_table=c.block_table.long()), TypeError), (dict(kv_len=c.kv_len[:1]), ValueError), (dict(mass=c.mass[0, :1]), ValueError),
                    (dict(positions=c.positions[0].cpu()), ValueError), (dict(slopes=torch.zeros(3, device="cuda")), ValueError),
                    (dict(block_table=c.block_table.T), ValueError), (dict(out=q[:, :, :32]), ValueError), (dict(softmax_scale=-1.0), B.MetokError),
                    (dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), ValueError)]:
        with pytest.raises(err):
            B.metok_paged_attention(**{**ok, **kw})
    with pytest.raises(B.MetokError):
        B.metok_paged_evict([c.k[0]], [c.v[0]], c.block_table, c.kv_len, c.mass, c.positions, 0, 1, 1)
    with pytest.raises(ValueError):
        B.metok_paged_evict([c.k[0]], [], c.block_table, c.kv_len, c.mass, c.positions, 4, 1, 1)
    with pytest.raises(B.MetokError):
        B.metok_paged_evict([c.k[0]], [c.v[0]], c.block_table, c.kv_len, c.mass, c.positions, 4, 1, 1, new_len=c.kv_len)
