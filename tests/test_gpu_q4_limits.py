"""The calls on heads and on a 4-bit cache at the ends of their ranges: offsets beyond 32 bits, long tables, two calls at once, other streams."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

from .test_gpu_q4 import Cache, num

pytestmark = pytest.mark.gpu


def test_pages_beyond_32_bits_of_bytes():
    """Pools of 4.8 GB: the same rows in their last pages and in a small pool give the same bits."""
    Hkv, dh, page, n = 4, 128, 16, 70
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((Hkv, n, dh), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((1, 8, dh), generator=g, device="cuda").bfloat16()
    table = torch.tensor([[3, 0, 4, 1, 5]], dtype=torch.int32, device="cuda")
    zero, offsets = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    res = []
    for n_pages in (6, (1 << 20) + 6):
        K, V = B.q4_pool(n_pages, Hkv, page, dh), B.q4_pool(n_pages, Hkv, page, dh)
        t = table + (n_pages - 6)
        mass, pos = torch.zeros((1, 5 * page), device="cuda"), torch.zeros((1, 5 * page), dtype=torch.int32, device="cuda")
        length = B.metok_paged_append_q4(k, v, K, V, t, zero, offsets, pos, None, mass)["new_len"]
        o = B.metok_paged_attention_q4(q, K, V, t, length, 0.1, mass=mass, with_lse=True)
        ev = B.metok_paged_evict([K], [V], t, length, mass[None], pos[None], 40, 2, 5)
        back = B.metok_paged_read_q4(K, V, t, ev["new_len"], torch.tensor([0, 40], dtype=torch.int32, device="cuda"), 40, positions=pos)
        torch.cuda.synchronize()
        assert int(length) == n and int(ev["new_len"]) == 40 and int(o["status"]) == int(ev["status"]) == int(back["status"]) == 0
        res.append([o["out"], o["lse"], mass, pos, ev["keep_idx"], back["k"], back["v"], back["positions"]])
        del K, V
    assert all(torch.equal(x, y) for x, y in zip(*res))
    held = A.q4_values(*A.q4_hold(num(k)))
    assert np.array_equal(num(res[0][5]), held[:, res[0][4][0, 0].cpu().numpy()])
    torch.cuda.empty_cache()


def test_rows_beyond_32_bits_of_elements():
    """Three rows 2^30 + 8 elements apart."""
    base = torch.empty(2 * ((1 << 30) + 8) + 6 * 64, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((6, 3, 64), (64, (1 << 30) + 8, 1))
    g = torch.Generator(device="cuda").manual_seed(2)
    x.copy_(torch.randn((6, 3, 64), generator=g, device="cuda"))
    f = (1e4 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().cuda()
    dense = x.contiguous()
    want = B.metok_rotate_heads(dense[:4], dense[4:], f, eps=1e-6)
    far = B.metok_rotate_heads(x[:4], x[4:], f, eps=1e-6)
    assert torch.equal(far["q"], want["q"]) and torch.equal(far["k"], want["k"])
    # rows that far apart into a cache, and a cache's rows out to such
    K, V = B.q4_pool(1, 2, 16, 64), B.q4_pool(1, 2, 16, 64)
    one = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    length = B.metok_paged_append_q4(x[4:], x[2:4], K, V, one, one[0], off)["new_len"]
    r = B.metok_paged_read_q4(K, V, one, length, off, 3, k_out=x[4:], v_out=x[2:4])
    torch.cuda.synchronize()
    assert int(length) == 3 and int(r["status"]) == 0
    assert np.array_equal(num(x[4:]), A.q4_values(*A.q4_hold(num(dense[4:])))) and np.array_equal(num(x[2:4]), A.q4_values(*A.q4_hold(num(dense[2:4]))))
    B.metok_rotate_heads(x[:4], None, f, eps=1e-6, q_out=x[:4])
    assert torch.equal(x[:2], want["q"][:2])
    del base, x
    torch.cuda.empty_cache()


def test_one_long_sequence_of_many_pages():
    """2^20 + 5 rows of one head, all alike but one: the softmax in closed form.  A lane adds up some 40 weights, then lanes, warps and partials
    are added in trees and one chain of 450: below 100 roundings of 2^-24 on the way, 6e-6 of a sum, and 6e-6 beside its logarithm of 14."""
    n, page, dh = (1 << 20) + 5, 256, 64
    n_pages = (n + page - 1) // page
    row = torch.full((1, 1, dh), 1.0, device="cuda")
    K, V = B.q4_pool(n_pages, 1, page, dh), B.q4_pool(n_pages, 1, page, dh)
    c, e = A.q4_hold(num(row)[0, 0])
    codes, scales = (torch.from_numpy(x).cuda() for x in (c, e))
    for pool in (K, V):
        pool[..., :8 * dh] = codes.repeat(16)
        pool[..., 8 * dh:] = scales.repeat(16)
    value = A.q4_values(c, e)[0]
    table = torch.randperm(n_pages, device="cuda").to(torch.int32)[None]
    length = torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    length = B.metok_paged_append_q4(2 * row, 3 * row, K, V, table, length)["new_len"]
    q = torch.full((1, 2, dh), 0.5, device="cuda")
    mass = torch.zeros((1, n_pages * page), device="cuda")
    got = B.metok_paged_attention_q4(q, K, V, table, length, 0.25, mass=mass, with_lse=True)
    torch.cuda.synchronize()
    k1, k2 = value, A.q4_values(*A.q4_hold(np.full(dh, 2.0)))[0]
    v2 = A.q4_values(*A.q4_hold(np.full(dh, 3.0)))[0]
    x1, x2 = 0.25 * 0.5 * dh * k1, 0.25 * 0.5 * dh * k2
    total = (n - 1) * np.exp(x1 - x2) + 1
    assert int(got["status"]) == 0 and int(length) == n
    assert np.allclose(num(got["lse"]), x2 + np.log(total), rtol=1e-6)
    assert np.allclose(num(got["out"]), ((n - 1) * np.exp(x1 - x2) * value + v2) / total, rtol=1e-5)
    assert np.allclose(num(mass)[0, [0, 12345, n - 2]], np.exp(x1 - x2) / total, rtol=1e-4) and np.isclose(num(mass)[0, n - 1], 1 / total, rtol=1e-4)
    assert not num(mass)[0, n:].any()


def test_two_calls_at_once():
    """The same cache attended from two streams, each call with buffers of its own, while a third turns heads."""
    c = Cache([3000, 17, 900], 2, 128, 64, seed=3)
    q = [torch.randn((3, 8, 128), generator=c.g, device="cuda").bfloat16() for _ in range(2)]
    x = torch.randn((6, 700, 128), generator=c.g, device="cuda").bfloat16()
    f = (1e4 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float().cuda()
    attend = lambda i: B.metok_paged_attention_q4(q[i], c.k[0], c.v[0], c.block_table, c.kv_len, 0.1, with_lse=True)
    want, turned = [attend(0), attend(1)], B.metok_rotate_heads(x[:4], x[4:], f)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [[], [], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(attend(i) if i < 2 else B.metok_rotate_heads(x[:4], x[4:], f))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(r["out"], want[i]["out"]) and torch.equal(r["lse"], want[i]["lse"]) for r in got[i])
    assert all(torch.equal(r["q"], turned["q"]) and torch.equal(r["k"], turned["k"]) for r in got[2])


def test_two_captured_calls_share_nothing():
    c = Cache([400, 90], 2, 64, 16, seed=4)
    q = [torch.randn((2, 4, 64), generator=c.g, device="cuda") for _ in range(2)]
    attend = lambda i: B.metok_paged_attention_q4(q[i], c.k[0], c.v[0], c.block_table, c.kv_len, 0.1, with_lse=True)
    want = [attend(i) for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                outs.append(attend(i))
        graphs.append((graph, s))
    for _ in range(10):
        for graph, s in graphs:
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i]["out"], want[i]["out"]) and torch.equal(outs[i]["lse"], want[i]["lse"])


def test_the_binding_refuses():
    c = Cache([20, 30], 2, 64, 16, seed=5)
    q = torch.zeros((2, 4, 64), device="cuda")
    ok = lambda **kw: B.metok_paged_attention_q4(**dict(dict(q=q, k_pool=c.k[0], v_pool=c.v[0], block_table=c.block_table, kv_len=c.kv_len, softmax_scale=0.1), **kw))
    ok()
    for kw, err in ((dict(q=q.half()), TypeError), (dict(k_pool=c.k[0].float()), TypeError), (dict(v_pool=c.v[0][:1]), ValueError), (dict(q=q[:1]), ValueError),
                    (dict(k_pool=c.k[0][..., 1:]), ValueError), (dict(kv_len=c.kv_len.long()), TypeError), (dict(q=q.cpu()), ValueError), (dict(out=q.bfloat16()), TypeError)):
        with pytest.raises(err):
            ok(**kw)
    off = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    read = lambda **kw: B.metok_paged_read_q4(**dict(dict(k_pool=c.k[0], v_pool=c.v[0], block_table=c.block_table, kv_len=c.kv_len, offsets=off, n_rows=8), **kw))
    read()
    for kw, err in ((dict(dtype=torch.float16), TypeError), (dict(offsets=None), TypeError), (dict(n_rows=-1), ValueError), (dict(offsets=off[:2]), ValueError),
                    (dict(k_out=torch.zeros((2, 7, 64), dtype=torch.bfloat16, device="cuda")), ValueError), (dict(first_row=off), ValueError)):
        with pytest.raises(err):
            read(**kw)
    f = torch.ones(32, device="cuda")
    x = torch.zeros((4, 3, 64), device="cuda")
    for kw, err in ((dict(k=x[:, :2]), ValueError), (dict(inv_freq=f.double()), TypeError), (dict(positions=torch.zeros(4, dtype=torch.int32, device="cuda")), ValueError),
                    (dict(pair_axis=[0] * 31), ValueError), (dict(pair_axis=[0] * 31 + [1]), B.MetokError), (dict(q_weight=f), ValueError), (dict(eps=0.1, q_weight=f), ValueError),
                    (dict(q_out=x[:, :2]), ValueError), (dict(q=x.transpose(1, 2)), ValueError), (dict(inv_freq=f[:5]), B.MetokError), (dict(eps=-1.0), B.MetokError)):
        with pytest.raises(err):
            B.metok_rotate_heads(**dict(dict(q=x, k=x.clone(), inv_freq=f), **kw))
