"""Attention of a prompt's rows against oracle/attention_oracle.py.

Tolerances: the oracle's bounds on fp32 arithmetic; half a step of the output's type (2^-8 of a bf16 value, 2^-24 of an fp32
one); for bf16 2^-8 of the sum of weight * |v| for the weights' own rounding."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float32]


def num(t):
    return None if t is None else t.detach().cpu().double().numpy()


def offsets(lens, start=0):
    return torch.from_numpy((start + np.concatenate([[0], np.cumsum(lens)])).astype(np.int32)).cuda()


def check(q, k, v, scale, seq_q=None, seq_k=None, prefix_len=None, causal=True, softcap=0.0, slopes=None, positions=None, out=None):
    kw = dict(seq_q=seq_q, seq_k=seq_k, prefix_len=prefix_len, causal=causal, softcap=softcap, slopes=slopes, positions=positions)
    got = B.metok_prefill_attention(q, k, v, scale, with_lse=True, out=out, **kw)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    as_np = {n: (x.cpu().numpy() if isinstance(x, torch.Tensor) else x) for n, x in kw.items()}
    want = A.prompt_attention(num(q), num(k), num(v), scale, **as_np)
    tol = want["out_err"] + HALF[q.dtype] * np.abs(want["out"]) + (2.0 ** -8 * want["absv"] if q.dtype == torch.bfloat16 else 0)
    o, lse = num(got["out"]), num(got["lse"])
    inside = ~np.isnan(want["lse"])
    assert np.isfinite(o[inside]).all()
    worst = float(np.max((np.abs(o - want["out"]) / np.maximum(tol, 1e-30))[inside], initial=0.0))
    assert worst <= 1, worst
    empty = want["lse"] == -np.inf
    assert np.all(lse[empty] == -np.inf) and np.all(o[empty] == 0)
    some = inside & ~empty
    assert (np.abs(lse - want["lse"]) <= want["lse_err"] + 2.0 ** -23 * np.abs(want["lse"]))[some].all()
    return got


def rows(g, heads, n, dh, dtype, scale=1.0):
    return (torch.randn((heads, n, dh), generator=g, device="cuda") * scale).to(dtype)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,dh", [(1, 1, 64), (7, 1, 128), (4, 2, 64), (3, 3, 128), (6, 2, 128)])
@pytest.mark.parametrize("n_q,n_k", [(1, 1), (1, 300), (17, 17), (64, 64), (65, 130), (128, 128), (129, 129), (257, 300), (200, 150), (5, 0), (384, 384)])
def test_lengths_and_heads(dtype, Hq, Hkv, dh, n_q, n_k):
    g = gen(n_q * 1000 + n_k)
    check(rows(g, Hq, n_q, dh, dtype, 1.5), rows(g, Hkv, n_k, dh, dtype), rows(g, Hkv, n_k, dh, dtype), dh ** -0.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("softcap,bias,causal,prefix", [(5.0, False, True, 0), (0.0, True, True, 0), (20.0, True, True, 150), (0.0, False, False, 0), (0.0, True, False, 7),
                                                       (0.0, False, True, 128), (0.0, False, True, 10 ** 6), (0.0, False, True, -3), (2.0, True, True, 301)])
def test_cap_bias_prefix(dtype, dh, softcap, bias, causal, prefix):
    g = gen(dh + int(softcap) + prefix)
    n = 301
    q, k, v = rows(g, 4, n, dh, dtype, 5.0 if softcap else 1.5), rows(g, 2, n, dh, dtype), rows(g, 2, n, dh, dtype)
    slopes = torch.tensor([0.5, 0.1, 0.01, 0.0], device="cuda") if bias else None
    pos = torch.cumsum(torch.randint(1, 6, (n,), generator=g, device="cuda"), 0).int() if bias else None
    pre = torch.tensor([prefix], dtype=torch.int32, device="cuda") if prefix else None
    check(q, k, v, dh ** -0.5, causal=causal, softcap=softcap, slopes=slopes, positions=pos, prefix_len=pre)
    if bias:
        check(q[:, 200:], k, v, dh ** -0.5, causal=causal, softcap=softcap, slopes=slopes, prefix_len=pre)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [64, 128])
def test_packed_documents(dtype, dh):
    """Documents of every kind side by side; rows before, between the ends and behind belong to nobody, and hold NaN."""
    g = gen(7)
    lq = [1, 0, 64, 130, 3, 200, 17, 128, 5]
    lk = [1, 9, 64, 130, 300, 90, 0, 256, 5]
    pre, post = 3, 11
    nq, nk = sum(lq) + pre + post, sum(lk) + pre + post
    q, k, v = rows(g, 4, nq, dh, dtype, 1.5), rows(g, 2, nk, dh, dtype), rows(g, 2, nk, dh, dtype)
    for t in (q, k, v):
        t[:, :pre] = float("nan")
        t[:, -post:] = float("nan")
    sq, sk = offsets(lq, pre), offsets(lk, pre)
    out = torch.full_like(q, 9.0)
    got = check(q, k, v, dh ** -0.5, sq, sk, out=out)
    assert (out[:, :pre] == 9).all() and (out[:, -post:] == 9).all()
    pl = torch.tensor([0, 3, 10, 0, 299, 50, 4, 200, 1], dtype=torch.int32, device="cuda")
    slopes = torch.rand(4, generator=g, device="cuda") * 0.1
    pos = torch.randint(0, 1 << 20, (nk,), generator=g, device="cuda", dtype=torch.int32)
    check(q, k, v, dh ** -0.5, sq, sk, prefix_len=pl, softcap=9.0, slopes=slopes * 1e-4, positions=pos)
    check(q, k, v, dh ** -0.5, sq, sk, prefix_len=pl, slopes=slopes)
    check(q, k, v, dh ** -0.5, sq, sk, causal=False)
    # a document is alone in what it sees: values elsewhere that are no numbers change nothing
    k2, v2 = k.clone(), v.clone()
    lo, hi = int(sk[4]), int(sk[5])
    k2[:, lo:hi] = float("nan")
    v2[:, lo:hi] = float("inf")
    again = B.metok_prefill_attention(q, k2, v2, dh ** -0.5, sq, sk)
    torch.cuda.synchronize()
    keep = torch.ones(nq, dtype=torch.bool, device="cuda")
    keep[int(sq[4]):int(sq[5])] = False
    keep[:pre] = keep[-post:] = False
    assert torch.equal(again["out"][:, keep], got["out"][:, keep])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_small_documents(dtype):
    rng = np.random.default_rng(3)
    lq = rng.integers(0, 9, 100)
    lk = lq + rng.integers(0, 30, 100)
    g = gen(5)
    check(rows(g, 2, int(lq.sum()), 64, dtype), rows(g, 1, int(lk.sum()), 64, dtype), rows(g, 1, int(lk.sum()), 64, dtype), 0.125, offsets(lq), offsets(lk))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh,n_q,n_k", [(64, 3, 5000), (128, 64, 2600), (64, 130, 4100)])
def test_few_rows_over_many_keys_are_split(dtype, dh, n_q, n_k):
    g = gen(n_q)
    q, k, v = rows(g, 4, n_q, dh, dtype, 1.5), rows(g, 2, n_k, dh, dtype), rows(g, 2, n_k, dh, dtype)
    slopes = torch.tensor([0.02, 0.01, 0.0, 0.1], device="cuda")
    check(q, k, v, dh ** -0.5)
    check(q, k, v, dh ** -0.5, slopes=slopes, softcap=4.0)
    # documents of which some have no key for some part
    lq, lk = [n_q - 2, 2, 0], [n_k - 700, 1, 699]
    pre = torch.tensor([0, 0, 5], dtype=torch.int32, device="cuda")
    check(q, k, v, dh ** -0.5, offsets(lq), offsets(lk), prefix_len=pre)
    bad = B.metok_prefill_attention(q, k, v, 0.1, offsets([n_q, 1]), offsets([5, 6]), out=torch.full_like(q, 5.0))
    torch.cuda.synchronize()
    assert int(bad["status"]) == -1 and (bad["out"] == 5).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_repeats(dtype):
    """Token-major rows, caches with room behind their rows, heads that share one array of keys; the same bits every time."""
    g = gen(11)
    dh, n, Hq, Hkv = 128, 333, 6, 2
    qkv = (torch.randn((n, Hq + 2 * Hkv, dh + 8), generator=g, device="cuda")).to(dtype)
    q, k, v = (x[..., :dh].transpose(0, 1) for x in (qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]))
    out = torch.zeros((n, Hq, dh), dtype=dtype, device="cuda").transpose(0, 1)
    first = check(q, k, v, dh ** -0.5, out=out)
    cache_k, cache_v = (torch.full((Hkv, 500, dh), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    cache_k[:, :n], cache_v[:, :n] = k, v
    for _ in range(10):
        again = B.metok_prefill_attention(q.contiguous(), cache_k[:, :n], cache_v[:, :n], dh ** -0.5, with_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(again["out"], first["out"]) and torch.equal(again["lse"], first["lse"])
    one = k[:1].expand(3, n, dh)                                   # stride 0 between heads
    check(q[:3], one, v[:1].expand(3, n, dh), dh ** -0.5)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_and_equal_logits(dtype):
    g = gen(13)
    k, v = rows(g, 1, 400, 64, dtype), rows(g, 1, 400, 64, dtype)
    check(torch.zeros((2, 400, 64), dtype=dtype, device="cuda"), k, v, 0.125)
    q = rows(g, 2, 400, 64, dtype, 60.0)
    got = B.metok_prefill_attention(q, k, v, 1.0, with_lse=True)   # logits of hundreds: nearly all weight on one row
    torch.cuda.synchronize()
    want = A.prompt_attention(num(q), num(k), num(v), 1.0)
    assert torch.isfinite(got["out"].float()).all()
    assert (np.abs(num(got["lse"]) - want["lse"]) <= want["lse_err"] + 2.0 ** -23 * np.abs(want["lse"])).all()
    # logits that grow by a lot from tile to tile, and fall again
    ramp = torch.linspace(-40, 40, 400, device="cuda")
    k2 = torch.zeros((1, 400, 64), device="cuda")
    k2[0, :, 0] = torch.where(torch.arange(400, device="cuda") % 2 == 0, ramp, -ramp)
    q2 = torch.zeros((2, 400, 64), device="cuda")
    q2[:, :, 0] = torch.tensor([[8.0], [-8.0]], device="cuda")
    check(q2.to(dtype), k2.to(dtype), v, 0.5)
    check(q2.to(dtype), k2.to(dtype), v, 0.5, causal=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_offsets_out_of_order_write_nothing(dtype):
    g = gen(17)
    q, k, v = rows(g, 2, 40, 64, dtype), rows(g, 1, 50, 64, dtype), rows(g, 1, 50, 64, dtype)
    for sq, sk in [([0, 20, 10, 40], [0, 20, 30, 50]), ([0, 20, 30, 41], [0, 20, 30, 50]), ([-1, 20, 30, 40], [0, 20, 30, 50]), ([0, 20, 30, 40], [0, 60, 30, 50]),
                   ([0, 20, 30, 40], [0, 20, 30, 51]), ([0, 20, 30, 40], [-2 ** 31, 20, 30, 50])]:
        out = torch.full_like(q, 4.0)
        got = B.metok_prefill_attention(q, k, v, 0.125, torch.tensor(sq, dtype=torch.int32, device="cuda"), torch.tensor(sk, dtype=torch.int32, device="cuda"),
                                        out=out)
        torch.cuda.synchronize()
        assert int(got["status"]) == -1 and (out == 4).all()


def test_no_rows():
    for dtype in TYPES:
        q, k = torch.zeros((2, 0, 64), dtype=dtype, device="cuda"), torch.zeros((1, 5, 64), dtype=dtype, device="cuda")
        got = B.metok_prefill_attention(q, k, k, 0.125, with_lse=True)
        torch.cuda.synchronize()
        assert got["out"].shape == (2, 0, 64) and int(got["status"]) == 0
        got = B.metok_prefill_attention(q.new_ones((2, 3, 64)), k[:, :0], k[:, :0], 0.125, with_lse=True)
        torch.cuda.synchronize()
        assert (got["out"] == 0).all() and (got["lse"] == -np.inf).all() and int(got["status"]) == 0


def test_captured_side_by_side():
    """Two graphs captured on one stream have workspaces of their own: replayed on two streams at once they do not disturb each other."""
    g = gen(19)
    calls = [[rows(g, 4, 40, 64, torch.bfloat16), rows(g, 2, 6000 + i, 64, torch.bfloat16), rows(g, 2, 6000 + i, 64, torch.bfloat16)] for i in range(2)]
    want = [B.metok_prefill_attention(*c, 0.125)["out"].clone() for c in calls]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(s):
        for c in calls:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                outs.append(B.metok_prefill_attention(*c, 0.125)["out"])
            graphs.append(graph)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_binding_refuses():
    q, k = torch.zeros((4, 8, 64), device="cuda"), torch.zeros((2, 9, 64), device="cuda")
    i = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    ok = dict(q=q, k=k, v=k, softmax_scale=0.1)
    for kw, err in [(dict(q=q.half(), k=k.half(), v=k.half()), TypeError), (dict(k=k.bfloat16()), TypeError), (dict(v=k[:, :8]), ValueError), (dict(q=q.cpu()), ValueError),
                    (dict(seq_q=i), ValueError), (dict(seq_q=i.long(), seq_k=i.long()), TypeError), (dict(seq_q=i, seq_k=i[:1]), ValueError),
                    (dict(prefix_len=i), ValueError), (dict(slopes=torch.zeros(3, device="cuda")), ValueError), (dict(positions=i), ValueError),
                    (dict(out=q[:, :, :32]), ValueError), (dict(q=q[:3]), B.MetokError), (dict(q=q[:, :, :32], k=k[:, :, :32], v=k[:, :, :32]), B.MetokError),
                    (dict(softcap=-1.0), B.MetokError), (dict(q=q.transpose(1, 2)), ValueError), (dict(q=q[0]), ValueError)]:
        with pytest.raises(err):
            B.metok_prefill_attention(**{**ok, **kw})
