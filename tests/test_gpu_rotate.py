"""Norms and rotary positions of heads against oracle/attention_oracle.py.

Tolerance, relative to the sum of the absolute values of the two elements that an output is made of: the sum of squares adds 16 and then up
to 8 numbers (19 roundings, half of it after the root), mean, eps, root, quotient and two products 6 more: 16 of 2^-24; the sine's argument is
rounded in units of half a turn (pi * 2^-25), sine and cosine by 2 steps, two products and a sum: below 2^-21.  Together below 2^-19; and half
a step of the output's type."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def num(t):
    return t.detach().cpu().double().numpy()


def freqs(r, base=1e4):
    return (base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().cuda()


def angles(freq, positions, axis, n):
    pos = np.arange(n)[None] if positions is None else np.atleast_2d(positions.cpu().numpy())
    return np.stack([pos[a].astype(np.float64) * f for a, f in zip(axis or [0] * len(freq), num(freq))], 1) if len(freq) else np.zeros((n, 0))


def check(got, x, ang, interleaved=False, eps=None, weight=None):
    want, size = A.rotate(num(x), ang, interleaved, eps, None if weight is None else num(weight))
    assert got.dtype == x.dtype
    assert (np.abs(num(got) - want) <= 2.0 ** -19 * size + HALF[x.dtype] * np.abs(want) + 1e-38).all()


def projections(n, Hq, Hkv, dh, dtype, seed):
    """Q and K of a layer as one product leaves them: token by token, V behind them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (torch.randn((n, Hq + 2 * Hkv, dh), generator=g, device="cuda") * 3).to(dtype)
    return g, qkv, qkv[:, :Hq].transpose(0, 1), qkv[:, Hq:Hq + Hkv].transpose(0, 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 2, 7, 130, 5000])
@pytest.mark.parametrize("Hq,Hkv,dh", [(1, 1, 64), (14, 2, 64), (28, 4, 128), (5, 5, 128), (9, 3, 64)])
def test_heads_rows_and_types(dtype, n, Hq, Hkv, dh):
    if n == 5000 and Hq != 14:
        n = 500
    g, _, q, k = projections(n, Hq, Hkv, dh, dtype, seed=n)
    pos = torch.randint(0, 20000, (3, n), generator=g, device="cuda", dtype=torch.int32)
    axis = [i % 3 for i in range(dh // 2)]
    wq, wk = (1 + 0.3 * torch.randn(dh, generator=g, device="cuda") for _ in range(2))
    f = freqs(dh)
    got = B.metok_rotate_heads(q, k, f, pos, pair_axis=axis, eps=1e-5, q_weight=wq, k_weight=wk)
    check(got["q"], q, angles(f, pos, axis, n), eps=1e-5, weight=wq)
    check(got["k"], k, angles(f, pos, axis, n), eps=1e-5, weight=wk)
    got = B.metok_rotate_heads(q, None, f, pos[0].contiguous(), interleaved=True)
    assert set(got) == {"q"}
    check(got["q"], q, angles(f, pos[:1], None, n), interleaved=True)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("part", [0, 16, 48, 64])
@pytest.mark.parametrize("interleaved", [False, True])
def test_part_of_the_elements(dh, part, interleaved):
    for dtype in (torch.bfloat16, torch.float32):
        g, _, q, k = projections(33, 6, 3, dh, dtype, seed=part)
        f = freqs(part) if part else None
        axis = ([0, 1, 2, 3] * part)[:part // 2] if part else None
        pos = torch.randint(-5000, 5000, (4, 33), generator=g, device="cuda", dtype=torch.int32)
        got = B.metok_rotate_heads(q, k, f, pos, pair_axis=axis, interleaved=interleaved, eps=1e-6)
        ang = angles(f if part else [], pos, axis, 33)
        check(got["q"], q, ang, interleaved, eps=1e-6)
        check(got["k"], k, ang, interleaved, eps=1e-6)
        plain = B.metok_rotate_heads(q, k, f, interleaved=interleaved)    # rows count themselves
        ang = angles(f if part else [], None, None, 33)
        check(plain["q"], q, ang, interleaved)
        if not part:
            assert torch.equal(plain["k"], k)


def test_far_positions():
    """An int32 position's angle is good to 2^-21 of a turn or better: it is reduced in 64 bits."""
    n = 64
    g, _, q, k = projections(n, 2, 1, 128, torch.float32, seed=3)
    pos = (torch.randint(-2 ** 31, 2 ** 31 - 1, (n,), generator=g, device="cuda", dtype=torch.int64)).to(torch.int32)
    pos[0], pos[1] = 2 ** 31 - 1, -2 ** 31
    f = freqs(128)
    check(B.metok_rotate_heads(q, k, f, pos)["q"], q, angles(f, pos, None, n))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place_and_strides(dtype):
    n = 77
    g, qkv, q, k = projections(n, 14, 2, 64, dtype, seed=4)
    f, w = freqs(64), torch.rand(64, generator=g, device="cuda")
    want = B.metok_rotate_heads(q, k, f, eps=1e-6, q_weight=w, k_weight=w)
    # into one buffer, beside one another, its other rows left alone
    whole = torch.full((n + 1, 20, 64), 7.0, dtype=dtype, device="cuda")
    got = B.metok_rotate_heads(q, k, f, eps=1e-6, q_weight=w, k_weight=w, q_out=whole[:n, 1:15].transpose(0, 1), k_out=whole[:n, 17:19].transpose(0, 1))
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["k"], want["k"])
    assert (whole[n] == 7).all() and (whole[:, 0] == 7).all() and (whole[:, 15:17] == 7).all() and (whole[:, 19] == 7).all()
    # in place
    before = qkv.clone()
    got = B.metok_rotate_heads(q, k, f, eps=1e-6, q_weight=w, k_weight=w, q_out=q, k_out=k)
    assert torch.equal(q, want["q"]) and torch.equal(k, want["k"]) and torch.equal(qkv[:, 16:], before[:, 16:])
    assert got["q"].data_ptr() == q.data_ptr()
    # outputs over inputs that are not theirs, over one another, over themselves
    for kw in (dict(k_out=q[:2]), dict(q_out=qkv.view(-1)[:14 * n * 64].view(14, n, 64)),
               dict(q_out=whole[:n, :14].transpose(0, 1), k_out=whole[:n, 13:15].transpose(0, 1))):
        with pytest.raises(B.MetokError):
            B.metok_rotate_heads(q, k, f, **kw)


def test_zeros_infinities_and_repeats():
    g, _, q, k = projections(40, 4, 2, 128, torch.bfloat16, seed=5)
    q, k = q.contiguous(), k.contiguous()
    f = freqs(128)
    q[0, 0] = 0
    k[1, 3, 5] = float("nan")
    k[0, 4, 7] = float("inf")
    first = B.metok_rotate_heads(q, k, f, eps=0.0)
    assert torch.isnan(first["q"][0, 0].float()).all()                  # 0 over 0
    assert (B.metok_rotate_heads(q, k, f, eps=1e-6)["q"][0, 0] == 0).all()
    assert torch.isnan(first["k"][1, 3].float()).all() and torch.isfinite(first["k"][1, 2].float()).all()
    assert torch.isfinite(first["k"][0, 3].float()).all() and torch.isfinite(first["k"][1, 4].float()).all()
    for _ in range(5):
        again = B.metok_rotate_heads(q, k, f, eps=0.0)
        assert torch.equal(again["q"].view(torch.int16), first["q"].view(torch.int16))
    for pos in (None, torch.zeros((3, 0), dtype=torch.int32, device="cuda")):
        empty = B.metok_rotate_heads(q[:, :0], k[:, :0], f, pos)
        assert empty["q"].shape == (4, 0, 128) and empty["k"].shape == (2, 0, 128)


def test_captured_and_on_another_stream():
    g, _, q, k = projections(50, 4, 2, 64, torch.bfloat16, seed=6)
    pos = torch.zeros(50, dtype=torch.int32, device="cuda")
    f = freqs(64)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        B.metok_rotate_heads(q, k, f, pos)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = B.metok_rotate_heads(q, k, f, pos)
    for start in (0, 1000):
        pos.copy_(torch.arange(start, start + 50, dtype=torch.int32, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        check(got["q"], q, angles(f, pos, None, 50))
