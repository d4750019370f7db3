"""Attention over a cache held in 4 bits: rows behind a sequence's last one, and what shared memory holds from other calls, change no bit."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

from .test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh", [(4, 2, 64), (14, 2, 128), (12, 1, 128), (9, 1, 64)])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (0.0, True), (20.0, False), (20.0, True)])
def test_what_unused_rows_hold(dtype, Hq, Hkv, dh, cap, bias):
    """Logits are far below the cap, those of the unused rows (were there any) far above it."""
    lens = [5, 33, 150, 131, 48, 0]
    c = Cache(lens, Hkv, dh, 64, seed=Hq)
    q = torch.randn((len(lens), Hq, dh), generator=c.g, device="cuda").to(dtype)
    slopes = torch.rand(Hq, generator=c.g, device="cuda") * 0.01 if bias else None
    pos = c.positions[0].contiguous() if bias else None

    def call(K, V):
        mass = torch.zeros_like(c.mass[0])
        r = B.metok_paged_attention_q4(q, K, V, c.block_table, c.kv_len, dh ** -0.5, softcap=cap, slopes=slopes, positions=pos, mass=mass, with_lse=True)
        assert int(r["status"]) == 0
        return r["out"], r["lse"], mass

    want = call(c.k[0], c.v[0])                                      # all bits set: scales of NaN
    loud = torch.full_like(c.k[0], 0x11)                             # codes of -7 and a scale, below, of 896: also what the calls in between leave in shared memory
    loud[..., 8 * dh:] = 0x53
    for fill in (0, 1, 2):
        K, V = c.k[0].clone(), c.v[0].clone()
        for pool, other in ((K, loud), (V, loud)):
            codes, scales = pool[..., :8 * dh].view(-1, 16, dh // 2), pool[..., 8 * dh:].view(-1, 16, dh // 16)
            ones = (scales == 255).all(-1)                           # places of no row
            for part, value in ((codes, other[..., :8 * dh]), (scales, other[..., 8 * dh:])):
                if fill:
                    part[ones] = value.reshape(part.shape)[ones]
            if fill:
                pool[..., :8 * dh], pool[..., 8 * dh:] = codes.reshape(pool.shape[:-1] + (-1,)), scales.reshape(pool.shape[:-1] + (-1,))
        if fill == 2:
            B.metok_paged_attention_q4(q, loud, loud, torch.zeros_like(c.block_table), torch.full_like(c.kv_len, c.S_cap), dh ** -0.5, softcap=cap)
        got = call(K, V)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), fill


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_other_calls_leave_in_shared_memory(dtype):
    """Calls over loud caches of many lengths between calls of which every sequence ends within a warp's rows."""
    Hq, Hkv, dh = 8, 1, 128
    lens = [33, 97, 161, 225, 1, 65] * 20
    c = Cache(lens, Hkv, dh, 16, seed=2)
    q = torch.randn((len(lens), Hq, dh), generator=c.g, device="cuda").to(dtype)
    loud = torch.full((1, Hkv, 1, 9 * dh), 0x11, dtype=torch.uint8, device="cuda")
    loud[..., 8 * dh:] = 0x53
    call = lambda: B.metok_paged_attention_q4(q, c.k[0], c.v[0], c.block_table, c.kv_len, dh ** -0.5, softcap=20.0, with_lse=True)
    want = call()
    for n in (128, 2000, 20000):
        one = torch.zeros((1, n // 16 + 1), dtype=torch.int32, device="cuda")
        B.metok_paged_attention_q4(q[:1], loud, loud, one, torch.full((1,), n, dtype=torch.int32, device="cuda"), 0.1, softcap=20.0)
        got = call()
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
