"""Attention over a cache held in 4 bits: how exactly weights enter the product with V.

Two rows whose weights are nearly equal and whose V are opposite leave a small output, in which what a rounded weight is off shows.  The logits
have one product each, so the oracle's bounds on fp32 arithmetic are small; a weight as two 11-bit numbers is off by 2^-11 * 2^-11 of itself."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

from .test_gpu_q4 import HALF, num

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh", [(4, 1, 64), (2, 2, 128), (12, 1, 128)])
@pytest.mark.parametrize("bent", [False, True])
def test_small_outputs_of_nearly_equal_weights(dtype, Hq, Hkv, dh, bent):
    n_seqs, page, scale = 40, 16, 0.25
    g = torch.Generator(device="cuda").manual_seed(Hq)
    K, V = B.q4_pool(n_seqs, Hkv, page, dh), B.q4_pool(n_seqs, Hkv, page, dh)
    table = torch.randperm(n_seqs, generator=g, device="cuda").to(torch.int32)[:, None].contiguous()
    off = (2 * torch.arange(n_seqs + 1, device="cuda")).to(torch.int32)
    k = torch.zeros((Hkv, 2 * n_seqs, dh), device="cuda")
    k[:, ::2, 5] = 1.0
    v = torch.randn((Hkv, n_seqs, dh), generator=g, device="cuda")
    v = torch.stack([v, -v], 2).view(Hkv, 2 * n_seqs, dh)
    length = B.metok_paged_append_q4(k, v, K, V, table, torch.zeros(n_seqs, dtype=torch.int32, device="cuda"), off)["new_len"]
    q = torch.zeros((n_seqs, Hq, dh), dtype=dtype, device="cuda")
    q[:, :, 5] = torch.rand((n_seqs, Hq), generator=g, device="cuda") * 0.2       # logits up to 0.05 apart
    got = B.metok_paged_attention_q4(q, K, V, table, length, scale, softcap=100.0 if bent else 0.0)
    torch.cuda.synchronize()
    assert int(got["status"]) == 0
    want = A.paged_attention(num(q), A.q4_pool_values(K.cpu().numpy()), A.q4_pool_values(V.cpu().numpy()), table.cpu().numpy(), [2] * n_seqs, scale)
    if bent:                                                        # 100 tanh(x / 100) of logits up to 0.05 is x but for (0.05 / 100)^2 / 3 = 8.4e-8 of 0.05
        want["out_err"] = want["out_err"] + (0.05 * 8.4e-8 + 8 * A.STEP * 0.05) * want["absv"]
    tol = want["out_err"] + HALF[dtype] * np.abs(want["out"]) + 2.0 ** -22 * want["absv"]
    assert (np.abs(num(got["out"]) - want["out"]) <= tol).all(), np.max(np.abs(num(got["out"]) - want["out"]) / np.maximum(tol, 1e-30))
