"""Norms of heads whose squares, or mean squares, fp32 does not hold; tolerances as in test_gpu_rotate.py."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

from .test_gpu_rotate import angles, check, freqs, projections

pytestmark = pytest.mark.gpu

# elements around 3 * size: squares of normal numbers, of the smallest ones, of none; numbers below the smallest normal ones
SIZES = [2.0 ** -40, 2.0 ** -48, 2.0 ** -63, 2.0 ** -75, 2.0 ** -100, 2.0 ** -130]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh", [(14, 2, 64), (5, 3, 128)])
@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-30, 1e-12])
def test_heads_of_small_elements(dtype, Hq, Hkv, dh, eps):
    """Rows of ordinary heads with a few of small elements among them."""
    n = 3 * len(SIZES)
    g, _, q, k = projections(n, Hq, Hkv, dh, dtype, seed=7)
    q, k = q.clone(), k.clone()
    for i, size in enumerate(SIZES):
        q[i % Hq, 3 * i] *= size
        q[(i + 1) % Hq, 3 * i + 1] *= size
        k[:, 3 * i + 1] *= size
    w = 1 + 0.3 * torch.randn(dh, generator=g, device="cuda")
    f = freqs(dh)
    got = B.metok_rotate_heads(q, k, f, eps=eps, q_weight=w, k_weight=w)
    ang = angles(f, None, None, n)
    eps = float(torch.tensor(eps, dtype=torch.float32))                # as the call takes it
    check(got["q"], q, ang, eps=eps, weight=w)
    check(got["k"], k, ang, eps=eps, weight=w)
