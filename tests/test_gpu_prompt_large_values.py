"""metok_prefill_attention (bf16): values of V near the largest that it takes, where the first keys taken weigh little and many follow.

Tolerances as in test_gpu_prompt_attention.py."""

import pytest
import torch

from . import test_gpu_prompt_attention as Q

pytestmark = pytest.mark.gpu


def keys(n, low, below, dtype):
    """K whose logits with q = 8 in the first element, scale 1/8, are 0, or -below where `low`."""
    k = torch.zeros((1, n, 64), device="cuda")
    k[0, :, 0] = torch.where(low, -below, 0.0)
    return k.to(dtype)


def queries(heads, n, dtype):
    q = torch.zeros((heads, n, 64), device="cuda")
    q[:, :, 0] = 8.0
    return q.to(dtype)


def values(n, g):
    return (1.2e30 + 2.0e28 * torch.randn((1, n, 64), generator=g, device="cuda")).to(torch.bfloat16)      # below 2^100


@pytest.mark.parametrize("below", [5.0, 12.375, 40.0])
@pytest.mark.parametrize("n_q", [64, 200])
def test_sums_over_many_keys_stay_in_range(below, n_q):
    """The keys are taken from the last tile down: its first 64 are 17.85 octaves below all that follow (or 7, or 58)."""
    n = 2600
    i = torch.arange(n, device="cuda")
    last = (n - 1) // 128 * 128
    dt = torch.bfloat16
    for low in (i >= last, i >= n - 1000, (i // 64) % 2 == 0, (i // 64) % 2 == 1):
        k, v = keys(n, low, below, dt), values(n, Q.gen(3))
        Q.check(queries(2, n_q, dt), k, v, 0.125, causal=False)
        Q.check(queries(2, n_q, dt), k, v, 0.125)


@pytest.mark.parametrize("heads,n_q,n", [(28, 64, 2304), (28, 64, 18496), (7, 3, 18496)])
def test_parts_of_cut_keys_stay_in_range(heads, n_q, n):
    """Few rows over many keys: every part's first group of keys weighs little."""
    i = torch.arange(n, device="cuda")
    dt = torch.bfloat16
    for low in ((i // 64) % 2 == 0, (i // 128) % 8 == 7):
        Q.check(queries(heads, n_q, dt), keys(n, low, 12.375, dt), values(n, Q.gen(4)), 0.125, causal=False)


@pytest.mark.parametrize("dtype", Q.TYPES)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n_q,n_k", [(400, 400), (7, 5000)])
def test_outputs_of_large_logits(dtype, dh, n_q, n_k):
    """Logits of hundreds: nearly all weight on one row, found anywhere among the keys."""
    g = Q.gen(13)
    q, k, v = Q.rows(g, 2, n_q, dh, dtype, 60.0), Q.rows(g, 1, n_k, dh, dtype), Q.rows(g, 1, n_k, dh, dtype)
    Q.check(q, k, v, 1.0)
    Q.check(q, k, v, 1.0, causal=False)
    Q.check(q, k, v, 1.0, softcap=300.0)
