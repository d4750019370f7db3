"""The attention kernels in the debug library: a copy that never comes makes their waits run out; they unwind, report it, and the next
call is as ever (see test_debug_build.py)."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

from .test_debug_build import TIMEOUT, debug_lib  # noqa: F401  (a fixture)
from .test_gpu_paged import Cache

pytestmark = pytest.mark.gpu

PAGED_ATTN, PROMPT_ATTN = 32, 64


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wait_runs_out_over_a_paged_cache(debug_lib, dtype):  # noqa: F811
    c = Cache([70, 300, 5], 2, 64, 16, dtype, seed=1)
    q = torch.randn((3, 4, 64), generator=c.g, device="cuda").to(dtype)
    call = lambda: B.metok_paged_attention(q, c.k[0], c.v[0], c.block_table, c.kv_len, 0.125, with_lse=True)
    want = call()
    torch.cuda.synchronize()
    assert int(want["status"]) == 0
    assert debug_lib.metok_debug_set(1, PAGED_ATTN) == 0
    got = call()
    torch.cuda.synchronize()
    assert int(got["status"]) == TIMEOUT
    assert debug_lib.metok_debug_set(1, 0) == 0
    again = call()
    torch.cuda.synchronize()
    assert int(again["status"]) == 0 and torch.equal(again["out"], want["out"]) and torch.equal(again["lse"], want["lse"])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (9.0, True)])
def test_wait_runs_out_over_a_prompt(debug_lib, dh, cap, bias):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((h, 700, dh), generator=g, device="cuda").bfloat16() for h in (6, 2, 2))
    slopes = torch.full((6,), 0.01, device="cuda") if bias else None
    call = lambda: B.metok_prefill_attention(q, k, v, dh ** -0.5, softcap=cap, slopes=slopes, with_lse=True)
    want = call()
    torch.cuda.synchronize()
    assert int(want["status"]) == 0
    assert debug_lib.metok_debug_set(1, PROMPT_ATTN) == 0
    got = call()
    torch.cuda.synchronize()
    assert int(got["status"]) == TIMEOUT
    assert debug_lib.metok_debug_set(1, 0) == 0
    again = call()
    torch.cuda.synchronize()
    assert int(again["status"]) == 0 and torch.equal(again["out"], want["out"]) and torch.equal(again["lse"], want["lse"])
