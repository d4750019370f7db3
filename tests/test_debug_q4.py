"""The attention over a cache held in 4 bits in the debug library: a copy that never comes makes its wait run out; it unwinds, reports it, and the
next call is as ever (see test_debug_build.py)."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

from .test_debug_build import TIMEOUT, debug_lib  # noqa: F401  (a fixture)
from .test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dh", [64, 128])
def test_wait_runs_out(debug_lib, dtype, dh):  # noqa: F811
    c = Cache([70, 300, 5], 2, dh, 16, seed=1)
    q = torch.randn((3, 4, dh), generator=c.g, device="cuda").to(dtype)
    call = lambda: B.metok_paged_attention_q4(q, c.k[0], c.v[0], c.block_table, c.kv_len, 0.125, with_lse=True)
    want = call()
    torch.cuda.synchronize()
    assert int(want["status"]) == 0
    assert debug_lib.metok_debug_set(1, 32) == 0
    got = call()
    torch.cuda.synchronize()
    assert int(got["status"]) == TIMEOUT
    assert debug_lib.metok_debug_set(1, 0) == 0
    again = call()
    torch.cuda.synchronize()
    assert int(again["status"]) == 0 and torch.equal(again["out"], want["out"]) and torch.equal(again["lse"], want["lse"])
