"""Heads turned where one row has millions of them."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
def test_millions_of_heads_of_one_row(in_place):
    """All at once they are what they are a part at a time."""
    H, dh = 5_000_003, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((H, 1, dh), generator=g, device="cuda", dtype=torch.bfloat16)
    f = (1e4 ** (-torch.arange(0, dh, 2, dtype=torch.float64) / dh)).float().cuda()
    pos = torch.tensor([12345], dtype=torch.int32, device="cuda")
    turn = lambda x, out=None: B.metok_rotate_heads(x, None, f, pos, eps=1e-6, q_out=out)["q"]
    want = torch.cat([turn(q[h:h + (1 << 18)]) for h in range(0, H, 1 << 18)])
    got = turn(q, q if in_place else torch.full_like(q, 7.0))
    assert torch.equal(got, want)
    del q, want, got
    torch.cuda.empty_cache()
