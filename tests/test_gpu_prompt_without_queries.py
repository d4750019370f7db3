"""metok_prefill_attention of no queries over any number of keys."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv", [(2, 1), (28, 4), (40, 40)])
@pytest.mark.parametrize("n_k", [0, 1, 255, 256, 5000, 70000])
def test_no_queries(dtype, Hq, Hkv, n_k):
    q, k = torch.zeros((Hq, 0, 64), dtype=dtype, device="cuda"), torch.zeros((Hkv, n_k, 64), dtype=dtype, device="cuda")
    got = B.metok_prefill_attention(q, k, k, 0.125, with_lse=True)
    torch.cuda.synchronize()
    assert got["out"].shape == (Hq, 0, 64) and got["lse"].shape == (Hq, 0) and int(got["status"]) == 0
    docs = torch.tensor([0, 0, 0, 0], dtype=torch.int32, device="cuda")
    keys = torch.tensor([0, n_k // 2, n_k // 2, n_k], dtype=torch.int32, device="cuda")
    got = B.metok_prefill_attention(q, k, k, 0.125, seq_q=docs, seq_k=keys, with_lse=True)
    torch.cuda.synchronize()
    assert got["out"].shape == (Hq, 0, 64) and int(got["status"]) == 0
    docs[1] = 1                                        # offsets that leave the queries are told even so
    got = B.metok_prefill_attention(q, k, k, 0.125, seq_q=docs, seq_k=keys)
    torch.cuda.synchronize()
    assert int(got["status"]) == -1
