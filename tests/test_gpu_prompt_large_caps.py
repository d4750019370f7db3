"""metok_prefill_attention with a cap far above most logits: rows whose logits pass it do not cost the others digits.

Tolerances: those of test_gpu_prompt_attention.py without the share that goes by the cap: an fp32 tanh is off by a few steps of its
own value, so a capped logit by 16 steps of itself."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

from . import test_gpu_prompt_attention as Q

pytestmark = pytest.mark.gpu


def expected(q, k, v, scale, cap):
    Hq, n_q, dh = q.shape
    G = Hq // k.shape[0]
    res = {n: np.zeros((Hq, n_q, dh)) for n in ("out", "err", "absv")}
    for h in range(Hq):
        x, err = A.logits(q[h], k[h // G], scale)          # (without a cap: no error that goes by it)
        x = cap * np.tanh(x / cap)
        err = err + 16 * A.STEP * np.abs(x)
        out, _, p, oe, _, _ = A.weigh(x, err, A.visible(n_q, k.shape[1]), v[h // G])
        res["out"][h], res["err"][h], res["absv"][h] = out, oe, p @ np.abs(v[h // G])
    return res


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("cap", [3.0, 200.0, 2.0e3, 1.0e5, 1.0e9, 1.0e37])
def test_rows_beside_one_that_passes_the_cap(dtype, dh, cap):
    g = Q.gen(dh)
    n = 300
    q, k, v = Q.rows(g, 2, n, dh, dtype, 2.0), Q.rows(g, 1, n, dh, dtype), Q.rows(g, 1, n, dh, dtype)
    far = torch.arange(n, device="cuda") % 37 == 5             # some rows of every warp
    q[:, far] *= 2.0 * cap
    got = B.metok_prefill_attention(q, k, v, dh ** -0.5, softcap=cap)["out"]
    torch.cuda.synchronize()
    assert torch.isfinite(got.float()).all()
    want = expected(Q.num(q), Q.num(k), Q.num(v), dh ** -0.5, cap)
    tol = want["err"] + Q.HALF[dtype] * np.abs(want["out"]) + (2.0 ** -8 * want["absv"] if dtype == torch.bfloat16 else 0)
    near = ~far.cpu().numpy()                                  # (those that pass it have errors of their own size)
    assert (np.abs(Q.num(got) - want["out"]) <= tol)[:, near].all()
