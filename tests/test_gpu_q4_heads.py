"""Attention over a cache held in 4 bits: as many heads as there may be, and a bias by the rows' own indices; reference and bounds of
test_gpu_q4_long_lines.py."""

import pytest
import torch

from paper_2506_02850_b200 import binding as B

from .test_gpu_q4 import HALF
from .test_gpu_q4_long_lines import STEP, Codes, check, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh", [(2048, 1, 64), (2048, 2048, 64), (2047, 89, 128), (17, 1, 128), (15, 1, 64), (8, 1, 128), (10, 10, 128)])
@pytest.mark.parametrize("bent", [False, True])
def test_head_counts(dtype, Hq, Hkv, dh, bent):
    check(Codes([150, 0, 33], Hkv, dh, 64, seed=Hq, growth=1), Hq, dtype, bent, True, bad=2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv", [(6, 2), (12, 1)])
def test_bias_by_indices_and_positions_without_a_bias(dtype, Hq, Hkv):
    c = Codes([500, 1, 77], Hkv, 64, 32, seed=3)
    q = torch.randn((3, Hq, 64), generator=c.g, device="cuda").to(dtype)
    slopes = torch.rand(Hq, generator=c.g, device="cuda") * 0.05
    slopes[0], slopes[1] = -0.01, 0.0                                # farther rows may count for more
    call = lambda **kw: B.metok_paged_attention_q4(q, c.k, c.v, c.block_table, c.kv_len, 0.125, with_lse=True, **kw)
    got, plain, same = call(slopes=slopes), call(), call(positions=c.positions)
    torch.cuda.synchronize()
    assert torch.equal(plain["out"], same["out"]) and torch.equal(plain["lse"], same["lse"])
    index = torch.arange(c.S_cap, dtype=torch.int32, device="cuda").repeat(3, 1)
    for b, n in enumerate(c.lens):
        (out, lse, _), (out_err, lse_err, _), absv, most = reference(c, q, 0.125, 0.0, slopes, index, b)
        tol = out_err + HALF[dtype] * out.abs() + 2.0 ** -22 * absv + 2.0 ** -37 * n * most
        assert bool(((got["out"][b].double() - out).abs() <= tol).all()) and bool(((got["lse"][b].double() - lse).abs() <= lse_err + STEP * lse.abs()).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,dh,n_seqs", [(28, 4, 128, 3), (28, 4, 128, 20), (12, 1, 64, 70), (5, 5, 64, 2)])
@pytest.mark.parametrize("cap", [0.0, 8.0])
def test_outputs_do_not_depend_on_weights_or_lse(dtype, Hq, Hkv, dh, n_seqs, cap):
    c = Codes([3000 // n_seqs + 37 * b for b in range(n_seqs)], Hkv, dh, 16, seed=4, growth=1)
    q = torch.randn((n_seqs, Hq, dh), generator=c.g, device="cuda").to(dtype)
    call = lambda mass, lse: B.metok_paged_attention_q4(q, c.k, c.v, c.block_table, c.kv_len, 0.1, softcap=cap, mass=mass, with_lse=lse)
    want, weighed, bare = call(None, True), call(c.mass.clone(), True), call(c.mass.clone(), False)
    torch.cuda.synchronize()
    assert torch.equal(weighed["out"], want["out"]) and torch.equal(weighed["lse"], want["lse"])
    assert torch.equal(bare["out"], want["out"]) and "lse" not in bare
