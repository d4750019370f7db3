"""From a pruned prompt to its answer, as a program runs the calls one after another: pruning at a layer, compaction of its K/V cache,
attention of the survivors (by their original positions, the video as a prefix), the paged cache, decoding with accumulated weights,
eviction, decoding on.  Every step is compared with oracle/attention_oracle.py on a plain model of the cache."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2506_02850_b200 import binding as B

from .test_gpu_paged import HALF, num

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cap,bias", [(0.0, True), (15.0, False)])
def test_prune_attend_append_decode_evict(dtype, cap, bias):
    g = torch.Generator(device="cuda").manual_seed(3)
    Hq, Hkv, dh, n_vis, Lt, page = 14, 2, 64, 500, 12, 32
    S = n_vis + Lt
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    scale = dh ** -0.5
    slopes = torch.rand(Hq, generator=g, device="cuda") * 0.02 if bias else None
    kw = dict(softcap=cap, slopes=slopes)
    q_all, k, v = rand(Hq, S, dh), rand(Hkv, S + 8, dh), rand(Hkv, S + 8, dh)
    k_full, v_full = k.clone(), v.clone()
    group = (torch.rand(n_vis, generator=g, device="cuda") < 0.5).to(torch.int32)

    # a pruning level, and the layer's cache compacted by its keep list
    pruned = B.metok_prefill_prune(q_all[:, n_vis:].contiguous(), k[:, :S].contiguous(), None, 0, n_vis, group, [90, 47], scale)
    torch.cuda.synchronize()
    n = int(pruned["S_out"])
    keep = pruned["keep_idx"][:n].clone()
    assert n == 90 + 47 + Lt and int(pruned["status"]) == 0
    B.metok_kv_compact([k], [v], S, B.KV_GIVEN, 0, n_vis, keep_idx=pruned["keep_idx"][:S].view(1, S), keep_len=pruned["S_out"])

    # attention of the survivors: the video is a prefix, distances go by the original positions
    q = q_all[:, keep.long()]
    prefix = torch.tensor([n - Lt], dtype=torch.int32, device="cuda")
    got = B.metok_prefill_attention(q, k[:, :n], v[:, :n], scale, prefix_len=prefix, positions=keep, with_lse=True, **kw)
    torch.cuda.synchronize()
    ks, vs, pos = num(k_full[:, keep.long()]), num(v_full[:, keep.long()]), keep.cpu().numpy()
    want = A.prompt_attention(num(q), ks, vs, scale, prefix_len=[n - Lt], softcap=cap, slopes=None if slopes is None else num(slopes), positions=pos)
    round_p = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    assert (np.abs(num(got["out"]) - want["out"]) <= want["out_err"] + HALF[dtype] * np.abs(want["out"]) + round_p * want["absv"]).all()

    # the paged cache, with the pruning's scores as the rows' first weights
    max_pages = 16
    pools = [torch.full((20, Hkv, page, dh), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    table = torch.randperm(20, generator=g, device="cuda")[:max_pages].to(torch.int32).view(1, max_pages)
    positions = torch.zeros((1, max_pages * page), dtype=torch.int32, device="cuda")
    mass = torch.zeros((1, max_pages * page), device="cuda")
    first = torch.zeros(S, device="cuda")
    first[:n_vis] = pruned["scores"]
    kept_mass = first[keep.long()].contiguous()
    length = torch.zeros(1, dtype=torch.int32, device="cuda")
    new = B.metok_paged_append(k[:, :n], v[:, :n], *pools, table, length, torch.tensor([0, n], dtype=torch.int32, device="cuda"), positions, keep, mass,
                               kept_mass)
    length = new["new_len"]
    model = {"k": ks, "v": vs, "pos": pos.astype(np.int64), "mass": num(kept_mass)}

    def token(length):
        kn, vn, qn = rand(Hkv, 1, dh), rand(Hkv, 1, dh), rand(1, Hq, dh)
        length = B.metok_paged_append(kn, vn, *pools, table, length, positions=positions, mass=mass)["new_len"]
        r = B.metok_paged_attention(qn, *pools, table, length, scale, positions=positions, mass=mass, with_lse=True, **kw)
        torch.cuda.synchronize()
        model["k"], model["v"] = np.concatenate([model["k"], num(kn)], 1), np.concatenate([model["v"], num(vn)], 1)
        model["pos"], model["mass"] = np.append(model["pos"], model["pos"][-1] + 1), np.append(model["mass"], 0.0)
        m = model["k"].shape[1]
        assert length.tolist() == [m]
        pool = lambda x: np.pad(x, ((0, 0), (0, -m % page), (0, 0))).reshape(Hkv, -1, page, dh).transpose(1, 0, 2, 3)
        want = A.paged_attention(num(qn), pool(model["k"]), pool(model["v"]), np.arange((m + page - 1) // page)[None], [m], scale, cap,
                                 None if slopes is None else num(slopes), model["pos"][None])
        small = 2.0 ** -16 * want["absv"] if dtype == torch.bfloat16 else 0
        assert (np.abs(num(r["out"]) - want["out"]) <= want["out_err"] + HALF[dtype] * np.abs(want["out"]) + small).all()
        assert np.array_equal(positions[0, :m].cpu().numpy(), model["pos"])
        model["mass"] = model["mass"] + want["p"][0].mean(0)
        assert (np.abs(num(mass)[0, :m] - model["mass"]) <= 2.0 ** -13 * model["mass"] + 1e-7).all()
        return length

    for _ in range(5):
        length = token(length)
    # eviction by the weights as the device has them
    on_device = num(mass)[0]
    out = B.metok_paged_evict([pools[0]], [pools[1]], table, length, mass, positions, 100, 4, 8)
    torch.cuda.synchronize()
    rows = A.evict_rows(on_device, model["pos"], model["k"].shape[1], 100, 4, 8)
    assert out["keep_idx"][0, 0].tolist() == rows.tolist() and out["new_len"].tolist() == [100]
    model.update(k=model["k"][:, rows], v=model["v"][:, rows], pos=model["pos"][rows], mass=on_device[rows])
    # the newest row went to some hole: the next token's position is told
    length, newest = out["new_len"], int(model["pos"].max())
    assert int(positions[0, :100].max()) == newest
    kn, vn = rand(Hkv, 1, dh), rand(Hkv, 1, dh)
    length = B.metok_paged_append(kn, vn, *pools, table, length, positions=positions, pos_new=torch.tensor([newest + 1], dtype=torch.int32, device="cuda"),
                                  mass=mass)["new_len"]
    model["k"], model["v"] = np.concatenate([model["k"], num(kn)], 1), np.concatenate([model["v"], num(vn)], 1)
    model["pos"], model["mass"] = np.append(model["pos"], newest + 1), np.append(model["mass"], 0.0)
    for _ in range(3):
        length = token(length)


def test_a_token_over_the_cache_is_the_last_row_of_the_prompt():
    """The prompt's last row by both calls: the same numbers up to bf16's rounding of weights and outputs."""
    g = torch.Generator(device="cuda").manual_seed(8)
    n, page = 1000, 64
    q, k, v = (torch.randn((h, n, 128), generator=g, device="cuda").bfloat16() for h in (28, 4, 4))
    whole = B.metok_prefill_attention(q, k, v, 128 ** -0.5, with_lse=True)
    pools = [torch.zeros((20, 4, page, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.randperm(20, generator=g, device="cuda")[:16].to(torch.int32).view(1, 16)
    length = B.metok_paged_append(k, v, *pools, table, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    one = B.metok_paged_attention(q[:, -1].unsqueeze(0).contiguous(), *pools, table, length["new_len"], 128 ** -0.5, with_lse=True)
    torch.cuda.synchronize()
    a, b = whole["out"][:, -1].float(), one["out"][0].float()
    absv = (torch.softmax(torch.einsum("hd,hnd->hn", q[:, -1].double(), k.double().repeat_interleave(7, 0)) * 128 ** -0.5, -1).unsqueeze(1)
            @ v.double().abs().repeat_interleave(7, 0))[:, 0]
    assert ((a - b).abs() <= 2.0 ** -7 * a.abs() + 1.1 * 2.0 ** -8 * absv).all()
    assert (whole["lse"][:, -1] - one["lse"][0]).abs().max() < 1e-4
