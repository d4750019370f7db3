"""Attention over what the compression leaves, and the paged cache that it reads: workloads and plain forms.

Four kinds of case, in the order in which a program that answers questions about a video uses them:

  prefill  attention of a prompt's rows (`metok_prefill_attention`): packed documents, causal or with a
           prefix (the video) that every row sees, scores capped by a tanh, a bias by the distance of the
           rows' original positions (pruning leaves gaps between them);
  append   new K/V rows into a paged cache (`metok_paged_append`): a whole prompt, or a row per sequence;
  decode   attention of one new token per sequence over the paged cache (`metok_paged_attention`), adding
           every row's attention weight to its account;
  evict    the rows with the least accumulated weight leave the cache (`metok_paged_evict`), all layers
           and sequences in one call.

Head shapes and lengths are those of the decoders and videos in `workloads.py`; `draw` covers the ranges
between them.  The plain forms are elementary torch operations in 32 bits; `exact` computes the same in 64
bits, sequence by sequence, from the definitions.
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}

# query heads, K/V heads, head size
DECODERS = {"one": (1, 1, 64), "small": (14, 2, 64), "base": (28, 4, 128), "large": (40, 40, 128)}


def _prefill(decoder, docs, n_k, n_q=0, prefix=0.0, cap=0.0, bias=False, causal=True, gaps=False, dtype="bf16", lens=1):
    """n_k keys in `docs` documents; n_q queries (0: as many as keys) are the documents' last rows."""
    return {"kind": "prefill", "decoder": decoder, "docs": docs, "n_k": n_k, "n_q": n_q, "prefix": prefix, "cap": cap, "bias": bias,
            "causal": causal, "gaps": gaps, "dtype": dtype, "lens": lens}


def _append(decoder, B, rows, page, cached, dtype="bf16", lens=1):
    """Up to `rows` new rows for each of B sequences that hold up to `cached` rows."""
    return {"kind": "append", "decoder": decoder, "B": B, "rows": rows, "page": page, "cached": cached, "dtype": dtype, "lens": lens}


def _decode(decoder, B, longest, page, cap=0.0, bias=False, mass=True, dtype="bf16", lens=1):
    return {"kind": "decode", "decoder": decoder, "B": B, "longest": longest, "page": page, "cap": cap, "bias": bias, "mass": mass,
            "dtype": dtype, "lens": lens}


def _evict(decoder, layers, B, longest, page, budget, sink, recent, dtype="bf16", lens=1):
    return {"kind": "evict", "decoder": decoder, "layers": layers, "B": B, "longest": longest, "page": page, "budget": budget,
            "sink": sink, "recent": recent, "dtype": dtype, "lens": lens}


def listed():
    return [
        # the smallest model's prompt in fp32, cap and all: launches and latency
        dict(_prefill("one", 1, 132, prefix=0.9, cap=30.0, dtype="f32"), name="prefill_132_f32"),
        # a video of 32 frames, of which every row sees all, and a question
        dict(_prefill("base", 1, 4624, prefix=0.9966), name="prefill_4624_prefix"),
        # prompts of several users packed into one batch, scores capped
        dict(_prefill("small", 9, 7001, cap=30.0), name="prefill_packed_cap"),
        # a chunk of a long prompt whose video was pruned: distances go by the rows' original positions
        dict(_prefill("base", 1, 18496, n_q=1999, bias=True, gaps=True), name="prefill_chunk_bias"),
        # a second question about a video that is in the cache: few rows, many keys
        dict(_prefill("base", 1, 18496, n_q=64), name="prefill_question"),
        # a new row for each sequence of a running batch
        dict(_append("base", 16, 1, 16, 9000), name="append_step"),
        # the prompts of four videos of 128 frames go into the cache
        dict(_append("base", 4, 18496, 64, 0), name="append_prompts"),
        # one long video, nothing removed from its cache
        dict(_decode("base", 1, 18496, 64), name="decode_one_long"),
        # a batch of conversations of different lengths, scores capped
        dict(_decode("base", 48, 9001, 16, cap=50.0, mass=False), name="decode_batch_cap"),
        # the small decoder in fp32, bias by distance
        dict(_decode("small", 5, 1263, 32, bias=True, dtype="f32"), name="decode_small_f32"),
        # the caches of four videos shrink once, after the prompt
        dict(_evict("base", 28, 4, 4736, 64, 1263, 16, 128), name="evict_28_layers"),
        # a running conversation loses what the last rows added
        dict(_evict("small", 6, 3, 1391, 16, 1263, 4, 64), name="evict_steady"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prefill", "prefill", "append", "decode", "decode", "evict"])
    decoder = rng.choice(["small", "base", "large"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    lens = rng.randrange(1 << 20)
    if kind == "prefill":
        Hq, _, dh = DECODERS[decoder]
        n_k = _log_int(rng, 40, 18000 if dtype == "bf16" else 4000)
        # pairs of rows within the largest listed case's work
        most = int(min(n_k, 28 * 128 * 1999 * 18496 / (Hq * dh * n_k) * (1.0 if dtype == "bf16" else 0.1)))
        n_q = _log_int(rng, 1, most)
        docs = _log_int(rng, 1, max(1, min(16, n_q // 4, n_k // 20)))
        return _prefill(decoder, docs, n_k, 0 if n_q == n_k else n_q, prefix=rng.choice([0.0, 0.0, rng.uniform(0.1, 0.98)]),
                        cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.4, causal=rng.random() < 0.85,
                        gaps=rng.random() < 0.5, dtype=dtype, lens=lens)
    page = rng.choice([16, 32, 64, 128])
    heads = DECODERS[decoder][1] * DECODERS[decoder][2] * BYTES[dtype]
    if kind == "append":
        B = _log_int(rng, 1, 40)
        rows = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, min(18496, 4 * 18496 * 1024 // heads // B)))
        return _append(decoder, B, rows, page, _log_int(rng, 1, 4000), dtype=dtype, lens=lens)
    B = _log_int(rng, 1, 48)
    if kind == "decode":
        longest = _log_int(rng, 20, max(40, min(18496, 48 * 9001 * 1024 // heads // B)))
        return _decode(decoder, B, longest, page, cap=rng.choice([0.0, 0.0, 30.0, 50.0]), bias=rng.random() < 0.4,
                       mass=rng.random() < 0.6, dtype=dtype, lens=lens)
    layers = _log_int(rng, 1, 28)
    B = min(B, 12)
    longest = _log_int(rng, 40, max(80, min(9000, 28 * 4 * 4736 * 1024 // heads // (B * layers))))
    budget = max(8, int(longest * rng.uniform(0.1, 0.95)))
    return _evict(decoder, layers, B, longest, page, budget, rng.randrange(0, max(1, min(17, budget // 4))),
                  rng.randrange(1, max(2, budget // 4)), dtype=dtype, lens=lens)


# --------------------------------------------------------------------------- sizes


def _split(rng, total, parts):
    """`parts` positive sizes that add up to `total`."""
    cut = sorted(rng.sample(range(1, total), parts - 1)) if parts > 1 else []
    return [b - a for a, b in zip([0] + cut, cut + [total])]


def _doc_lens(case):
    """Keys and queries of each document."""
    rng = random.Random(case["lens"])
    lk = _split(rng, case["n_k"], case["docs"])
    if not case["n_q"]:
        return lk, list(lk)
    lq = [0] * len(lk)                                   # shares in proportion, none above its document's keys
    left = case["n_q"]
    for d, n in enumerate(lk):
        lq[d] = min(n, case["n_q"] * n // case["n_k"])
        left -= lq[d]
    for d, n in enumerate(lk):
        more = min(left, n - lq[d])
        lq[d] += more
        left -= more
    return lk, lq


def _prefix(case, lk):
    return [int(case["prefix"] * n) for n in lk]


def _seq_lens(case):
    """Rows of each sequence: the first has `longest`, the others between a quarter of it and all."""
    rng = random.Random(case["lens"])
    n = case["longest"]
    return [n] + [rng.randint(max(1, n // 4), n) for _ in range(case["B"] - 1)]


def _append_lens(case):
    rng = random.Random(case["lens"])
    n = case["rows"]
    new = [n] + [rng.randint((n + 1) // 2, n) for _ in range(case["B"] - 1)]
    return new, [rng.randint(0, case["cached"]) for _ in new]


def _pages(total_rows, page):
    return (total_rows + page - 1) // page


# --------------------------------------------------------------------------- inputs


def _slopes(Hq, dev):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32, device=dev)


def _positions(n, gaps, g, dev):
    """Ascending positions; `gaps`: about half of the rows in between were pruned."""
    step = torch.randint(1, 4, (n,), generator=g, device=dev, dtype=torch.int32) if gaps else torch.ones(n, dtype=torch.int32, device=dev)
    return (torch.cumsum(step, 0) - step[0]).to(torch.int32)


def _i32(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _table(B, max_pages, n_pages, g, dev):
    """Pages of the sequences, in no order: the first n_pages entries of a permutation."""
    return torch.randperm(n_pages, generator=g, device=dev)[: B * max_pages].to(torch.int32).view(B, max_pages)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 17)
    Hq, Hkv, dh = DECODERS[case["decoder"]]
    dt = DTYPES[case["dtype"]]
    s = dict(case, scale=dh ** -0.5)

    def randn(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device=dev) * scale).to(dt)

    if case["kind"] == "prefill":
        lk, lq = _doc_lens(case)
        # logits of deviation 1; where they are capped they are large enough to feel it
        q = randn(Hq, sum(lq), dh, scale=6.0 if case["cap"] else 1.0)
        s.update(q=q, k=randn(Hkv, sum(lk), dh), v=randn(Hkv, sum(lk), dh),
                 seq_q=_i32(np.concatenate([[0], np.cumsum(lq)]), dev), seq_k=_i32(np.concatenate([[0], np.cumsum(lk)]), dev),
                 prefix_len=_i32(_prefix(case, lk), dev) if case["prefix"] else None, slopes=_slopes(Hq, dev) if case["bias"] else None,
                 positions=torch.cat([_positions(n, case["gaps"], g, dev) for n in lk]) if case["bias"] else None)
        return s

    B, page = case["B"], case["page"]
    if case["kind"] == "append":
        new, old = _append_lens(case)
        total = sum(new)
        most = max(a + b for a, b in zip(new, old))
    else:
        lens = _seq_lens(case)
        most = max(lens) + 1
    max_pages = _pages(most, page)
    n_pages = B * max_pages + 3
    S_cap = max_pages * page
    s.update(block_table=_table(B, max_pages, n_pages, g, dev))
    if case["kind"] == "append":
        # the projections of the layer lie token by token
        s.update(k_new=randn(total, Hkv, dh).transpose(0, 1), v_new=randn(total, Hkv, dh).transpose(0, 1),
                 k_pool=randn(n_pages, Hkv, page, dh), v_pool=randn(n_pages, Hkv, page, dh), kv_len=_i32(old, dev),
                 new_offsets=_i32(np.concatenate([[0], np.cumsum(new)]), dev),
                 positions=torch.arange(S_cap, dtype=torch.int32, device=dev).repeat(B, 1), mass=torch.rand((B, S_cap), generator=g, device=dev),
                 pos_new=torch.cat([_positions(n, True, g, dev) + o for n, o in zip(new, old)]),
                 mass_new=torch.rand((total,), generator=g, device=dev))
        return s
    if case["kind"] == "decode":
        s.update(q=randn(B, Hq, dh, scale=6.0 if case["cap"] else 1.0), k_pool=randn(n_pages, Hkv, page, dh),
                 v_pool=randn(n_pages, Hkv, page, dh), kv_len=_i32(lens, dev), slopes=_slopes(Hq, dev) if case["bias"] else None,
                 positions=torch.stack([_positions(S_cap, True, g, dev) for _ in range(B)]) if case["bias"] else None,
                 mass=torch.rand((B, S_cap), generator=g, device=dev) * 1e-3 if case["mass"] else None)
        return s
    L = case["layers"]
    k_pool, v_pool = randn(L, n_pages, Hkv, page, dh), randn(L, n_pages, Hkv, page, dh)
    # weights fall off steeply, and rows that nobody has looked at yet have none
    mass0 = torch.randn((L, B, S_cap), generator=g, device=dev).mul_(2.0).exp_()
    mass0 *= torch.rand((L, B, S_cap), generator=g, device=dev) > 0.02
    # an earlier eviction has left the rows in another order than that of their positions, but for the newest
    pos0 = torch.arange(S_cap, dtype=torch.int32, device=dev).repeat(L, B, 1)
    third = max(1, min(lens) // 3)
    pos0[:, :, :third] = torch.rand((L, B, third), generator=g, device=dev).argsort(dim=-1).to(torch.int32)
    s.update(k_pool=k_pool, v_pool=v_pool, k_layers=list(k_pool.unbind(0)), v_layers=list(v_pool.unbind(0)), kv_len=_i32(lens, dev),
             mass0=mass0, pos0=pos0, mass=mass0.clone(), positions=pos0.clone())
    return s


# --------------------------------------------------------------------------- plain forms


def _plain_prefill(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    Hq, nq, dh = q.shape
    Hkv, nk, _ = k.shape
    dev = q.device
    sq, sk = s["seq_q"].long(), s["seq_k"].long()
    i, j = torch.arange(nq, device=dev), torch.arange(nk, device=dev)
    dq = torch.searchsorted(sq[1:], i, right=True)
    dk = torch.searchsorted(sk[1:], j, right=True)
    at = i - sq[1:][dq] + sk[1:][dq]                     # the key at which a query sits
    seen = dq[:, None] == dk[None, :]
    if s["causal"]:
        near = j[None, :] <= at[:, None]
        if s["prefix_len"] is not None:
            near = near | (j - sk[:-1][dk] < s["prefix_len"].long()[dk])[None, :]
        seen = seen & near
    x = torch.matmul(q.view(Hkv, Hq // Hkv * nq, dh), k.transpose(1, 2)).view(Hkv, Hq // Hkv, nq, nk).mul_(s["scale"])
    if s["cap"]:
        x = x.div_(s["cap"]).tanh_().mul_(s["cap"])
    if s["slopes"] is not None:
        far = (s["positions"].long()[at][:, None] - s["positions"].long()[None, :]).abs().float()
        x = x.sub_(s["slopes"].view(Hkv, Hq // Hkv, 1, 1) * far)
    x = x.masked_fill_(~seen, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = x.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p.view(Hkv, Hq // Hkv * nq, nk), v).view(Hkv, Hq // Hkv, nq, dh) / torch.where(total > 0, total, torch.ones_like(total))
    lse = total.log() + top
    return {"out": out.view(Hq, nq, dh).to(s["q"].dtype), "lse": lse.view(Hq, nq)}


def _slot(s, seq, row):
    """Page and offset of the rows `row` of the sequences `seq`."""
    page = s["page"]
    return s["block_table"].long()[seq, row // page], row % page


def _plain_append(s):
    off, old = s["new_offsets"].long(), s["kv_len"].long()
    i = torch.arange(s["k_new"].shape[1], device=off.device)
    seq = torch.searchsorted(off[1:], i, right=True)
    row = old[seq] + i - off[seq]
    page, at = _slot(s, seq, row)
    s["k_pool"][page, :, at] = s["k_new"].transpose(0, 1)
    s["v_pool"][page, :, at] = s["v_new"].transpose(0, 1)
    s["positions"][seq, row] = s["pos_new"]
    s["mass"][seq, row] = s["mass_new"]
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "positions": s["positions"], "mass": s["mass"],
            "new_len": (old + off[1:] - off[:-1]).int()}


def _plain_decode(s):
    q = s["q"].float()
    B, Hq, dh = q.shape
    n_pages, Hkv, page, _ = s["k_pool"].shape
    S_cap = s["block_table"].shape[1] * page
    table = s["block_table"].long()
    k = s["k_pool"][table].transpose(1, 2).reshape(B, Hkv, S_cap, dh).float()
    v = s["v_pool"][table].transpose(1, 2).reshape(B, Hkv, S_cap, dh).float()
    x = torch.matmul(q.view(B, Hkv, Hq // Hkv, dh), k.transpose(2, 3)).mul_(s["scale"])
    if s["cap"]:
        x = x.div_(s["cap"]).tanh_().mul_(s["cap"])
    n = s["kv_len"].long()
    if s["slopes"] is not None:
        pos = s["positions"].long()
        far = (pos.gather(1, n[:, None] - 1) - pos).abs().float()
        x = x.sub_(s["slopes"].view(1, Hkv, Hq // Hkv, 1) * far[:, None, None, :])
    seen = torch.arange(S_cap, device=q.device)[None, :] < n[:, None]
    x = x.masked_fill_(~seen[:, None, None, :], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    p = p.div_(total)
    out = torch.matmul(p, v).view(B, Hq, dh).to(s["q"].dtype)
    res = {"out": out, "lse": (total.log() + top).view(B, Hq)}
    if s["mass"] is not None:
        s["mass"].add_(p.view(B, Hq, S_cap).sum(dim=1) / Hq)
        res["mass"] = s["mass"]
    return res


def _plain_evict(s):
    mass, pos = s["mass"], s["positions"]
    mass.copy_(s["mass0"])
    pos.copy_(s["pos0"])
    L, B, S_cap = mass.shape
    dev = mass.device
    n = s["kv_len"].long()
    kept = torch.clamp(n, max=s["budget"])
    row = torch.arange(S_cap, device=dev)
    newest = pos.gather(2, (n - 1).view(1, B, 1).expand(L, B, 1))
    safe = (pos < s["sink"]) | (pos > newest - s["recent"])
    # weights are not negative: their bits are in their order; a lower row goes first among equals
    rank = (mass + 0.0).view(torch.int32).long()
    rank = torch.where(safe, torch.full_like(rank, (1 << 31) - 1), rank)
    key = (rank << 24) + ((1 << 24) - 1 - row)
    key = torch.where(row < n[:, None], key, torch.full_like(key, -1))
    order = key.argsort(dim=2, descending=True)
    keep = torch.zeros((L, B, S_cap), dtype=torch.bool, device=dev)
    keep.scatter_(2, order, (row < kept[:, None]).expand(L, B, S_cap))
    low = row < kept[:, None]                            # rows of the new cache
    hole, mover = low & ~keep, ~low & keep
    nth_hole, nth_mover = hole.long().cumsum(2) - 1, mover.long().cumsum(2) - 1
    movers = torch.zeros((L, B, S_cap + 1), dtype=torch.long, device=dev)
    movers.scatter_(2, torch.where(mover, nth_mover, torch.full_like(nth_mover, S_cap)), row.expand(L, B, S_cap).contiguous())
    src = torch.where(hole, movers.gather(2, nth_hole.clamp(min=0)), row.expand(L, B, S_cap))[:, :, : s["budget"]]
    there = low[:, : s["budget"]].expand(L, B, s["budget"])
    first = src[:, :, :1].expand_as(src)
    src = torch.where(there, src, first)
    dst = torch.where(there, row[: s["budget"]].expand_as(src), torch.zeros_like(src))
    seq = torch.arange(B, device=dev).view(1, B, 1).expand_as(src)
    layer = torch.arange(L, device=dev).view(L, 1, 1).expand_as(src)
    (p0, a0), (p1, a1) = _slot(s, seq, src), _slot(s, seq, dst)
    for pool in (s["k_pool"], s["v_pool"]):
        pool[layer, p1, :, a1] = pool[layer, p0, :, a0]
    new_mass, new_pos = mass.gather(2, src), pos.gather(2, src)
    mass.masked_fill_((row < n[:, None]).expand(L, B, S_cap), 0.0)
    mass.scatter_(2, dst, new_mass)
    pos.scatter_(2, dst, new_pos)
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "mass": mass, "positions": pos,
            "keep_idx": torch.where(there, src, torch.full_like(src, -1)).int(), "new_len": kept.int()}


def run(state):
    s = state
    if not own:
        return {"prefill": _plain_prefill, "append": _plain_append, "decode": _plain_decode, "evict": _plain_evict}[s["kind"]](s)
    from paper_2506_02850_b200 import binding as B
    if s["kind"] == "prefill":
        r = B.metok_prefill_attention(s["q"], s["k"], s["v"], s["scale"], seq_q=s["seq_q"], seq_k=s["seq_k"], prefix_len=s["prefix_len"],
                                      causal=s["causal"], softcap=s["cap"], slopes=s["slopes"], positions=s["positions"], with_lse=True)
        return {"out": r["out"], "lse": r["lse"]}
    if s["kind"] == "append":
        r = B.metok_paged_append(s["k_new"], s["v_new"], s["k_pool"], s["v_pool"], s["block_table"], s["kv_len"],
                                 new_offsets=s["new_offsets"], positions=s["positions"], pos_new=s["pos_new"], mass=s["mass"],
                                 mass_new=s["mass_new"])
        return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "positions": s["positions"], "mass": s["mass"], "new_len": r["new_len"]}
    if s["kind"] == "decode":
        r = B.metok_paged_attention(s["q"], s["k_pool"], s["v_pool"], s["block_table"], s["kv_len"], s["scale"], softcap=s["cap"],
                                    slopes=s["slopes"], positions=s["positions"], mass=s["mass"], with_lse=True)
        res = {"out": r["out"], "lse": r["lse"]}
        if s["mass"] is not None:
            res["mass"] = s["mass"]
        return res
    s["mass"].copy_(s["mass0"])
    s["positions"].copy_(s["pos0"])
    r = B.metok_paged_evict(s["k_layers"], s["v_layers"], s["block_table"], s["kv_len"], s["mass"], s["positions"], s["budget"], s["sink"],
                            s["recent"])
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "mass": s["mass"], "positions": s["positions"], "keep_idx": r["keep_idx"],
            "new_len": r["new_len"]}


# --------------------------------------------------------------------------- work


def _pairs(case):
    """Pairs of a query and a key that it sees."""
    lk, lq = _doc_lens(case)
    total = 0
    for nk, nq, prefix in zip(lk, lq, _prefix(case, lk)):
        if not case["causal"]:
            total += nq * nk
            continue
        first = nk - nq                                  # the key of the first query; query i sees max(first + i + 1, prefix)
        flat = min(nq, max(0, prefix - first))           # queries that see the prefix and no more
        rest = nq - flat
        total += flat * prefix + rest * (first + flat + 1) + rest * (rest - 1) // 2
    return total


def work(case):
    Hq, Hkv, dh = DECODERS[case["decoder"]]
    e = BYTES[case["dtype"]]
    if case["kind"] == "prefill":
        lk, lq = _doc_lens(case)
        nq, nk = sum(lq), sum(lk)
        return {"bytes": (2 * Hq * nq + 2 * Hkv * nk) * dh * e + 4 * Hq * nq + (4 * nk if case["bias"] else 0), "flops": 4 * dh * Hq * _pairs(case)}
    row = 2 * Hkv * dh * e                               # K and V
    if case["kind"] == "append":
        n = sum(_append_lens(case)[0])
        return {"bytes": n * (2 * row + 16), "flops": 0}
    lens = _seq_lens(case)
    n = sum(lens)
    tables = 4 * sum(_pages(m, case["page"]) for m in lens)
    if case["kind"] == "decode":
        return {"bytes": n * (row + (8 if case["mass"] else 0) + (4 if case["bias"] else 0)) + 2 * case["B"] * Hq * dh * e + tables,
                "flops": 4 * dh * Hq * n}
    moved = kept = 0.0
    for m in lens:
        n_new = min(m, case["budget"])
        kept += n_new
        if m > n_new:                                    # the newest rows lie at the end; the others are kept from everywhere
            safe = min(n_new, case["recent"])
            moved += min(safe, m - n_new) + (n_new - safe) * max(0, m - n_new - safe) / max(1, m - safe)
    return {"bytes": case["layers"] * (8 * n + 4 * kept + moved * (2 * row + 16) + 4 * (n - kept)) + tables, "flops": 0}


# --------------------------------------------------------------------------- the definitions, in 64 bits


def _logits(s, q, k, slopes, far):
    x = torch.matmul(q.double(), k.double().T) * s["scale"]
    if s["cap"]:
        x = s["cap"] * torch.tanh(x / s["cap"])
    if slopes is not None:
        x = x - float(slopes) * far
    return x


def _exact_prefill(s):
    Hq, nq, dh = s["q"].shape
    rep = Hq // s["k"].shape[0]
    out = torch.zeros((Hq, nq, dh), dtype=torch.float64, device="cuda")
    lse = torch.full((Hq, nq), -math.inf, dtype=torch.float64, device="cuda")
    lk, lq = _doc_lens(s)
    prefix = _prefix(s, lk)
    q0 = k0 = 0
    for d, (nk_d, nq_d) in enumerate(zip(lk, lq)):
        for lo in range(0, nq_d, 2048):
            hi = min(nq_d, lo + 2048)
            at = torch.arange(lo, hi, device="cuda") + nk_d - nq_d
            key = torch.arange(nk_d, device="cuda")
            hidden = (key[None, :] > at[:, None]) & (key[None, :] >= (prefix[d] if s["prefix_len"] is not None else 0)) & bool(s["causal"])
            far = None
            if s["slopes"] is not None:
                pos = s["positions"][k0:k0 + nk_d].double()
                far = (pos[at][:, None] - pos[None, :]).abs()
            for h in range(Hq):
                x = _logits(s, s["q"][h, q0 + lo:q0 + hi], s["k"][h // rep, k0:k0 + nk_d], s["slopes"][h] if s["slopes"] is not None else None, far)
                x[hidden] = -math.inf
                lse[h, q0 + lo:q0 + hi] = torch.logsumexp(x, dim=1)
                out[h, q0 + lo:q0 + hi] = torch.softmax(x, dim=1) @ s["v"][h // rep, k0:k0 + nk_d].double()
        q0, k0 = q0 + nq_d, k0 + nk_d
    return {"out": out, "lse": lse}


def _exact_decode(s):
    B, Hq, dh = s["q"].shape
    Hkv = s["k_pool"].shape[1]
    out = torch.zeros((B, Hq, dh), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, Hq), dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if s["mass"] is not None else None
    for b, n in enumerate(_seq_lens(s)):
        pages = s["block_table"][b, : _pages(n, s["page"])].long()
        far = None
        if s["slopes"] is not None:
            pos = s["positions"][b, :n].double()
            far = (pos[n - 1] - pos).abs()[None, :]
        for h in range(Hq):
            k = s["k_pool"][pages, h * Hkv // Hq].reshape(-1, dh)[:n]
            v = s["v_pool"][pages, h * Hkv // Hq].reshape(-1, dh)[:n]
            x = _logits(s, s["q"][b, h:h + 1], k, s["slopes"][h] if s["slopes"] is not None else None, far)
            p = torch.softmax(x, dim=1)
            lse[b, h] = torch.logsumexp(x, dim=1)[0]
            out[b, h] = (p @ v.double())[0]
            if mass is not None:
                mass[b, :n] += p[0] / Hq
    return {"out": out, "lse": lse, "mass": mass}


def _exact_append(s):
    k_pool, v_pool, pos, mass = (s[x].clone() for x in ("k_pool", "v_pool", "positions", "mass"))
    new, old = _append_lens(s)
    i = 0
    for b, (n, o) in enumerate(zip(new, old)):
        done = 0
        while done < n:                                  # page by page
            page, at = int(s["block_table"][b, (o + done) // s["page"]]), (o + done) % s["page"]
            m = min(n - done, s["page"] - at)
            k_pool[page, :, at:at + m] = s["k_new"][:, i + done:i + done + m]
            v_pool[page, :, at:at + m] = s["v_new"][:, i + done:i + done + m]
            done += m
        pos[b, o:o + n] = s["pos_new"][i:i + n]
        mass[b, o:o + n] = s["mass_new"][i:i + n]
        i += n
    return {"k_pool": k_pool, "v_pool": v_pool, "positions": pos, "mass": mass.double(),
            "new_len": _i32([a + b for a, b in zip(new, old)], "cuda")}


def _exact_evict(s):
    lens, budget, page = _seq_lens(s), s["budget"], s["page"]
    mass, pos, table = s["mass0"].cpu().numpy().astype(np.float64), s["pos0"].cpu().numpy(), s["block_table"].cpu().numpy()
    L, B, _ = mass.shape
    keep_idx = np.full((L, B, budget), -1, dtype=np.int32)
    k_pool, v_pool = s["k_pool"].clone(), s["v_pool"].clone()
    for layer in range(L):
        for b, n in enumerate(lens):
            m, p = mass[layer, b, :n].copy(), pos[layer, b, :n].copy()
            safe = (p < s["sink"]) | (p > p[-1] - s["recent"])
            order = np.lexsort((np.arange(n), -m, ~safe))
            left = min(n, budget)
            kept = np.sort(order[:left])
            row = np.arange(left)
            row[np.setdiff1d(row, kept)] = kept[kept >= left]
            keep_idx[layer, b, :left] = row
            mass[layer, b, :n] = 0.0
            mass[layer, b, :left] = m[row]
            pos[layer, b, :left] = p[row]
            moved = np.nonzero(row != np.arange(left))[0]
            src, dst = (torch.from_numpy(x).cuda() for x in (row[moved], moved))
            t = torch.from_numpy(table[b]).cuda().long()
            for pool in (k_pool[layer], v_pool[layer]):
                pool[t[dst // page], :, dst % page] = pool[t[src // page], :, src % page]
    return {"k_pool": k_pool, "v_pool": v_pool, "mass": torch.from_numpy(mass), "positions": torch.from_numpy(pos),
            "keep_idx": torch.from_numpy(keep_idx), "new_len": torch.tensor([min(n, budget) for n in lens], dtype=torch.int32)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"prefill": _exact_prefill, "append": _exact_append, "decode": _exact_decode, "evict": _exact_evict}[case["kind"]](s)
