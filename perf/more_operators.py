"""From a layer's projections into a cache held in 4 bits, and attention over it: workloads and plain forms.

Four kinds of case, in the order in which a program that answers questions about a video uses them:

  rotate  the norm of each head of Q and K and the rotary positions of a video's rows (time, height and width axes), in
          one pass (`metok_rotate_heads`);
  append  new K/V rows into a paged cache of 4 bits (`metok_paged_append_q4`), and what they stand for there, read back
          (`metok_paged_read_q4`): the prompt's own attention may use the values that the tokens after it will see;
  read    all rows of the sequences out of such a cache, for the prompt attention of a next question
          (`metok_paged_read_q4`);
  decode  attention of one new token per sequence over that cache, adding every row's attention weight to its account
          (`metok_paged_attention_q4`).

The format: 16 neighbouring elements of a head's row share a scale S = 16 e, where e is the smallest number of type e5m2
(at most 56) with max |x| <= 7.5 S; an element is held as n = x / S, rounded to nearest even and held to [-7, 7], in a
nibble n + 8.  A pool is uint8 [n_pages][Hkv][page_size / 16][9 dh]: of 16 rows the codes [16][dh / 2] (element d in the
nibble d % 2 of byte d / 2, low one first), then the scales [16][dh / 16].

Head shapes and lengths are those of the decoders and videos in `workloads.py`; `draw` covers the ranges between them.
The plain forms are elementary torch operations in 32 bits (angles and codes in 64); `exact` computes the same in 64 bits from the
definitions.
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
DECODERS = {"small": (14, 2, 64), "base": (28, 4, 128), "large": (40, 40, 128)}


def _rotate(decoder, n, axes=3, turns=False, norm=True, part=1.0, interleaved=False, far=0, dtype="bf16"):
    """n rows; `axes` positions each, whose pairs of elements lie in sections or in turns; `part` of the elements turn; `far`: a position
    that the rows begin at."""
    return {"kind": "rotate", "decoder": decoder, "n": n, "axes": axes, "turns": turns, "norm": norm, "part": part,
            "interleaved": interleaved, "far": far, "dtype": dtype}


def _append(decoder, B, rows, page, cached, dtype="bf16", lens=1):
    """Up to `rows` new rows for each of B sequences that hold up to `cached` rows."""
    return {"kind": "append", "decoder": decoder, "B": B, "rows": rows, "page": page, "cached": cached, "dtype": dtype, "lens": lens}


def _read(decoder, B, longest, page, dtype="bf16", lens=1):
    return {"kind": "read", "decoder": decoder, "B": B, "longest": longest, "page": page, "dtype": dtype, "lens": lens}


def _decode(decoder, B, longest, page, cap=0.0, bias=False, mass=True, dtype="bf16", lens=1):
    return {"kind": "decode", "decoder": decoder, "B": B, "longest": longest, "page": page, "cap": cap, "bias": bias, "mass": mass,
            "dtype": dtype, "lens": lens}


def listed():
    return [
        # a token for each sequence of a running batch, on the way to its layer's cache: a launch
        dict(_rotate("base", 16, far=18496), name="rotate_step"),
        # the prompt of a video of 128 frames
        dict(_rotate("base", 18496), name="rotate_prompt"),
        # a pruned prompt of the small decoder in fp32: pairs side by side, half of the elements, far along a stream of videos
        dict(_rotate("small", 1263, turns=True, norm=False, part=0.5, interleaved=True, far=1 << 20, dtype="f32"), name="rotate_pruned_f32"),
        # a new row for each sequence of a running batch
        dict(_append("base", 16, 1, 16, 9000), name="append_step"),
        # the prompts of four videos of 128 frames go into the cache
        dict(_append("base", 4, 18496, 64, 0), name="append_prompts"),
        # short prompts of the small decoder in fp32
        dict(_append("small", 5, 333, 32, 100, dtype="f32"), name="append_short_f32"),
        # a second question about a video of 128 frames: its prompt attention wants the rows as they are
        dict(_read("base", 1, 18496, 64), name="read_video"),
        # several short conversations of the small decoder
        dict(_read("small", 7, 1263, 16, dtype="f32"), name="read_short_f32"),
        # one long video, nothing removed from its cache
        dict(_decode("base", 1, 18496, 64), name="decode_one_long"),
        # a batch of conversations of different lengths, scores capped
        dict(_decode("base", 48, 9001, 16, cap=50.0, mass=False), name="decode_batch_cap"),
        # heads that share nothing, distances
        dict(_decode("large", 3, 6313, 128, bias=True), name="decode_large_bias"),
        # the small decoder in fp32, bias by distance
        dict(_decode("small", 5, 1263, 32, bias=True, dtype="f32"), name="decode_small_f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "append", "read", "decode", "decode", "decode"])
    decoder = rng.choice(["small", "base", "large"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    lens = rng.randrange(1 << 20)
    Hq, Hkv, dh = DECODERS[decoder]
    if kind == "rotate":
        n = _log_int(rng, 1, 18496 * 32 * 128 * 2 // ((Hq + Hkv) * dh * BYTES[dtype]))
        return _rotate(decoder, n, axes=rng.choice([1, 3, 3]), turns=rng.random() < 0.4, norm=rng.random() < 0.6,
                       part=rng.choice([1.0, 1.0, 0.5, 0.25]), interleaved=rng.random() < 0.3,
                       far=rng.choice([0, 0, _log_int(rng, 100, 1 << 22)]), dtype=dtype)
    page = rng.choice([16, 32, 64, 128])
    heads = Hkv * dh
    B = _log_int(rng, 1, 48)
    if kind == "append":
        rows = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(2, min(18496, 4 * 18496 * 512 // (heads * BYTES[dtype] // 2) // B)))
        return _append(decoder, B, rows, page, _log_int(rng, 1, 4000), dtype=dtype, lens=lens)
    if kind == "read":
        longest = _log_int(rng, 20, max(40, min(18496, 18496 * 512 // (heads * BYTES[dtype] // 2) // B)))
        return _read(decoder, B, longest, page, dtype=dtype, lens=lens)
    longest = _log_int(rng, 20, max(40, min(18496, 48 * 9001 * 512 // heads // B)))
    return _decode(decoder, B, longest, page, cap=rng.choice([0.0, 0.0, 30.0, 50.0]), bias=rng.random() < 0.4,
                   mass=rng.random() < 0.6, dtype=dtype, lens=lens)


# --------------------------------------------------------------------------- sizes


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


def _rotary(case):
    """Elements of a head that turn, and the axis of each of their pairs."""
    dh = DECODERS[case["decoder"]][2]
    r = int(dh * case["part"])
    half = r // 2
    if case["axes"] == 1:
        return r, [0] * half
    if case["turns"]:
        return r, [i % 3 for i in range(half)]
    a, b = half // 4, half // 4 + (half - half // 4) // 2
    return r, [0 if i < a else 1 if i < b else 2 for i in range(half)]


# --------------------------------------------------------------------------- the format, plain


def _pack(x):
    """Codes (uint8 [..., dh / 2]) and scales (uint8 [..., dh / 16]) of rows [..., dh]."""
    b = x.double().unflatten(-1, (-1, 16))               # in 64 bits: elements lie on the borders between two codes
    top = b.abs().amax(dim=-1)
    want = top / torch.full_like(top, 120.0)             # 7.5 * 16
    ex = torch.frexp(want).exponent
    quantum = torch.exp2((ex - 3).clamp(min=-16).double())
    e = torch.where(top > 0, torch.ceil(want / quantum) * quantum, torch.zeros_like(want)).clamp(max=56.0)
    S = (e * 16.0).unsqueeze(-1)
    n = torch.where(S > 0, torch.round(b / S), torch.zeros_like(b)).clamp(-7, 7)
    c = (n + 8).to(torch.uint8).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), (e.half().view(torch.int16) >> 8).to(torch.uint8)


def _unpack(codes, scales):
    """fp32 values of codes and scales."""
    n = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float() - 8.0
    e = (scales.to(torch.int16) << 8).view(torch.float16).float() * 16.0
    return n * e.repeat_interleave(16, dim=-1)


def _parts(pool, dh):
    """Codes [n_pages][Hkv][page_size][dh / 2] and scales [...][dh / 16] of a pool: views."""
    codes = pool[..., : 8 * dh].unflatten(-1, (16, dh // 2))
    scales = pool[..., 8 * dh:].unflatten(-1, (16, dh // 16))
    return codes, scales


def _slot(s, seq, row):
    """Page, piece of 16 rows and row of the piece of the rows `row` of the sequences `seq`."""
    page = s["page"]
    return s["block_table"].long()[seq, row // page], (row % page) // 16, row % 16


# --------------------------------------------------------------------------- inputs


def _slopes(Hq, dev):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32, device=dev)


def _positions(n, g, dev):
    """Ascending positions; about half of the rows in between were pruned."""
    step = torch.randint(1, 4, (n,), generator=g, device=dev, dtype=torch.int32)
    return (torch.cumsum(step, 0) - step[0]).to(torch.int32)


def _i32(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _pool(n_pages, Hkv, page, dh, g, dev):
    """A pool of quantised normal numbers, a few pages at a time."""
    pool = torch.empty((n_pages, Hkv, page // 16, 9 * dh), dtype=torch.uint8, device=dev)
    at_once = max(1, (1 << 24) // (Hkv * page * dh))
    for p in range(0, n_pages, at_once):
        m = min(at_once, n_pages - p)
        codes, scales = _pack(torch.randn((m, Hkv, page // 16, 16, dh), generator=g, device=dev))
        pool[p:p + m, ..., : 8 * dh] = codes.flatten(-2)
        pool[p:p + m, ..., 8 * dh:] = scales.flatten(-2)
    return pool


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 23)
    Hq, Hkv, dh = DECODERS[case["decoder"]]
    dt = DTYPES[case["dtype"]]
    s = dict(case, scale=dh ** -0.5)

    def randn(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device=dev) * scale).to(dt)

    if case["kind"] == "rotate":
        n = case["n"]
        # Q, K and V of a row lie behind one another, as one product leaves them
        qkv = randn(n, Hq + 2 * Hkv, dh, scale=3.0)
        r, axis = _rotary(case)
        # rows of a frame of 12 x 12 places, of which about half are left; one axis: the place in the prompt
        at = _positions(n, g, dev)
        pos = [at] if case["axes"] == 1 else [at // 144, (at % 144) // 12, at % 12]
        s.update(q=qkv[:, :Hq].transpose(0, 1), k=qkv[:, Hq:Hq + Hkv].transpose(0, 1), axis=axis,
                 positions=torch.stack([p + case["far"] for p in pos]).to(torch.int32),
                 inv_freq=(1e6 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().to(dev),
                 q_weight=1.0 + 0.2 * torch.randn((dh,), generator=g, device=dev) if case["norm"] else None,
                 k_weight=1.0 + 0.2 * torch.randn((dh,), generator=g, device=dev) if case["norm"] else None, eps=1e-6)
        return s

    B, page = case["B"], case["page"]
    if case["kind"] == "append":
        new, old = _append_lens(case)
        total, most = sum(new), max(a + b for a, b in zip(new, old))
    else:
        lens = _seq_lens(case)
        total, most = sum(lens), max(lens) + 1
    max_pages = _pages(most, page)
    n_pages = B * max_pages + 3
    S_cap = max_pages * page
    table = torch.randperm(n_pages, generator=g, device=dev)[: B * max_pages].to(torch.int32).view(B, max_pages)
    s.update(block_table=table, total=total)
    if case["kind"] == "append":
        pool = lambda: torch.zeros((n_pages, Hkv, page // 16, 9 * dh), dtype=torch.uint8, device=dev)
        # the projections of the layer lie token by token
        s.update(k_new=randn(total, Hkv, dh, scale=2.0).transpose(0, 1), v_new=randn(total, Hkv, dh).transpose(0, 1), k_pool=pool(),
                 v_pool=pool(), kv_len=_i32(old, dev), new_offsets=_i32(np.concatenate([[0], np.cumsum(new)]), dev),
                 positions=torch.arange(S_cap, dtype=torch.int32, device=dev).repeat(B, 1), mass=torch.rand((B, S_cap), generator=g, device=dev),
                 pos_new=torch.cat([_positions(n, g, dev) + o for n, o in zip(new, old)]),
                 mass_new=torch.rand((total,), generator=g, device=dev))
        return s
    s.update(k_pool=_pool(n_pages, Hkv, page, dh, g, dev), v_pool=_pool(n_pages, Hkv, page, dh, g, dev), kv_len=_i32(lens, dev))
    if case["kind"] == "read":
        s.update(offsets=_i32(np.concatenate([[0], np.cumsum(lens)]), dev), positions=torch.stack([_positions(S_cap, g, dev) for _ in range(B)]))
        return s
    s.update(q=randn(B, Hq, dh, scale=6.0 if case["cap"] else 1.0), slopes=_slopes(Hq, dev) if case["bias"] else None,
             positions=torch.stack([_positions(S_cap, g, dev) for _ in range(B)]) if case["bias"] else None,
             mass=torch.rand((B, S_cap), generator=g, device=dev) * 1e-3 if case["mass"] else None)
    return s


# --------------------------------------------------------------------------- plain forms


def _plain_rotate(s):
    angle = s["positions"].double()[torch.tensor(s["axis"], device=s["positions"].device)].T * s["inv_freq"].double()    # [n][pairs]
    cos, sin = angle.cos().float(), angle.sin().float()
    half = cos.shape[1]

    def turn(x, w):
        y = x.float()
        if s["norm"]:
            y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + s["eps"]) * w
        else:
            y = y.clone()
        if s["interleaved"]:
            a, b = y[..., 0:2 * half:2].clone(), y[..., 1:2 * half:2].clone()
            y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = y[..., :half].clone(), y[..., half:2 * half].clone()
            y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
        return y.to(x.dtype)

    return {"q": turn(s["q"], s["q_weight"]), "k": turn(s["k"], s["k_weight"])}


def _plain_rows(s, seq, row, dtype):
    """Values of rows of sequences, [Hkv][rows][dh]."""
    dh = DECODERS[s["decoder"]][2]
    page, piece, at = _slot(s, seq, row)
    res = []
    for pool in (s["k_pool"], s["v_pool"]):
        codes, scales = _parts(pool, dh)
        res.append(_unpack(codes[page, :, piece, at], scales[page, :, piece, at]).to(dtype).transpose(0, 1).contiguous())
    return res


def _plain_append(s):
    dh = DECODERS[s["decoder"]][2]
    off, old = s["new_offsets"].long(), s["kv_len"].long()
    i = torch.arange(s["k_new"].shape[1], device=off.device)
    seq = torch.searchsorted(off[1:], i, right=True)
    row = old[seq] + i - off[seq]
    page, piece, at = _slot(s, seq, row)
    for pool, new in ((s["k_pool"], s["k_new"]), (s["v_pool"], s["v_new"])):
        codes, scales = _parts(pool, dh)
        c, e = _pack(new.transpose(0, 1))
        codes[page, :, piece, at] = c
        scales[page, :, piece, at] = e
    s["positions"][seq, row] = s["pos_new"]
    s["mass"][seq, row] = s["mass_new"]
    k, v = _plain_rows(s, seq, row, s["k_new"].dtype)
    return {"k": k, "v": v, "positions": s["positions"], "mass": s["mass"], "new_len": (old + off[1:] - off[:-1]).int()}


def _plain_read(s):
    off = s["offsets"].long()
    i = torch.arange(s["total"], device=off.device)
    seq = torch.searchsorted(off[1:], i, right=True)
    row = i - off[seq]
    k, v = _plain_rows(s, seq, row, DTYPES[s["dtype"]])
    return {"k": k, "v": v, "positions": s["positions"][seq, row]}


def _plain_decode(s):
    q = s["q"].float()
    B, Hq, dh = q.shape
    Hkv = s["k_pool"].shape[1]
    page = s["page"]
    S_cap = s["block_table"].shape[1] * page
    table = s["block_table"].long()

    def rows(pool):
        codes, scales = _parts(pool, dh)
        return _unpack(codes[table], scales[table]).transpose(1, 2).reshape(B, Hkv, S_cap, dh)

    x = torch.matmul(q.view(B, Hkv, Hq // Hkv, dh), rows(s["k_pool"]).transpose(2, 3)).mul_(s["scale"])
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
    out = torch.matmul(p, rows(s["v_pool"])).view(B, Hq, dh).to(s["q"].dtype)
    res = {"out": out, "lse": (total.log() + top).view(B, Hq)}
    if s["mass"] is not None:
        s["mass"].add_(p.view(B, Hq, S_cap).sum(dim=1) / Hq)
        res["mass"] = s["mass"]
    return res


def run(state):
    s = state
    if not own:
        return {"rotate": _plain_rotate, "append": _plain_append, "read": _plain_read, "decode": _plain_decode}[s["kind"]](s)
    from paper_2506_02850_b200 import binding as B
    if s["kind"] == "rotate":
        r = B.metok_rotate_heads(s["q"], s["k"], s["inv_freq"], s["positions"], pair_axis=s["axis"], interleaved=s["interleaved"],
                                 eps=s["eps"] if s["norm"] else None, q_weight=s["q_weight"], k_weight=s["k_weight"])
        return {"q": r["q"], "k": r["k"]}
    if s["kind"] == "append":
        new_len = B.metok_paged_append_q4(s["k_new"], s["v_new"], s["k_pool"], s["v_pool"], s["block_table"], s["kv_len"],
                                          new_offsets=s["new_offsets"], positions=s["positions"], pos_new=s["pos_new"], mass=s["mass"],
                                          mass_new=s["mass_new"])["new_len"]
        r = B.metok_paged_read_q4(s["k_pool"], s["v_pool"], s["block_table"], new_len, s["new_offsets"], s["total"], first_row=s["kv_len"],
                                  dtype=s["k_new"].dtype)
        return {"k": r["k"], "v": r["v"], "positions": s["positions"], "mass": s["mass"], "new_len": new_len}
    if s["kind"] == "read":
        r = B.metok_paged_read_q4(s["k_pool"], s["v_pool"], s["block_table"], s["kv_len"], s["offsets"], s["total"], positions=s["positions"],
                                  dtype=DTYPES[s["dtype"]])
        return {"k": r["k"], "v": r["v"], "positions": r["positions"]}
    r = B.metok_paged_attention_q4(s["q"], s["k_pool"], s["v_pool"], s["block_table"], s["kv_len"], s["scale"], softcap=s["cap"],
                                   slopes=s["slopes"], positions=s["positions"], mass=s["mass"], with_lse=True)
    res = {"out": r["out"], "lse": r["lse"]}
    if s["mass"] is not None:
        res["mass"] = s["mass"]
    return res


# --------------------------------------------------------------------------- work


def work(case):
    Hq, Hkv, dh = DECODERS[case["decoder"]]
    e = BYTES[case["dtype"]]
    if case["kind"] == "rotate":
        n = case["n"]
        x = n * (Hq + Hkv) * dh
        return {"bytes": 2 * x * e + 4 * n * case["axes"], "flops": (4 if case["norm"] else 0) * x + int(3 * x * case["part"])}
    row, row4 = 2 * Hkv * dh * e, 2 * Hkv * dh * 9 // 16            # K and V: as numbers, and in 4 bits
    if case["kind"] == "append":
        n = sum(_append_lens(case)[0])
        return {"bytes": n * (2 * row + 2 * row4 + 16), "flops": 0}
    lens = _seq_lens(case)
    n = sum(lens)
    tables = 4 * sum(_pages(m, case["page"]) for m in lens)
    if case["kind"] == "read":
        return {"bytes": n * (row + row4 + 8) + tables, "flops": 0}
    return {"bytes": n * (row4 + (8 if case["mass"] else 0) + (4 if case["bias"] else 0)) + 2 * case["B"] * Hq * dh * e + tables,
            "flops": 4 * dh * Hq * n}


# --------------------------------------------------------------------------- the definitions, in 64 bits


def _held(x):
    """What elements [..., dh] stand for in the cache, in 64 bits: the scale is looked up among all numbers of its type."""
    scale = np.array([m * 2.0 ** e for e in range(-16, 4) for m in (4, 5, 6, 7)] + [m * 2.0 ** -16 for m in (0, 1, 2, 3)])
    scale = torch.from_numpy(np.sort(scale[scale <= 56.0]) * 16.0).to(x.device)
    b = x.double().reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    at = torch.searchsorted(7.5 * scale, b.abs().max(dim=-1).values.contiguous()).clamp(max=len(scale) - 1)
    S = scale[at][..., None]
    n = torch.where(S > 0, b / torch.where(S > 0, S, torch.ones_like(S)), torch.zeros_like(b)).round().clamp(-7, 7)
    return (n * S).reshape(x.shape)


def _stand_for(pool, page, head, dh):
    """Values of all rows of one head in the pages `page`, in 64 bits."""
    raw = pool[page, head]                               # [pages][page_size / 16][9 dh]
    codes = raw[..., : 8 * dh].reshape(-1, dh // 2)
    byte = raw[..., 8 * dh:].reshape(-1, dh // 16).long()
    ex, man = byte >> 2, (byte & 3).double()
    e = torch.where(ex > 0, (4 + man) * torch.exp2(ex.double() - 17.0), man * 2.0 ** -16)
    n = torch.zeros((codes.shape[0], dh), dtype=torch.float64, device=pool.device)
    n[:, 0::2] = (codes % 16).double() - 8
    n[:, 1::2] = (codes // 16).double() - 8
    return n * torch.repeat_interleave(16.0 * e, 16, dim=1)


def _exact_rotate(s):
    half = len(s["axis"])
    angle = torch.stack([s["positions"][a].double() * s["inv_freq"][i].double() for i, a in enumerate(s["axis"])], dim=1)
    turn = torch.polar(torch.ones_like(angle), angle)    # a + ib goes to (a + ib) e^(i angle)
    res = {}
    for name in ("q", "k"):
        y = s[name].double()
        if s["norm"]:
            y = y / torch.sqrt((y ** 2).sum(dim=-1, keepdim=True) / y.shape[-1] + s["eps"]) * s[name + "_weight"].double()
        if s["interleaved"]:
            z = torch.complex(y[..., 0:2 * half:2].contiguous(), y[..., 1:2 * half:2].contiguous()) * turn
            y[..., 0:2 * half:2], y[..., 1:2 * half:2] = z.real, z.imag
        else:
            z = torch.complex(y[..., :half].contiguous(), y[..., half:2 * half].contiguous()) * turn
            y[..., :half], y[..., half:2 * half] = z.real, z.imag
        res[name] = y
    return res


def _exact_append(s):
    pos, mass = s["positions"].clone(), s["mass"].clone()
    new, old = _append_lens(s)
    i = 0
    for b, (n, o) in enumerate(zip(new, old)):
        pos[b, o:o + n] = s["pos_new"][i:i + n]
        mass[b, o:o + n] = s["mass_new"][i:i + n]
        i += n
    return {"k": _held(s["k_new"]), "v": _held(s["v_new"]), "positions": pos, "mass": mass.double(),
            "new_len": _i32([a + b for a, b in zip(new, old)], "cuda")}


def _exact_read(s):
    _, Hkv, dh = DECODERS[s["decoder"]]
    res = {"k": [], "v": [], "positions": []}
    for b, n in enumerate(_seq_lens(s)):
        page = s["block_table"][b, : _pages(n, s["page"])].long()
        for name in ("k", "v"):
            res[name].append(torch.stack([_stand_for(s[name + "_pool"], page, h, dh)[:n] for h in range(Hkv)]))
        res["positions"].append(s["positions"][b, :n])
    return {"k": torch.cat(res["k"], dim=1), "v": torch.cat(res["v"], dim=1), "positions": torch.cat(res["positions"])}


def _exact_decode(s):
    B, Hq, dh = s["q"].shape
    Hkv = s["k_pool"].shape[1]
    out = torch.zeros((B, Hq, dh), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, Hq), dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if s["mass"] is not None else None
    for b, n in enumerate(_seq_lens(s)):
        pages = s["block_table"][b, : _pages(n, s["page"])].long()
        for hk in range(Hkv):
            k, v = (_stand_for(s[name], pages, hk, dh)[:n] for name in ("k_pool", "v_pool"))
            for h in range(hk * Hq // Hkv, (hk + 1) * Hq // Hkv):
                x = k @ s["q"][b, h].double() * s["scale"]
                if s["cap"]:
                    x = s["cap"] * torch.tanh(x / s["cap"])
                if s["slopes"] is not None:
                    pos = s["positions"][b, :n].double()
                    x = x - s["slopes"][h].double() * (pos[n - 1] - pos).abs()
                p = torch.softmax(x, dim=0)
                lse[b, h] = torch.logsumexp(x, dim=0)
                out[b, h] = p @ v
                if mass is not None:
                    mass[b, :n] += p / Hq
    res = {"out": out, "lse": lse}
    if mass is not None:
        res["mass"] = mass
    return res


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "read": _exact_read, "decode": _exact_decode}[case["kind"]](s)
