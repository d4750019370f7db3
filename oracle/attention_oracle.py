"""CPU oracle of the attention over what the compression leaves and of the paged cache, in float64 from the definitions in
include/metok.h.  Shares no code with the library.

Every attention function also says how far fp32 arithmetic may be off, from the roundings that it cannot avoid:

  a logit x = scale * <q, k> in fp32: a chain of dh products and sums, each off by at most one step of 2^-23 relative to the sum
  of the products' absolute values (rounded or truncated), the scale, cap and conversion to powers of two a few steps of 2^-23 of
  |x| (the cap's derivative is at most 1; a tanh from 1 - 2 / (1 + e^2x) is off by a few steps of 1, so of the cap), the bias's
  product and difference a few of slope * distance;
  a weight e^x: e^(error of x), and 2^-21 for the exponential itself;
  a sum of n weights: n steps of 2^-24.
"""

import numpy as np

STEP = 2.0 ** -23


def logits(q, k, scale, softcap=0.0, slope=0.0, far=None):
    """(x, bound on its fp32 error) of the rows q [n, dh] and k [m, dh]."""
    q, k = np.asarray(q, np.float64), np.asarray(k, np.float64)
    dh = q.shape[-1]
    x = scale * (q @ k.T)
    err = scale * (np.abs(q) @ np.abs(k).T) * (dh * STEP)
    if softcap > 0:
        x = softcap * np.tanh(x / softcap)
        err = err + 8 * STEP * softcap
    err = err + 8 * STEP * np.abs(x)
    if far is not None:
        x = x - slope * far
        err = err + 8 * STEP * abs(slope) * far + 2 * STEP * np.abs(x)
    return x, err


def weigh(x, err, seen, v):
    """Softmax over the keys seen: (out, lse, weights, bounds on the fp32 errors of the three)."""
    n, m = x.shape
    v = np.asarray(v, np.float64)
    out = np.zeros((n, v.shape[1]))
    lse = np.full(n, -np.inf)
    p = np.zeros((n, m))
    out_err, lse_err, p_err = np.zeros_like(out), np.zeros(n), np.zeros_like(p)
    for i in range(n):
        s = np.nonzero(seen[i])[0]
        if not len(s):
            continue
        xi = x[i, s]
        top = xi.max()
        e = np.exp(xi - top)
        w = e / e.sum()
        lse[i] = top + np.log(e.sum())
        p[i, s] = w
        out[i] = w @ v[s]
        # a weight's own error, and the error of the normaliser (its mean over the weights)
        rel = np.expm1(err[i, s]) + 4 * STEP
        norm = w @ rel + len(s) * STEP / 2
        p_err[i, s] = w * (rel + norm)
        out_err[i] = (w * (rel + norm + len(s) * STEP / 2)) @ np.abs(v[s])
        lse_err[i] = norm + 4 * STEP * max(abs(lse[i]), abs(top), 1.0)
    return out, lse, p, out_err, lse_err, p_err


def visible(Lq, Lk, causal=True, prefix=0):
    """[Lq, Lk]: which keys the document's last Lq rows see."""
    c = Lk - Lq + np.arange(Lq)[:, None]
    j = np.arange(Lk)[None, :]
    return np.ones((Lq, Lk), bool) if not causal else (j <= c) | (j < prefix)


def prompt_attention(q, k, v, scale, seq_q=None, seq_k=None, prefix_len=None, causal=True, softcap=0.0, slopes=None, positions=None):
    """q [Hq, n_q, dh], k and v [Hkv, n_k, dh] -> dict of out, lse, their error bounds, and absv = sum of weight * |v|.
    Rows outside every document are NaN in out and lse."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    Hq, n_q, dh = q.shape
    Hkv, n_k, _ = k.shape
    seq_q = np.array([0, n_q]) if seq_q is None else np.asarray(seq_q)
    seq_k = np.array([0, n_k]) if seq_k is None else np.asarray(seq_k)
    res = {"out": np.full(q.shape, np.nan), "lse": np.full((Hq, n_q), np.nan), "out_err": np.zeros(q.shape), "lse_err": np.zeros((Hq, n_q)),
           "absv": np.zeros(q.shape)}
    for d in range(len(seq_q) - 1):
        q0, q1, k0, k1 = seq_q[d], seq_q[d + 1], seq_k[d], seq_k[d + 1]
        Lq, Lk = q1 - q0, k1 - k0
        seen = visible(Lq, Lk, causal, 0 if prefix_len is None else prefix_len[d])
        pos = np.arange(Lk, dtype=np.float64) if positions is None else np.asarray(positions, np.float64)[k0:k1]
        far = None
        if slopes is not None and Lk:
            c = np.clip(Lk - Lq + np.arange(Lq), 0, None)
            far = np.abs(pos[c][:, None] - pos[None, :])
        for h in range(Hq):
            g = h // (Hq // Hkv)
            x, err = logits(q[h, q0:q1], k[g, k0:k1], scale, softcap, 0.0 if slopes is None else float(slopes[h]), far)
            o, lse, p, oe, le, _ = weigh(x, err, seen, v[g, k0:k1])
            res["out"][h, q0:q1], res["lse"][h, q0:q1], res["out_err"][h, q0:q1], res["lse_err"][h, q0:q1] = o, lse, oe, le
            res["absv"][h, q0:q1] = p @ np.abs(v[g, k0:k1])
    return res


def cache_rows(pool, table, n):
    """The first n rows [Hkv, n, dh] of a sequence: pool [n_pages, Hkv, page, dh], its row of the block table."""
    page = pool.shape[2]
    rows = [pool[table[r // page], :, r % page] for r in range(n)]
    return np.stack(rows, axis=1) if rows else np.zeros((pool.shape[1], 0, pool.shape[3]))


def paged_attention(q, k_pool, v_pool, block_table, kv_len, scale, softcap=0.0, slopes=None, positions=None):
    """q [B, Hq, dh] -> dict of out, lse, weights [B][Hq, n] (a list), and their error bounds."""
    q, k_pool, v_pool = (np.asarray(t, np.float64) for t in (q, k_pool, v_pool))
    B, Hq, dh = q.shape
    Hkv = k_pool.shape[1]
    res = {"out": np.zeros(q.shape), "lse": np.full((B, Hq), -np.inf), "out_err": np.zeros(q.shape), "lse_err": np.zeros((B, Hq)),
           "absv": np.zeros(q.shape), "p": [], "p_err": []}
    for b in range(B):
        n = int(kv_len[b])
        k, v = cache_rows(k_pool, block_table[b], n), cache_rows(v_pool, block_table[b], n)
        ps, pe = np.zeros((Hq, n)), np.zeros((Hq, n))
        for h in range(Hq):
            if n == 0:
                continue
            g = h // (Hq // Hkv)
            pos = np.arange(n) if positions is None else np.asarray(positions[b], np.float64)[:n]
            x, err = logits(q[b, h:h + 1], k[g], scale, softcap, 0.0 if slopes is None else float(slopes[h]),
                            None if slopes is None else np.abs(pos[n - 1] - pos)[None])
            o, lse, p, oe, le, p_err = weigh(x, err, np.ones((1, n), bool), v[g])
            res["out"][b, h], res["lse"][b, h], res["out_err"][b, h], res["lse_err"][b, h] = o[0], lse[0], oe[0], le[0]
            res["absv"][b, h] = p[0] @ np.abs(v[g])
            ps[h], pe[h] = p[0], p_err[0]
        res["p"].append(ps)
        res["p_err"].append(pe)
    return res


def evict_rows(mass, positions, n, budget, n_sink, n_recent):
    """The row that each kept row holds afterwards: one layer of one sequence of n rows."""
    if n <= budget:
        return np.arange(n)
    mass, positions = np.asarray(mass[:n], np.float64), np.asarray(positions[:n], np.int64)
    safe = (positions < n_sink) | (positions > positions[n - 1] - n_recent)
    kind = np.where(safe, 0, np.where(np.isnan(mass), 1, 2))
    rank = sorted(range(n), key=lambda i: (kind[i], -mass[i] if kind[i] == 2 else 0.0, i))
    kept = sorted(rank[:budget])
    rows = np.arange(budget)
    holes = sorted(set(range(budget)) - set(kept))
    for hole, mover in zip(holes, [i for i in kept if i >= budget]):
        rows[hole] = mover
    return rows


# ---- heads turned by their positions, and a cache held in 4 bits ------------------------------------------------------


def rotate(x, angles, interleaved=False, eps=None, weight=None):
    """x [H, n, dh] by angles [n, pairs]; eps: heads normed first.  Returns the values and, for each element, the sum of the absolute values of the
    two that it is made of."""
    y = np.array(x, np.float64)
    if eps is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else np.asarray(weight, np.float64))
    size = np.abs(y)
    half = angles.shape[1]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, v = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = u * np.cos(angles) - v * np.sin(angles), v * np.cos(angles) + u * np.sin(angles)
    size[..., a] = size[..., b] = np.abs(u) + np.abs(v)
    return y, size


# every number of type e5m2 from 0 to 56, in order: byte i stands for E5M2[i]
E5M2 = np.array([m * 2.0 ** -16 for m in range(4)] + [(4 + m) * 2.0 ** (e - 17) for e in range(1, 21) for m in range(4)])
E5M2 = E5M2[E5M2 <= 56.0]


def q4_hold(x):
    """Rows [..., dh] -> codes uint8 [..., dh / 2] and scales uint8 [..., dh / 16]."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    sound = np.isfinite(b).all(-1)
    b = np.where(sound[..., None], b, 0.0)
    e = np.minimum(np.searchsorted(120.0 * E5M2, np.abs(b).max(-1)), len(E5M2) - 1)
    S = 16.0 * E5M2[e][..., None]
    n = np.clip(np.rint(np.divide(b, S, out=np.zeros_like(b), where=S > 0)), -7, 7)
    c = (n + 8).astype(np.uint8).reshape(x.shape)
    return c[..., 0::2] | c[..., 1::2] << 4, np.where(sound, e, 0x7F).astype(np.uint8)


def q4_values(codes, scales):
    """What rows held as q4_hold says stand for."""
    n = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1]).astype(np.float64) - 8
    e = np.append(E5M2, np.full(256 - len(E5M2), np.nan))[scales]
    return n * np.repeat(16.0 * e, 16, axis=-1)


def q4_parts(pool):
    """Views of a pool [n_pages, Hkv, page / 16, 9 dh]: codes [n_pages, Hkv, page / 16, 16, dh / 2], scales [..., 16, dh / 16]."""
    dh = pool.shape[-1] // 9
    return pool[..., :8 * dh].reshape(*pool.shape[:-1], 16, dh // 2), pool[..., 8 * dh:].reshape(*pool.shape[:-1], 16, dh // 16)


def q4_pool_values(pool):
    """A whole pool's values, [n_pages, Hkv, page, dh]."""
    v = q4_values(*q4_parts(pool))
    return v.reshape(*v.shape[:2], -1, v.shape[-1])
