"""float64 oracle of multi-head attention over packed documents and paged
caches, with its gradients, and of the cache's bookkeeping.

Written from the definitions in include/attention_mi355x.h, one document and
head at a time.  Beside each value stands the bound that an implementation
with fp32 sums, statistics and exponentials may be off by, for inputs and
outputs of a type of unit roundoff u (weights and score gradients rounded to
it once where the type has 16 bits):

    score      e_x = (d + 4) 2^-24 |scale| sum |q k| + 2^-22 |x| + 2^-20 cap
               (a dot product's rounding, the scaling, shift and exponent
               argument's, and the tanh's few ulp)
    weight     e_p = 2 e_x + 2^-19, relative: numerator and sum
    o          u |o| + sum_j P_j (u_w + e_p) |v_j|
    dv         u |dv| + sum_i P_i (u_w + e_p) |do_i|
    D          sum_c |do_c| (error of o_c) + d 2^-23 sum_c |do_c o_c|
    ds         P (e_p + u_w + 2^-18) |dP - D| |x'|
               + P (d 2^-23 sum_c |do_c v_c| + error of D) |x'|
    dq, dk     u |.| + sum (error of ds) |k| or |q|, + d 2^-23 as for o

and, for 16-bit floats of a small range, the step of the denormal numbers for
each rounded weight and output.
"""
from __future__ import annotations

import numpy as np

UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def seen_keys(lq: int, lk: int, causal: bool, prefix: int) -> np.ndarray:
    """Boolean [lq, lk]."""
    i, j = np.arange(lq)[:, None] + (lk - lq), np.arange(lk)[None, :]
    return (j <= i) | (j < prefix) if causal else np.ones((lq, lk), bool)


def head(q, k, v, *, dtype, scale, cap=0.0, slope=0.0, causal=True, prefix=0, dout=None,
         held=None):
    """One head of one document: dict of values and of bounds ("e_" names).
    ``held`` [lk]: keys that exist at all."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    lq, lk, d = len(q), len(k), q.shape[1]
    u, tiny = UNIT[dtype], TINY[dtype]
    u_w = 0.0 if dtype == "f32" else u
    seen = seen_keys(lq, lk, causal, min(prefix, lk))
    if held is not None:
        seen = seen & held[None, :]
    x = scale * (q @ k.T)
    e_x = (d + 4) * 2.0 ** -24 * abs(scale) * (np.abs(q) @ np.abs(k).T)
    dcap = np.ones_like(x)
    if cap:
        t = np.tanh(x / cap)
        x, dcap = cap * t, 1.0 - t * t
    if slope:
        x = x - slope * np.abs(np.arange(lq)[:, None] + (lk - lq) - np.arange(lk)[None, :])
    e_x = e_x + 2.0 ** -22 * np.abs(x) + 2.0 ** -20 * cap
    some = seen.any(1)
    top = np.where(some, np.max(np.where(seen, x, -np.inf), 1, initial=-np.inf), 0.0)
    e = np.where(seen, np.exp(np.minimum(x - top[:, None], 0.0)), 0.0)
    total = e.sum(1)
    p = e / np.where(some, total, 1.0)[:, None]
    lse = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
    worst = np.max(np.where(seen, e_x, 0.0), 1, initial=0.0)[:, None]
    e_p = 2.0 * worst + 2.0 ** -19
    o = p @ v
    e_o = u * np.abs(o) + (p * (u_w + e_p)) @ np.abs(v) + tiny * (1.0 + seen @ np.abs(v))
    out = {"o": o, "lse": lse, "e_o": e_o,
           "e_lse": worst[:, 0] + 2.0 ** -19 + 2.0 ** -22 * np.abs(np.where(some, lse, 0.0))}
    if dout is None:
        return out
    do = np.asarray(dout, np.float64)
    dp = do @ v.T
    delta = (do * o).sum(1, keepdims=True)
    ds = p * (dp - delta) * dcap
    e_d = (np.abs(do) * e_o).sum(1, keepdims=True) + d * 2.0 ** -23 * (
        np.abs(do) * np.abs(o)).sum(1, keepdims=True)
    e_ds = p * (e_p + u_w + 2.0 ** -18) * np.abs(dp - delta) * dcap \
        + p * (1.0 + u_w) * (d * 2.0 ** -23 * (np.abs(do) @ np.abs(v).T) + e_d) \
        + p * np.abs(dp - delta) * (2.0 ** -19 if cap else 0.0) + tiny * seen
    out["dv"] = p.T @ do
    out["e_dv"] = u * np.abs(out["dv"]) + (p * (u_w + e_p)).T @ np.abs(do) \
        + tiny * (1.0 + seen.T @ np.abs(do))
    out["dq"], out["dk"] = scale * (ds @ k), scale * (ds.T @ q)
    e_ds = e_ds + d * 2.0 ** -23 * np.abs(ds)
    out["e_dq"] = u * np.abs(out["dq"]) + abs(scale) * (e_ds @ np.abs(k)) + tiny
    out["e_dk"] = u * np.abs(out["dk"]) + abs(scale) * (e_ds.T @ np.abs(q)) + tiny
    return out


def packed(q, k, v, cu_q, cu_k, *, dtype, scale=None, cap=0.0, slopes=None, causal=True,
           prefix=None, dout=None):
    """All documents and heads: q [tokens, heads, d], k and v [tokens,
    kv_heads, d]; as head()."""
    heads, kv_heads, d = q.shape[1], k.shape[1], q.shape[2]
    scale = d ** -0.5 if scale is None else scale
    out = {"o": np.zeros(q.shape), "e_o": np.zeros(q.shape),
           "lse": np.full(q.shape[:2], -np.inf), "e_lse": np.zeros(q.shape[:2])}
    if dout is not None:
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            out[name], out["e_" + name] = np.zeros(like.shape), np.zeros(like.shape)
    for b in range(len(cu_q) - 1):
        a, c = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        for h in range(heads):
            g = h // (heads // kv_heads)
            got = head(q[a, h], k[c, g], v[c, g], dtype=dtype, scale=scale, cap=cap,
                       slope=0.0 if slopes is None else float(slopes[h]), causal=causal,
                       prefix=0 if prefix is None else int(prefix[b]),
                       dout=None if dout is None else dout[a, h])
            for name, x in got.items():
                if name.endswith(("dk", "dv")):
                    out[name][c, g] += x
                else:
                    out[name][a, h] = x
    return out


def paged(q, k_cache, v_cache, table, cu_q, key_lens, *, dtype, scale=None, cap=0.0, slopes=None,
          causal=True, prefix=None):
    """Requests over caches [blocks, size, kv_heads, d]; as packed()."""
    heads, kv_heads, d = q.shape[1], k_cache.shape[2], q.shape[2]
    blocks, size = k_cache.shape[:2]
    scale = d ** -0.5 if scale is None else scale
    out = {"o": np.zeros(q.shape), "e_o": np.zeros(q.shape),
           "lse": np.full(q.shape[:2], -np.inf), "e_lse": np.zeros(q.shape[:2])}
    for b in range(len(key_lens)):
        a = slice(cu_q[b], cu_q[b + 1])
        j = np.arange(min(max(int(key_lens[b]), 0), table.shape[1] * size))
        page = table[b, j // size]
        held = (page >= 0) & (page < blocks)
        page = np.where(held, page, 0)
        for h in range(heads):
            g = h // (heads // kv_heads)
            k, v = (np.where(held[:, None], c[page, j % size, g], 0.0)
                    for c in (k_cache, v_cache))
            got = head(q[a, h], k, v, dtype=dtype, scale=scale, cap=cap,
                       slope=0.0 if slopes is None else float(slopes[h]), causal=causal,
                       prefix=0 if prefix is None else int(prefix[b]), held=held)
            for name, x in got.items():
                out[name][a, h] = x
    return out


def cache_slots(context, new, table, free, count, total, size):
    """The bookkeeping of a serving step, one token at a time."""
    table = np.array(table)
    count = min(max(int(count), 0), len(free))
    had, missing, slots, cu, lens = count, 0, [], [0], []
    for b, (c, x) in enumerate(zip(context, new)):
        c, x = max(int(c), 0), max(int(x), 0)
        for col in range(-(-c // size), -(-(c + x) // size)):
            if col >= table.shape[1]:
                missing += 1
            elif count > 0:
                count -= 1
                table[b, col] = free[count]
            else:
                missing += 1
                table[b, col] = -1
        for pos in range(c, c + x):
            col = pos // size
            entry = table[b, col] if col < table.shape[1] else -1
            slots.append(int(entry) * size + pos % size if entry >= 0 else -1)
        cu.append(cu[-1] + x)
        lens.append(c + x)
    assert had >= count
    slots = (slots + [-1] * total)[:total]
    return {"table": table, "cu_q": np.array(cu), "key_lens": np.array(lens),
            "slots": np.array(slots, dtype=np.int64), "free_count": np.array([count]),
            "missing": np.array([missing])}
