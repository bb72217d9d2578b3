"""The operators of a language model's attention, as cases to time and compare.

A case is one pass through one of the entry points that a training step or a
serving step calls:

    op "slots"    softmax_cache_slots          requests' lengths -> block table, slot map
    op "append"   softmax_cache_append         new keys and values into the paged cache
    op "paged"    softmax_paged_attention_fwd  chunks of new tokens over the paged cache
    op "packed"   softmax_packed_attention_fwd / _bwd
                  attention of packed documents, with its gradients where "train"

Lengths follow from the case alone (``lens``), values from the seed.

The plain forms below compute the same in elementary torch operations, in 32
bits: dense scores over all keys, with a mask for what a query does not see.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
LOWEST = torch.finfo(torch.float32).min


# ---------------------------------------------------------------------------
# The cases

def _slots(name, n, context, new, total, width, block, short):
    return {"name": name, "op": "slots", "n": n, "context": context, "new": new, "total": total,
            "width": width, "block": block, "short": short, "lens": 1}


def _append(name, tokens, heads, d, dtype, block, blocks):
    return {"name": name, "op": "append", "tokens": tokens, "heads": heads, "d": d,
            "dtype": dtype, "block": block, "blocks": blocks}


def _paged(name, singles, chunks, chunk, context, heads, kv_heads, d, dtype, block, cap, bias,
           prefix=0):
    return {"name": name, "op": "paged", "singles": singles, "chunks": chunks, "chunk": chunk,
            "context": context, "heads": heads, "kv_heads": kv_heads, "d": d, "dtype": dtype,
            "block": block, "cap": cap, "bias": bias, "prefix": prefix, "lens": 1}


def _packed(name, tokens, longest, heads, kv_heads, d, dtype, causal, cap, bias, prefix, train):
    return {"name": name, "op": "packed", "tokens": tokens, "longest": longest, "heads": heads,
            "kv_heads": kv_heads, "d": d, "dtype": dtype, "causal": causal, "cap": cap,
            "bias": bias, "prefix": prefix, "train": train, "lens": 1}


def listed():
    return [
        # A decode step of a small batch: one new token for each of 8
        # requests.  The smallest call: launch and host time.
        _slots("slots_decode_8", 8, 2048, 1, 8, 256, 16, False),
        # A serving step of a large batch, decodes and prompt chunks mixed:
        # 2048 requests, up to 65536 new tokens, tables 1024 blocks wide.
        _slots("slots_mixed_2048", 2048, 8192, 320, 65536, 1024, 16, False),
        # One decode step's keys and values of 64 requests.
        _append("append_decode_64", 64, 8, 128, "bf16", 16, 4096),
        # The keys and values of a step of long prompts, as slices of the
        # projection that made them.
        _append("append_prompt_16384", 16384, 8, 128, "f16", 64, 2048),
        # One request that decodes over a few thousand tokens of context:
        # latency, and work that has to be split to fill the device.
        _paged("paged_decode_1x4001", 1, 0, 0, 4001, 32, 8, 128, "f16", 16, 0.0, False),
        # A batch of decodes over contexts of all lengths up to 8192.
        _paged("paged_decode_64x8192", 64, 0, 0, 8192, 32, 8, 128, "bf16", 16, 0.0, False),
        # A step of mixed serving: decodes beside chunks of prompts, with
        # capped scores.
        _paged("paged_mixed_12_4x509", 12, 4, 509, 8192, 16, 4, 128, "bf16", 32, 30.0, False),
        # One chunk of a long prompt over its context, with a bias that falls
        # with distance: the largest serving call.
        _paged("paged_chunk_2048x65536", 0, 1, 2048, 65536, 32, 8, 128, "bf16", 64, 0.0, True),
        # A step of training in float32 on a few short documents of odd
        # lengths and head width.
        _packed("packed_f32_101", 101, 64, 4, 4, 80, "f32", True, 0.0, False, False, True),
        # A step of training on packed documents of all lengths up to 2048.
        _packed("packed_docs_8192", 8192, 2048, 32, 8, 128, "bf16", True, 0.0, False, False, True),
        # Documents with a prefix that all of their tokens see, capped scores
        # and a bias that falls with distance.
        _packed("packed_prefix_4099", 4099, 1531, 16, 16, 64, "f16", True, 30.0, True, True,
                True),
        # One long document, few key and value heads: the largest call.
        _packed("packed_long_16384", 16384, 16384, 16, 2, 128, "bf16", True, 0.0, False, False,
                True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# Most scores that a drawn case's plain form holds: those of the largest
# listed cases.
MOST_SCORES = 1 << 32


def draw(rng):
    op = rng.choice(["slots", "append", "paged", "paged", "paged", "packed", "packed", "packed"])
    lens = rng.randint(2, 1 << 20)
    if op == "slots":
        n, block = _log_uniform(rng, 1, 2048), rng.choice([8, 16, 32, 64, 128])
        context, new = _log_uniform(rng, 16, 8192), _log_uniform(rng, 1, 320)
        total = min(65536, n if new == 1 else n * new)
        return {"op": op, "n": n, "context": context, "new": new, "total": total,
                "width": -(-(context + new) // block) + rng.randint(0, 9), "block": block,
                "short": rng.random() < 0.3, "lens": lens}
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    d = rng.choice([64, 128, 128, 8 * rng.randint(2, 32)])
    if op == "append":
        tokens, block = _log_uniform(rng, 1, 16384), rng.choice([8, 16, 32, 64, 128])
        heads = rng.choice([1, 2, 4, 8])
        tokens = min(tokens, (1 << 24) // (heads * d))
        return {"op": op, "tokens": tokens, "heads": heads, "d": min(d, 128), "dtype": dtype,
                "block": block, "blocks": -(-2 * tokens // block) + rng.randint(1, 100)}
    group, kv_heads = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 4, 8])
    heads = group * kv_heads
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    bias = rng.random() < 0.3
    most = MOST_SCORES // 2 if dtype == "f32" else MOST_SCORES
    if op == "paged":
        kind = rng.choice(["single", "chunk", "mixed"])
        context = _log_uniform(rng, 1, 65536)
        singles = 0 if kind == "chunk" else _log_uniform(rng, 1, 200)
        chunks = 0 if kind == "single" else rng.randint(1, 4)
        chunk = _log_uniform(rng, 2, 2048) if chunks else 0
        d = min(d, 128) if dtype == "f32" else d
        heads, kv_heads = (heads, kv_heads) if heads <= 32 else (32, 8)
        # The gathered keys and values of the plain form, then its scores.
        context = max(1, min(context, (1 << 29) // ((singles + chunks) * kv_heads * d)))
        chunk = min(chunk, max(2, most // 4 // ((singles + chunks) * heads * (context + chunk + 1)))) \
            if chunks else 0
        return {"op": op, "singles": singles, "chunks": chunks, "chunk": chunk,
                "context": context, "heads": heads, "kv_heads": kv_heads, "d": d, "dtype": dtype,
                "block": rng.choice([8, 16, 32, 64, 128]), "cap": cap, "bias": bias,
                "prefix": rng.choice([0, 0, 1]), "lens": lens}
    tokens = _log_uniform(rng, 1, 16384)
    heads, kv_heads = (heads, kv_heads) if heads <= 32 else (32, 8)
    tokens = min(tokens, int((most // heads) ** 0.5) // (2 if d > 128 else 1))
    if dtype == "f32":
        tokens = min(tokens, 4096)
    return {"op": op, "tokens": tokens, "longest": _log_uniform(rng, max(1, tokens // 32), tokens),
            "heads": heads, "kv_heads": kv_heads, "d": d, "dtype": dtype,
            "causal": rng.random() < 0.8, "cap": cap, "bias": bias,
            "prefix": rng.random() < 0.25, "train": rng.random() < 0.75, "lens": lens}


# ---------------------------------------------------------------------------
# Lengths, from the case alone

def _slot_lens(case):
    """(tokens in the cache, new tokens) of each request."""
    rng = random.Random(case["lens"])
    ctx = [rng.randint(0, case["context"]) for _ in range(case["n"])]
    if case["new"] == 1:
        new = [1] * case["n"]
    else:  # decodes, prompt chunks, and now and then a request with nothing new
        new = [rng.choice([0, 1, 1, rng.randint(1, case["new"]), rng.randint(1, case["new"])])
               for _ in ctx]
    left = case["total"]
    for i, x in enumerate(new):
        new[i] = min(x, left)
        left -= new[i]
    return ctx, new


def _paged_lens(case):
    """(new tokens, tokens in the cache with the new ones) of each request."""
    rng = random.Random(case["lens"])
    new = [1] * case["singles"] + [case["chunk"]] * case["chunks"]
    if case["singles"] + case["chunks"] == 1:
        return new, [max(new[0], case["context"])]
    # Contexts of all lengths, the longest among them.
    keys = [max(x, rng.randint(1, case["context"])) for x in new]
    keys[-1] = max(new[-1], case["context"])
    order = list(range(len(new)))
    rng.shuffle(order)
    return [new[i] for i in order], [keys[i] for i in order]


def _doc_lens(case):
    rng = random.Random(case["lens"])
    left, longest, lens = case["tokens"], case["longest"], []
    while left:
        n = longest if longest == case["tokens"] else \
            int(round(math.exp(rng.uniform(0.0, math.log(longest)))))
        lens.append(max(1, min(left, n)))
        left -= lens[-1]
    return lens


def _prefixes(case, lens):
    """Tokens at each document's start that all of its tokens see."""
    rng = random.Random(case["lens"] + 1)
    return [rng.randint(0, n) // 2 for n in lens] if case["prefix"] else None


def _sums(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _seen(new, keys, causal, prefix):
    """Pairs of a query and a key that it sees."""
    total = 0
    for b, (lq, lk) in enumerate(zip(new, keys)):
        pre = min(prefix[b], lk) if prefix else 0
        if not causal:
            total += lq * lk
            continue
        first = lk - lq + 1  # keys that the first query sees
        last = lk
        if pre <= first:
            total += lq * (first + last) // 2
        else:
            flat = min(lq, pre - first)
            total += flat * pre + (lq - flat) * (first + flat + last) // 2
    return total


# ---------------------------------------------------------------------------
# Inputs

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _normal(g, dtype, *shape):
    return torch.randn(*shape, device=DEVICE, generator=g).to(TYPES[dtype])


def _slopes(case):
    """Slopes of the bias, a falling geometric sequence over the heads."""
    if not case["bias"]:
        return None
    h = case["heads"]
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device=DEVICE)


def _prepare_slots(case, g):
    ctx, new = _slot_lens(case)
    block, width = case["block"], case["width"]
    held = [-(-c // block) for c in ctx]
    more = sum(-(-(c + x) // block) - h for c, x, h in zip(ctx, new, held))
    spare = more // 2 if case["short"] else more + 64
    ids = torch.randperm(sum(held) + spare, device=DEVICE, generator=g).to(torch.int32)
    base, h = _ints(_sums(held)[:-1])[:, None], _ints(held)[:, None]
    col = torch.arange(width, device=DEVICE)[None]
    at = (base + col).clamp(max=ids.numel() - 1)
    table = torch.where(col < h, ids[at.long()], -1).to(torch.int32).contiguous()
    free = torch.cat([ids[sum(held):], ids.new_full((8,), -1)])
    return {"ctx": _ints(ctx), "new": _ints(new), "table": table, "free": free,
            "count": _ints([spare])}


def _prepare_append(case, g):
    t, h, d, block = case["tokens"], case["heads"], case["d"], case["block"]
    # Keys and values as a fused projection leaves them: slices of one row.
    rows = _normal(g, case["dtype"], t, 2 * h * d + 8 * d)
    k = rows[:, 8 * d:8 * d + h * d].unflatten(1, (h, d))
    v = rows[:, 8 * d + h * d:].unflatten(1, (h, d))
    slots = torch.randperm(case["blocks"] * block, device=DEVICE, generator=g)[:t].clone()
    if t > 8:  # padding of the step
        slots[-3:] = -1
    caches = _normal(g, case["dtype"], 2, case["blocks"], block, h, d)
    return {"k": k, "v": v, "k_cache": caches[0], "v_cache": caches[1], "slots": slots}


def _prepare_paged(case, g):
    new, keys = _paged_lens(case)
    block, n = case["block"], len(new)
    width = -(-max(keys) // block)
    held = [-(-x // block) for x in keys]
    ids = torch.randperm(sum(held) + 3, device=DEVICE, generator=g).to(torch.int32)
    base, h = _ints(_sums(held)[:-1])[:, None], _ints(held)[:, None]
    col = torch.arange(width, device=DEVICE)[None]
    table = torch.where(col < h, ids[(base + col).clamp(max=ids.numel() - 1).long()], -1)
    caches = _normal(g, case["dtype"], 2, ids.numel(), block, case["kv_heads"], case["d"])
    prefix = _prefixes(case, keys)
    return {"q": _normal(g, case["dtype"], sum(new), case["heads"], case["d"]),
            "k_cache": caches[0], "v_cache": caches[1],
            "table": table.to(torch.int32).contiguous(), "cu_q": _ints(_sums(new)),
            "key_lens": _ints(keys), "cap": case["cap"], "slopes": _slopes(case),
            "prefix": None if prefix is None else _ints(prefix), "longest": max(new)}


def _prepare_packed(case, g):
    lens = _doc_lens(case)
    t, h, hk, d = case["tokens"], case["heads"], case["kv_heads"], case["d"]
    # One fused projection's row holds the queries, keys and values.
    rows = _normal(g, case["dtype"], t, (h + 2 * hk) * d)
    q, k, v = rows.split([h * d, hk * d, hk * d], 1)
    prefix = _prefixes(case, lens)
    return {"q": q.unflatten(1, (h, d)), "k": k.unflatten(1, (hk, d)),
            "v": v.unflatten(1, (hk, d)), "do": _normal(g, case["dtype"], t, h, d),
            "cu": _ints(_sums(lens)), "causal": case["causal"], "cap": case["cap"],
            "slopes": _slopes(case), "prefix": None if prefix is None else _ints(prefix),
            "train": case["train"]}


def prepare(case, seed):
    make = {"slots": _prepare_slots, "append": _prepare_append, "paged": _prepare_paged,
            "packed": _prepare_packed}[case["op"]]
    state = make(case, _generator(seed))
    state["op"], state["block"], state["total"] = case["op"], case.get("block"), case.get("total")
    return state


# ---------------------------------------------------------------------------
# Plain forms

def _plain_slots(s):
    table, free, block = s["table"], s["free"], s["block"]
    ctx, new, width = s["ctx"].long(), s["new"].long(), s["table"].shape[1]
    first = ((ctx + block - 1) // block).clamp(max=width)
    wanted = (ctx + new + block - 1) // block - (ctx + block - 1) // block
    last = (first + wanted).clamp(max=width)
    end = (last - first).cumsum(0)
    start = end - (last - first)
    col = torch.arange(width, device=table.device)[None]
    k = start[:, None] + col - first[:, None]
    fresh = (col >= first[:, None]) & (col < last[:, None])
    ids = free[(s["count"] - 1 - k).clamp(0, free.numel() - 1)]
    table.copy_(torch.where(fresh, torch.where(k < s["count"], ids, -1), table))
    taken = torch.minimum(end[-1:], s["count"].long())
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    t = torch.arange(s["total"], device=table.device)
    b = torch.bucketize(t, cu[1:], right=True).clamp(max=new.numel() - 1)
    pos = ctx[b] + t - cu[b]
    entry = table[b, (pos // block).clamp(max=width - 1)].long()
    fine = (t < cu[-1]) & (pos // block < width) & (entry >= 0)
    return {"table": table, "cu_q": cu.int(), "key_lens": (ctx + new).int(),
            "slots": torch.where(fine, entry * block + pos % block, -1),
            "free_count": (s["count"] - taken).int(), "missing": (wanted.sum() - taken).int()}


def _plain_append(s):
    fine = s["slots"] >= 0
    at = s["slots"][fine]
    for_k, for_v = s["k_cache"].flatten(0, 1), s["v_cache"].flatten(0, 1)
    for_k[at] = s["k"][fine]
    for_v[at] = s["v"][fine]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _scores(qk, q_pos, k_pos, seen, scale, cap, slopes):
    """Masked scores, and the derivative of the cap's tanh (1 without one)."""
    x = qk * scale
    slope = 1.0
    if cap:
        t = torch.tanh(x / cap)
        x, slope = cap * t, 1.0 - t * t
    if slopes is not None:
        x = x - slopes * (q_pos - k_pos).abs()
    return torch.where(seen, x, LOWEST), slope


def _weights(x, seen):
    """(softmax over the keys that are seen, log of its sum)."""
    m = x.amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(x - m), 0.0)
    total = e.sum(-1, keepdim=True)
    some = total > 0
    lse = torch.where(some, m + torch.log(total), -math.inf)
    return torch.where(some, e / torch.where(some, total, 1.0), 0.0), lse[..., 0]


def _plain_paged(s):
    q, cu, lens, block = s["q"], s["cu_q"].long(), s["key_lens"].long(), s["block"]
    tokens, heads, d = q.shape
    kv_heads = s["k_cache"].shape[2]
    n, keys = lens.numel(), s["table"].shape[1] * block
    new = cu[1:] - cu[:-1]
    j = torch.arange(keys, device=q.device)
    page = s["table"].clamp(min=0).long()[:, j // block]
    held = (j[None] < lens[:, None])[:, :, None, None]
    k, v = (torch.where(held, c[page, j % block].float(), 0.0).permute(0, 2, 3, 1).contiguous()
            for c in (s["k_cache"], s["v_cache"]))                    # [n, kv_heads, d, keys]
    i = torch.arange(s["longest"], device=q.device)
    at = (cu[:-1, None] + i).clamp(max=tokens - 1)
    qs = q.float()[at].unflatten(2, (kv_heads, heads // kv_heads)).permute(0, 2, 3, 1, 4)
    q_pos = (lens - new)[:, None, None, None, None] + i[:, None]
    seen = (j <= q_pos) & (j < lens[:, None, None, None, None])
    if s["prefix"] is not None:
        ahead = torch.minimum(s["prefix"].long(), lens)[:, None, None, None, None]
        seen = seen | (j < ahead)
    slopes = None if s["slopes"] is None else s["slopes"].view(1, kv_heads, -1, 1, 1)
    qk = torch.matmul(qs.flatten(2, 3).contiguous(), k).view(*qs.shape[:4], keys)
    x, _ = _scores(qk, q_pos, j, seen, d ** -0.5, s["cap"], slopes)
    p, _ = _weights(x, seen)
    o = torch.matmul(p.flatten(2, 3), v.transpose(2, 3).contiguous()).view(*qs.shape)
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)                        # [n, longest, heads, d]
    t = torch.arange(tokens, device=q.device)
    b = torch.bucketize(t, cu[1:], right=True)
    return o[b, t - cu[b]].to(q.dtype)


def _plain_packed(s):
    tokens, heads, d = s["q"].shape
    kv_heads = s["k"].shape[1]
    group, scale = heads // kv_heads, d ** -0.5
    q = s["q"].float().unflatten(1, (kv_heads, group)).permute(1, 2, 0, 3).contiguous()
    k, v = (s[x].float().permute(1, 0, 2)[:, None].contiguous() for x in ("k", "v"))
    i = torch.arange(tokens, device=q.device)
    doc = torch.bucketize(i, s["cu"][1:].long(), right=True)
    pos = i - s["cu"].long()[doc]
    seen = doc[:, None] == doc
    if s["causal"]:
        ahead = pos <= pos[:, None]
        if s["prefix"] is not None:
            ahead = ahead | (pos < s["prefix"].long()[doc][:, None])
        seen = seen & ahead
    slopes = None if s["slopes"] is None else s["slopes"].view(kv_heads, group, 1, 1)
    x, slope = _scores(torch.matmul(q, k.transpose(2, 3)), pos[:, None], pos, seen, scale,
                       s["cap"], slopes)
    p, lse = _weights(x, seen)
    del x
    o = torch.matmul(p, v)
    out = {"o": _tokens_first(o, s["q"]), "lse": lse.flatten(0, 1).t().contiguous()}
    if s["train"]:
        do = s["do"].float().unflatten(1, (kv_heads, group)).permute(1, 2, 0, 3).contiguous()
        dv = torch.matmul(p.transpose(2, 3), do).sum(1)
        dp = torch.matmul(do, v.transpose(2, 3))
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * slope * scale
        out["dq"] = _tokens_first(torch.matmul(ds, k), s["q"])
        out["dk"] = torch.matmul(ds.transpose(2, 3), q).sum(1).permute(1, 0, 2).to(s["k"].dtype)
        out["dv"] = dv.permute(1, 0, 2).to(s["v"].dtype)
    return out


def _tokens_first(x, like):
    return x.flatten(0, 1).permute(1, 0, 2).to(like.dtype)


# ---------------------------------------------------------------------------
# The framework's calls

def _own_slots(s):
    import paper_1904_12380_amd as sm
    return sm.softmax_cache_slots(s["ctx"], s["new"], s["table"], s["free"], s["count"],
                                  s["total"], s["block"])


def _own_append(s):
    import paper_1904_12380_amd as sm
    sm.softmax_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_paged(s):
    import paper_1904_12380_amd as sm
    return sm.softmax_paged_attention_fwd(s["q"], s["k_cache"], s["v_cache"], s["table"],
                                          s["cu_q"], s["key_lens"], cap=s["cap"],
                                          slopes=s["slopes"], prefix=s["prefix"])


def _own_packed(s):
    import paper_1904_12380_amd as sm
    how = {"causal": s["causal"], "cap": s["cap"], "slopes": s["slopes"],
           "prefix": s["prefix"] if s["causal"] else None}
    o, lse = sm.softmax_packed_attention_fwd(s["q"], s["k"], s["v"], s["cu"], **how)
    out = {"o": o, "lse": lse}
    if s["train"]:
        out["dq"], out["dk"], out["dv"] = sm.softmax_packed_attention_bwd(
            s["do"], s["q"], s["k"], s["v"], o, lse, s["cu"], **how)
    return out


def run(state):
    forms = {"slots": (_plain_slots, _own_slots), "append": (_plain_append, _own_append),
             "paged": (_plain_paged, _own_paged), "packed": (_plain_packed, _own_packed)}
    return forms[state["op"]][1 if own else 0](state)


# ---------------------------------------------------------------------------
# What a pass cannot do without

def work(case):
    op = case["op"]
    if op == "slots":
        # Lengths in, sums and lengths out, new table entries with the free
        # ids they come from, and the slots.
        ctx, new = _slot_lens(case)
        block = case["block"]
        fresh = sum(-(-(c + x) // block) - -(-c // block) for c, x in zip(ctx, new))
        return {"bytes": 16 * case["n"] + 8 * fresh + 8 * case["total"],
                "flops": 4 * case["total"]}
    if op == "append":
        return {"bytes": case["tokens"] * (4 * case["heads"] * case["d"] * SIZE[case["dtype"]] + 8),
                "flops": 0}
    h, hk, d, size = case["heads"], case["kv_heads"], case["d"], SIZE[case["dtype"]]
    if op == "paged":
        new, keys = _paged_lens(case)
        seen = _seen(new, keys, True, _prefixes(case, keys))
        table = sum(-(-x // case["block"]) for x in keys)
        return {"bytes": size * d * (2 * sum(new) * h + 2 * sum(keys) * hk) + 4 * table,
                "flops": 4 * d * h * seen}
    lens = _doc_lens(case)
    t = case["tokens"]
    seen = _seen(lens, lens, case["causal"], _prefixes(case, lens) if case["causal"] else None)
    io = size * d * t * (2 * h + 2 * hk) + 4 * t * h
    if not case["train"]:
        return {"bytes": io, "flops": 4 * d * h * seen}
    # Forward: two products.  Backward: five, from q, k, v, o, do and the
    # statistics to three gradients.
    return {"bytes": io + size * d * t * (4 * h + 4 * hk) + 4 * t * h, "flops": 14 * d * h * seen}


# ---------------------------------------------------------------------------
# The definitions in 64 bits

def _exact_append(s):
    out = {}
    slots = s["slots"].tolist()
    rows = [r for r, at in enumerate(slots) if at >= 0]
    for name in ("k", "v"):
        cache = s[name + "_cache"].double().clone()
        flat = cache.view(-1, *cache.shape[2:])
        flat.index_copy_(0, s["slots"][rows], s[name].double()[rows])
        out[name + "_cache"] = cache
    return out


def _exact_head(q, k, v, first, prefix, causal, cap, slope, do=None):
    """One head of one document: q [lq, d] at positions first.., k and v
    [lk, d], all in 64 bits."""
    scale = float(q.shape[1]) ** -0.5
    rows = torch.arange(q.shape[0], device=q.device, dtype=torch.float64)[:, None] + first
    cols = torch.arange(k.shape[0], device=q.device, dtype=torch.float64)[None, :]
    raw = q.mm(k.t()) * scale
    s = raw.div(cap).tanh_().mul_(cap) if cap else raw
    if slope:
        s = s - slope * (rows - cols).abs()
    if causal:
        s = s.masked_fill((cols > rows) & (cols >= prefix), -math.inf)
    lse = s.logsumexp(1, keepdim=True)
    p = (s - lse).exp_()
    p.masked_fill_(lse == -math.inf, 0.0)
    o = p.mm(v)
    if do is None:
        return o, lse[:, 0]
    dp = do.mm(v.t())
    ds = p * (dp - (do * o).sum(1, keepdim=True)) * scale
    if cap:
        ds *= 1.0 - (raw / cap).tanh().square()
    return o, lse[:, 0], ds.mm(k), ds.t().mm(q), p.t().mm(do)


def _exact_paged(case, s):
    new, keys = _paged_lens(case)
    pre = _prefixes(case, keys) or [0] * len(new)
    q, group = s["q"].double(), case["heads"] // case["kv_heads"]
    out = torch.empty_like(q)
    start = _sums(new)
    for b, (lq, lk) in enumerate(zip(new, keys)):
        pages = s["table"][b, :-(-lk // case["block"])].long()
        for hk in range(case["kv_heads"]):
            k, v = (c[pages, :, hk].flatten(0, 1)[:lk].double()
                    for c in (s["k_cache"], s["v_cache"]))
            for h in range(hk * group, hk * group + group):
                slope = float(s["slopes"][h]) if case["bias"] else 0.0
                at = slice(start[b], start[b] + lq)
                out[at, h] = _exact_head(q[at, h], k, v, lk - lq, pre[b], True, case["cap"],
                                         slope)[0]
    return out


def _exact_packed(case, s):
    lens = _doc_lens(case)
    pre = _prefixes(case, lens) or [0] * len(lens)
    q, k, v, do = (s[x].double() for x in ("q", "k", "v", "do"))
    group, train = case["heads"] // case["kv_heads"], case["train"]
    o, dq, dk, dv = (torch.zeros_like(x) for x in (q, q, k, v))
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    start = _sums(lens)
    for b in range(len(lens)):
        at = slice(start[b], start[b + 1])
        for h in range(case["heads"]):
            hk = h // group
            slope = float(s["slopes"][h]) if case["bias"] else 0.0
            got = _exact_head(q[at, h], k[at, hk], v[at, hk], 0, pre[b], case["causal"],
                              case["cap"], slope, do[at, h] if train else None)
            o[at, h], lse[at, h] = got[0], got[1]
            if train:
                dq[at, h] = got[2]
                dk[at, hk] += got[3]
                dv[at, hk] += got[4]
    return {"o": o, "lse": lse, **({"dq": dq, "dk": dk, "dv": dv} if train else {})}


def exact(case, seed):
    if case["op"] == "slots":
        return None
    state = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(state)
    # Many short documents cost a launch for each step of each head.
    lens = _paged_lens(case)[0] if case["op"] == "paged" else _doc_lens(case)
    if len(lens) * case["heads"] > 20000:
        return None
    return _exact_paged(case, state) if case["op"] == "paged" else _exact_packed(case, state)
