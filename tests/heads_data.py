"""Inputs of the multi-head attention tests, and the comparison with the
oracle's values and bounds."""
import numpy as np

import oracle.heads_f64 as ref


def types(torch):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def sums(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def draw(torch, rng, dtype, *shape, scale=1.0):
    """A tensor of the type, and its values in float64."""
    t = torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32))
    t = t.to(types(torch)[dtype])
    return t, t.double().numpy()


def assert_within(got, out, names):
    for name in names:
        value, want, bound = got[name].double().cpu().numpy(), out[name], out["e_" + name]
        assert value.shape == want.shape, name
        same = np.isneginf(want) & np.isneginf(value)
        with np.errstate(invalid="ignore"):
            excess = np.where(same, -1.0, np.abs(value - want) - bound)
        assert not np.isnan(excess).any(), f"{name}: NaN"
        worst = np.unravel_index(np.argmax(excess), excess.shape) if excess.size else None
        assert excess.size == 0 or excess[worst] <= 0, (
            f"{name}{list(worst)}: {value[worst]} against {want[worst]}, bound {bound[worst]}")


def slopes_of(heads):
    return np.array([2.0 ** (-8.0 * (i + 1) / heads) for i in range(heads)], np.float32)


def to_i32(torch, x):
    return torch.tensor([int(i) for i in x], dtype=torch.int32)


class Packed:
    """Packed documents of the given (queries, keys) lengths, on the GPU and
    in float64."""

    def __init__(self, torch, seed, dtype, docs, heads, kv_heads, d, *, spare=(0, 0), scale=None,
                 cap=0.0, bias=False, causal=True, prefix=None, spread=1.0):
        rng = np.random.default_rng(seed)
        lq, lk = [a for a, _ in docs], [b for _, b in docs]
        self.cu_q, self.cu_k = sums(lq), sums(lk)
        tq, tk = int(self.cu_q[-1]) + spare[0], int(self.cu_k[-1]) + spare[1]
        made = {"q": draw(torch, rng, dtype, tq, heads, d, scale=spread),
                "k": draw(torch, rng, dtype, tk, kv_heads, d),
                "v": draw(torch, rng, dtype, tk, kv_heads, d),
                "dout": draw(torch, rng, dtype, tq, heads, d)}
        self.t = {n: x[0].cuda() for n, x in made.items()}
        self.f = {n: x[1] for n, x in made.items()}
        self.dtype = dtype
        self.how = dict(scale=scale, cap=cap, causal=causal)
        slopes = slopes_of(heads) if bias else None
        self.ref = dict(slopes=slopes, prefix=prefix, **self.how)
        self.own = dict(slopes=None if slopes is None else torch.from_numpy(slopes).cuda(),
                        prefix=None if prefix is None else to_i32(torch, prefix).cuda(),
                        **self.how)
        self.cu = (to_i32(torch, self.cu_q).cuda(), to_i32(torch, self.cu_k).cuda())

    def oracle(self, train=True):
        f = self.f
        return ref.packed(f["q"], f["k"], f["v"], self.cu_q, self.cu_k, dtype=self.dtype,
                          dout=f["dout"] if train else None, **self.ref)

    def run(self, sm, train=True, **tensors):
        t = {**self.t, **tensors}
        o, lse = sm.softmax_packed_attention_fwd(t["q"], t["k"], t["v"], *self.cu, **self.own)
        got = {"o": o, "lse": lse}
        if train:
            got["dq"], got["dk"], got["dv"] = sm.softmax_packed_attention_bwd(
                t["dout"], t["q"], t["k"], t["v"], o, lse, *self.cu, **self.own)
        return got


class Paged:
    """Requests of the given (new tokens, keys) over a shuffled paged cache.
    Slots that hold no key are NaN."""

    def __init__(self, torch, seed, dtype, requests, heads, kv_heads, d, size, *, spare=0,
                 width=0, heads_first=False, scale=None, cap=0.0, bias=False, causal=True,
                 prefix=None):
        rng = np.random.default_rng(seed)
        new, keys = [a for a, _ in requests], [b for _, b in requests]
        self.cu_q, self.keys = sums(new), keys
        held = [-(-x // size) for x in keys]
        width = max([width, 1] + held)
        ids = rng.permutation(sum(held) + 2)
        blocks = len(ids)
        self.table = np.full((len(requests), width), -1, np.int64)
        self.q, self.fq = draw(torch, rng, dtype, int(self.cu_q[-1]) + spare, heads, d)
        caches = [draw(torch, rng, dtype, blocks, size, kv_heads, d) for _ in range(2)]
        live = np.zeros((blocks, size), bool)
        at = 0
        for b, x in enumerate(keys):
            self.table[b, :held[b]] = ids[at:at + held[b]]
            at += held[b]
            j = np.arange(x)
            live[self.table[b, j // size], j % size] = True
        dead = torch.from_numpy(~live)
        self.f, self.t = [], []
        for t, f in caches:
            t[dead] = float("nan")
            f[~live] = np.nan
            t = t.cuda()
            if heads_first:  # [blocks, heads, size, d] in memory
                t = t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            self.t.append(t)
            self.f.append(f)
        slopes = slopes_of(heads) if bias else None
        self.dtype = dtype
        how = dict(scale=scale, cap=cap, causal=causal)
        self.ref = dict(slopes=slopes, prefix=prefix, **how)
        self.own = dict(slopes=None if slopes is None else torch.from_numpy(slopes).cuda(),
                        prefix=None if prefix is None else to_i32(torch, prefix).cuda(), **how)
        self.torch = torch

    def oracle(self):
        return ref.paged(self.fq, *self.f, self.table, self.cu_q, self.keys, dtype=self.dtype,
                         **self.ref)

    def run(self, sm, **more):
        torch = self.torch
        lse = torch.empty(self.fq.shape[:2], device="cuda")
        o = sm.softmax_paged_attention_fwd(
            self.q.cuda(), *self.t, torch.from_numpy(self.table).to(torch.int32).cuda(),
            to_i32(torch, self.cu_q).cuda(), to_i32(torch, self.keys).cuda(), lse=lse,
            **self.own, **more)
        return {"o": o, "lse": lse}
