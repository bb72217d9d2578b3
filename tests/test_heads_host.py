"""Multi-head attention and the paged cache without a GPU: the entry points
refuse bad arguments before any HIP call, the binding refuses bad tensors, and
the oracle agrees with sums over single pairs, differences and invariants."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

import oracle.heads_f64 as ref
import paper_1904_12380_amd as sm
from paper_1904_12380_amd import attention as at

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "attention_mi355x.h")).read()
P = [i << 32 for i in range(1, 20)]      # far apart, never dereferenced
BAD = sm.ERR_INVALID_ARG


def heads(i, tokens=100, n=4, d=64, ts=None, hs=None):
    return at._Heads(P[i], tokens, n, d, n * d if ts is None else ts, d if hs is None else hs)


def cache(i, blocks=10, size=16, n=2, d=64, ts=None):
    return at._Cache(P[i], blocks, size, n, d, size * n * d, n * d if ts is None else ts, d)


def score(scale=0.125, cap=0.0, causal=1, slopes=None, prefix=None):
    return at._Score(scale, cap, causal, slopes, prefix)


def fwd(q=None, k=None, v=None, o=P[3], lse=P[4], cu=P[5], docs=2, sc=None, dtype=2):
    fn = sm.load_library().softmax_packed_attention_fwd
    return fn(q or heads(0), k or heads(1, n=2), v or heads(2, n=2), o, lse, cu, cu, docs,
              sc or score(), dtype, None)


def bwd(q=None, k=None, v=None, o=None, dout=None, dq=P[8], room=1 << 30, work=P[11], dtype=2,
        sc=None):
    fn = sm.load_library().softmax_packed_attention_bwd
    return fn(dout or heads(6), q or heads(0), k or heads(1, n=2), v or heads(2, n=2),
              o or heads(3), P[4], dq, P[9], P[10], P[5], P[5], 2, sc or score(), dtype, work,
              room, None)


def paged(q=None, k=None, v=None, width=4, requests=3, sc=None, dtype=2, o=P[3], cu=P[5]):
    fn = sm.load_library().softmax_paged_attention_fwd
    return fn(q or heads(0), k or cache(1), v or cache(2), P[6], width, cu, P[7], requests,
              sc or score(), dtype, o, None, P[8], 1 << 40, None)


def test_header_and_binding_agree():
    for name, value in (("HEADS_MAX_DIM", sm.HEADS_MAX_DIM), ("F32", 0), ("F16", 1), ("BF16", 2)):
        assert re.search(rf"#define SOFTMAX_{name} (\d+)", HEADER).group(1) == str(value)
    for name in ("softmax_packed_attention_fwd", "softmax_packed_attention_bwd",
                 "softmax_paged_attention_fwd", "softmax_cache_slots", "softmax_cache_append"):
        assert re.search(rf"SOFTMAX_API int {name}\(", HEADER) and name in sm.__all__


LAYOUTS = [dict(tokens=-1), dict(d=7), dict(d=4), dict(d=264), dict(d=0), dict(ts=260),
           dict(hs=68), dict(ts=-256), dict(ts=(1 << 23) + 8), dict(hs=-64), dict(n=-1),
           dict(tokens=(1 << 30) + 1), dict(hs=1 << 62)]


@pytest.mark.parametrize("layout", LAYOUTS)
def test_layouts_are_refused(layout):
    for dtype in (1, 2):
        assert fwd(q=heads(0, **layout), dtype=dtype) == BAD
        assert fwd(k=heads(1, **{"n": 2, **layout}), v=heads(2, **{"n": 2, **layout}),
                   dtype=dtype) == BAD
        assert bwd(dout=heads(6, **layout), dtype=dtype) == BAD
        assert paged(q=heads(0, **layout), dtype=dtype) == BAD
    odd = heads(0)
    odd.data = P[0] + 8                      # not 16-byte aligned
    assert fwd(q=odd) == BAD and bwd(q=odd) == BAD and paged(q=odd) == BAD


def test_shapes_that_do_not_match_are_refused():
    assert fwd(k=heads(1, n=3), v=heads(2, n=3)) == BAD          # 4 heads over 3
    assert fwd(k=heads(1, n=2, tokens=99)) == BAD                # k and v differ
    assert fwd(k=heads(1, n=2, d=72), v=heads(2, n=2, d=72)) == BAD
    assert fwd(k=heads(1, n=0), v=heads(2, n=0)) == BAD
    assert fwd(docs=-1) == BAD
    assert bwd(o=heads(3, tokens=99)) == BAD and bwd(dout=heads(6, n=2)) == BAD
    assert paged(k=cache(1, size=12), v=cache(2, size=12)) == BAD     # no power of two
    assert paged(k=cache(1, size=0), v=cache(2, size=0)) == BAD
    assert paged(v=cache(2, blocks=9)) == BAD and paged(v=cache(2, n=4)) == BAD
    assert paged(k=cache(1, ts=100), v=cache(2, ts=100)) == BAD       # not whole strips
    assert paged(width=-1) == BAD and paged(requests=-1) == BAD
    assert paged(width=(1 << 27)) == BAD                              # 2^31 keys
    assert paged(q=heads(0, n=3)) == BAD


@pytest.mark.parametrize("sc", [
    dict(scale=math.nan), dict(scale=math.inf), dict(cap=-1.0), dict(cap=math.nan),
    dict(cap=math.inf), dict(cap=1e-31), dict(causal=2), dict(causal=0, prefix=P[9])])
def test_scores_are_refused(sc):
    assert fwd(sc=score(**sc)) == BAD
    assert bwd(sc=score(**sc)) == BAD
    assert paged(sc=score(**sc)) == BAD


def test_pointers_types_and_workspaces_are_refused():
    lib = sm.load_library()
    assert fwd(dtype=3) == BAD and bwd(dtype=-1) == BAD and paged(dtype=9) == BAD
    assert fwd(o=P[0] + 16) == BAD                   # o overlaps q
    assert fwd(o=P[3] + 8) == BAD                    # misaligned
    assert fwd(lse=P[3] + 64) == BAD                 # lse overlaps o
    assert fwd(o=None) == BAD and fwd(cu=None) == BAD and fwd(lse=None) == BAD
    assert bwd(room=100) == BAD                      # too little workspace
    assert bwd(work=P[11] + 4) == BAD and bwd(dq=P[1]) == BAD
    assert lib.softmax_packed_attention_fwd(None, heads(1), heads(2), P[3], P[4], P[5], P[5], 2,
                                            score(), 2, None) == BAD
    assert lib.softmax_packed_attention_fwd(heads(0), heads(1), heads(2), P[3], P[4], P[5], P[5],
                                            2, None, 2, None) == BAD
    # nothing to do
    none = heads(0, tokens=0)
    none.data = None
    assert fwd(q=none) == sm.OK and paged(q=none) == sm.OK


def test_workspace_sizes():
    lib = sm.load_library()
    size = lib.softmax_packed_attention_bwd_workspace
    assert size(100, 100, 4, 2, 64, 0) == 8 * 400            # fp32: the statistics alone
    assert size(0, 100, 4, 2, 64, 2) == 0
    assert size(1 << 14, 1 << 14, 16, 2, 128, 2) > 8 * (1 << 18)
    for bad in ((-1, 100, 4, 2, 64, 2), (100, 100, 4, 3, 64, 2), (100, 100, 4, 2, 7, 2),
                (100, 100, 4, 2, 64, 5), (1 << 30, 100, 4, 2, 64, 2), (100, 100, 4, 0, 64, 2)):
        assert size(*bad) == -1


def slots(requests=3, width=4, capacity=5, size=16, total=7, out=P[8], table=P[3]):
    return sm.load_library().softmax_cache_slots(
        P[1], P[2], requests, table, width, P[4], capacity, P[5], size, P[6], P[7], out, total,
        P[9], P[10], None)


def append(k=None, v=None, kc=None, vc=None, at_=P[5], dtype=2):
    return sm.load_library().softmax_cache_append(
        k or heads(0, n=2), v or heads(1, n=2), kc or cache(2), vc or cache(3), at_, dtype, None)


def test_cache_arguments_are_refused():
    assert slots(requests=-1) == BAD and slots(requests=65537) == BAD
    assert slots(width=-1) == BAD and slots(capacity=-1) == BAD and slots(total=-1) == BAD
    assert slots(size=0) == BAD and slots(size=24) == BAD
    assert slots(out=P[1] + 4) == BAD                 # slots over context_lens
    assert slots(table=P[8]) == BAD                   # outputs over each other
    assert slots(out=None) == BAD
    assert append(k=heads(0, n=4)) == BAD             # heads of the cache
    assert append(v=heads(1, n=2, tokens=9)) == BAD
    assert append(kc=cache(2, size=3)) == BAD and append(vc=cache(3, blocks=9)) == BAD
    assert append(at_=None) == BAD and append(dtype=4) == BAD
    assert append(kc=cache(0)) == BAD                 # the cache over k
    none = heads(0, n=2, tokens=0)
    assert append(k=none, v=none) == sm.OK


def test_cpu_tensors_and_wrong_types_are_refused():
    torch = pytest.importorskip("torch")
    q = torch.zeros(5, 2, 64)
    cu = torch.tensor([0, 5], dtype=torch.int32)
    with pytest.raises(ValueError):
        sm.softmax_packed_attention_fwd(q, q, q, cu)
    with pytest.raises(TypeError):
        sm.softmax_packed_attention_fwd([1.0], q, q, cu)
    with pytest.raises(ValueError):
        sm.softmax_cache_slots(cu, cu, torch.zeros(2, 3, dtype=torch.int32), cu, cu, 3, 16)
    with pytest.raises(ValueError):
        sm.softmax_cache_append(q, q, q[None], q[None], cu)


# ---------------------------------------------------------------------------
# The oracle

HOW = [dict(), dict(causal=False), dict(cap=2.0), dict(slope=0.3), dict(prefix=4),
       dict(cap=3.0, slope=0.1, prefix=2)]


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("lq,lk", [(5, 5), (3, 7), (6, 2)])
def test_oracle_against_sums_over_pairs(how, lq, lk):
    rng = np.random.default_rng(1)
    d = 8
    q, k, v = (rng.standard_normal((n, d)) for n in (lq, lk, lk))
    got = ref.head(q, k, v, dtype="f32", scale=0.4, **how)
    for i in range(lq):
        pos, terms = i + lk - lq, []
        for j in range(lk):
            if how.get("causal", True) and j > pos and j >= how.get("prefix", 0):
                continue
            x = 0.4 * sum(float(q[i, c]) * float(k[j, c]) for c in range(d))
            if "cap" in how:
                x = how["cap"] * math.tanh(x / how["cap"])
            terms.append((x - how.get("slope", 0.0) * abs(pos - j), j))
        if not terms:
            assert got["lse"][i] == -np.inf and not got["o"][i].any()
            continue
        total = math.fsum(math.exp(x) for x, _ in terms)
        assert abs(got["lse"][i] - math.log(total)) < 1e-12
        want = sum(math.exp(x) / total * v[j] for x, j in terms)
        assert np.abs(got["o"][i] - want).max() < 1e-12


@pytest.mark.parametrize("how", HOW)
def test_oracle_gradients_against_differences(how):
    rng = np.random.default_rng(2)
    lq, lk, d, h = 4, 6, 8, 1e-5
    x = {n: rng.standard_normal((m, d)) for n, m in (("q", lq), ("k", lk), ("v", lk))}
    dout = rng.standard_normal((lq, d))
    run = lambda y: float((ref.head(y["q"], y["k"], y["v"], dtype="f32", scale=0.4,  # noqa: E731
                                    **how)["o"] * dout).sum())
    got = ref.head(x["q"], x["k"], x["v"], dtype="f32", scale=0.4, dout=dout, **how)
    for name in x:
        for at_ in np.ndindex(x[name].shape):
            up, down = ({**x, name: x[name].copy()} for _ in range(2))
            up[name][at_] += h
            down[name][at_] -= h
            assert abs((run(up) - run(down)) / (2 * h) - got["d" + name][at_]) < 1e-8


def test_oracle_invariants():
    rng = np.random.default_rng(3)
    q, k, v, dout = (rng.standard_normal((9, 16)) for _ in range(4))
    one = ref.head(q, k, v, dtype="f32", scale=0.2, dout=dout)
    # a shift of all keys along one vector shifts every score of a row alike
    moved = ref.head(q, k + 0.5, v, dtype="f32", scale=0.2, dout=dout)
    assert np.abs(one["o"] - moved["o"]).max() < 1e-12
    # constant values come back, and leave no gradient in q and k
    flat = ref.head(q, k, np.ones_like(v), dtype="f32", scale=0.2, dout=dout)
    assert np.abs(flat["o"] - 1).max() < 1e-12
    assert np.abs(flat["dq"]).max() < 1e-12 and np.abs(flat["dk"]).max() < 1e-12
    # every weight is given out once
    assert np.abs(one["dv"].sum(0) - dout.sum(0)).max() < 1e-12
    # a paged cache is its gathered keys
    cu = ref.packed(q[:, None], k[:, None], v[:, None], [0, 9], [0, 9], dtype="f32", scale=0.2)
    pages = np.array([[2, 0, 1]])
    pad = np.concatenate([k, np.full((3, 16), np.nan)]).reshape(3, 4, 1, 16)
    vad = np.concatenate([v, np.full((3, 16), np.nan)]).reshape(3, 4, 1, 16)
    order = [1, 2, 0]
    got = ref.paged(q[:, None], pad[order], vad[order], pages, [0, 9], [9], dtype="f32", scale=0.2)
    assert np.array_equal(got["o"], cu["o"]) and np.array_equal(got["lse"], cu["lse"])


def test_oracle_slots_by_hand():
    # 3 requests with blocks of 4: 5 + 2 tokens, 0 + 5, 4 + 0; 2 free blocks
    table = np.array([[7, 3, -1], [-1, -1, -1], [5, -1, -1]])
    got = ref.cache_slots([5, 0, 4], [2, 5, 0], table, [9, 8], 2, 8, 4)
    assert got["cu_q"].tolist() == [0, 2, 7, 7] and got["key_lens"].tolist() == [7, 5, 4]
    assert got["table"].tolist() == [[7, 3, -1], [8, 9, -1], [5, -1, -1]]
    assert got["slots"].tolist() == [13, 14, 32, 33, 34, 35, 36, -1]
    assert got["free_count"].tolist() == [0] and got["missing"].tolist() == [0]
    short = ref.cache_slots([5, 0, 4], [2, 5, 1], table, [9, 8], 1, 8, 4)
    # one id on the stack: its lowest entry
    assert short["table"].tolist() == [[7, 3, -1], [9, -1, -1], [5, -1, -1]]
    assert short["slots"].tolist() == [13, 14, 36, 37, 38, 39, -1, -1]
    assert short["missing"].tolist() == [2]


def test_oracle_bounds_hold_for_rounded_weights():
    """The bounds cover a float32 computation with weights and score gradients
    rounded to float16, which is what they are for."""
    rng = np.random.default_rng(4)
    f = np.float32
    q, k, v, do = (rng.standard_normal((70, 32)).astype(np.float16) for _ in range(4))
    want = ref.head(q, k, v, dtype="f16", scale=0.17, dout=do)
    x = f(0.17) * (q.astype(f) @ k.astype(f).T)
    x[np.triu_indices(70, 1)] = -np.inf
    e = np.exp(x - x.max(1, keepdims=True))
    p = e / e.sum(1, keepdims=True)
    o = (p.astype(np.float16).astype(f) @ v.astype(f)).astype(np.float16)
    delta = (o.astype(f) * do.astype(f)).sum(1, keepdims=True)
    ds = (p * (do.astype(f) @ v.astype(f).T - delta)).astype(np.float16).astype(f)
    got = {"o": o, "dv": p.astype(np.float16).astype(f).T @ do.astype(f),
           "dq": f(0.17) * ds @ k.astype(f), "dk": f(0.17) * ds.T @ q.astype(f)}
    for name, value in got.items():
        off = np.abs(value.astype(np.float16).astype(np.float64) - want[name])
        assert (off <= want["e_" + name]).all(), name


def test_structs_match_the_header():
    """Field order and sizes of the structs, as a C compiler lays them out."""
    for struct, name in ((at._Heads, "softmax_heads_t"), (at._Cache, "softmax_cache_t"),
                         (at._Score, "softmax_score_t")):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), HEADER, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = re.findall(r"(\w+)\s*;", body)
        assert fields == [n for n, _ in struct._fields_]
    assert ctypes.sizeof(at._Heads) == 48 and ctypes.sizeof(at._Cache) == 64
    assert ctypes.sizeof(at._Score) == 32
