"""Multi-head attention of packed documents and of paged caches against the
float64 oracle, within the bounds that stand beside its values."""
import numpy as np
import pytest

from tests.heads_data import Packed, Paged, assert_within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = ("f32", "f16", "bf16")
TRAIN = ("o", "lse", "dq", "dk", "dv")


@pytest.fixture(scope="module")
def sm():
    import paper_1904_12380_amd
    return paper_1904_12380_amd


def self_docs(*lens):
    return [(n, n) for n in lens]


# Documents of one token, of the edges of a tile (16, 32, 64, 128 rows or
# keys), empty ones, and tokens of no document at the end.
LENS = {"one": (1,), "short": (2, 1, 0, 5, 3), "tile": (63, 64, 65), "edge": (15, 16, 17, 31, 33),
        "long": (127, 130, 0, 257), "many": tuple(range(70))}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 64), (6, 2, 128), (5, 1, 80)])
def test_packed_documents(sm, dtype, lens, heads, kv_heads, d):
    case = Packed(torch, 1, dtype, self_docs(*LENS[lens]), heads, kv_heads, d, spare=(3, 3))
    got = case.run(sm)
    assert_within(got, case.oracle(), TRAIN)
    # tokens of no document
    assert not got["o"][-3:].any() and torch.isneginf(got["lse"][-3:]).all()
    assert not got["dq"][-3:].any() and not got["dk"][-3:].any() and not got["dv"][-3:].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8, 24, 56, 64, 72, 128, 136, 192, 256])
def test_packed_head_widths(sm, dtype, d):
    case = Packed(torch, 2, dtype, self_docs(70, 33), 2, 1, d)
    assert_within(case.run(sm), case.oracle(), TRAIN)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", [
    dict(causal=False), dict(cap=5.0), dict(cap=30.0, causal=False), dict(bias=True),
    dict(bias=True, causal=False, cap=20.0), dict(prefix=[0, 40, 70, 200]),
    dict(prefix=[1, 64, 65, 66], cap=8.0, bias=True), dict(scale=0.0), dict(scale=-0.7),
    dict(scale=2.0)])
@pytest.mark.parametrize("d", [64, 128])
def test_packed_scores(sm, dtype, how, d):
    case = Packed(torch, 3, dtype, self_docs(1, 65, 140, 97), 4, 2, d, **how)
    assert_within(case.run(sm), case.oracle(), TRAIN)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("docs", [
    [(1, 300), (70, 200)],              # chunks at the end of longer keys
    [(100, 30), (5, 0), (0, 9)],        # queries before every key; no keys; no queries
    [(64, 63), (64, 65), (200, 1)]])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_keys_of_other_lengths(sm, dtype, docs, causal):
    case = Packed(torch, 4, dtype, docs, 4, 2, 64, causal=causal)
    got, want = case.run(sm), case.oracle()
    assert_within(got, want, TRAIN)
    empty = torch.from_numpy(np.isneginf(want["lse"]))
    assert torch.equal(torch.isneginf(got["lse"]).cpu(), empty)
    assert not got["o"].cpu()[empty].any() and not got["dq"].cpu()[empty].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("spread", [30.0, 1000.0])
def test_packed_large_scores(sm, dtype, spread):
    """Weights of nearly one key: the running maximum moves far."""
    case = Packed(torch, 5, dtype, self_docs(150, 80), 2, 1, 64, spread=spread)
    got = case.run(sm)
    # The gradients' bounds do not hold sums of such scores' errors apart.
    assert_within(got, case.oracle(), ("o", "lse"))
    assert all(torch.isfinite(got[x]).all() for x in ("dq", "dk", "dv"))


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_strides(sm, dtype):
    """Slices of a fused projection, heads before tokens, shared heads."""
    case = Packed(torch, 6, dtype, self_docs(33, 70), 4, 2, 64)
    want = case.run(sm)
    t = case.t
    rows = torch.cat([t[n].flatten(1) for n in ("q", "k", "v")], 1)
    q, k, v = (x.unflatten(1, (-1, 64)) for x in rows.split([256, 128, 128], 1))
    for other in (dict(q=q, k=k, v=v),
                  {n: t[n].transpose(0, 1).contiguous().transpose(0, 1)
                   for n in ("q", "k", "v", "dout")}):
        got = case.run(sm, **other)
        for name in TRAIN:
            assert torch.equal(got[name], want[name]), name
    # broadcast heads and tokens
    one = {"k": t["k"][:, :1].expand(-1, 2, -1), "dout": t["dout"][:1].expand(103, -1, -1)}
    got = case.run(sm, **one)
    want = case.run(sm, **{n: x.contiguous() for n, x in one.items()})
    for name in TRAIN:
        assert torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_documents_do_not_touch_each_other(sm, dtype):
    """NaN and infinity in one document leave the others' results alone."""
    case = Packed(torch, 7, dtype, self_docs(40, 75, 90), 4, 2, 64, spare=(5, 5))
    want = case.run(sm)
    bad = {n: x.clone() for n, x in case.t.items()}
    for n in bad:
        bad[n][40:115] = float("nan")
        bad[n][-5:] = float("inf")
    got = case.run(sm, **bad)
    for name in TRAIN:
        keep = torch.ones(len(got[name]), dtype=torch.bool)
        keep[40:115] = False
        assert torch.equal(got[name].cpu()[keep], want[name].cpu()[keep]), name
        assert name == "lse" or torch.isnan(got[name][40:115]).any(), name


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_is_deterministic_and_takes_outputs_and_streams(sm, dtype):
    case = Packed(torch, 8, dtype, self_docs(300, 41, 700), 8, 2, 128)
    want = case.run(sm)
    t, side = case.t, torch.cuda.Stream()
    out = torch.full_like(t["q"], float("nan"))
    lse = torch.full(t["q"].shape[:2], float("nan"), device="cuda")
    grads = {n: torch.full_like(t[m], float("nan")) for n, m in
             (("dq", "q"), ("dk", "k"), ("dv", "v"))}
    side.wait_stream(torch.cuda.current_stream())
    o, s = sm.softmax_packed_attention_fwd(t["q"], t["k"], t["v"], *case.cu, out=out, lse=lse,
                                           stream=side, **case.own)
    assert o is out and s is lse
    got = sm.softmax_packed_attention_bwd(t["dout"], t["q"], t["k"], t["v"], o, s, *case.cu,
                                          stream=side, **grads, **case.own)
    side.synchronize()
    for name, x in zip(TRAIN, (o, s, *got)):
        assert torch.equal(x, want[name]), name


def test_packed_gradients_against_differences(sm):
    """Directional differences of the forward pass in float32, summed in
    float64.  The difference of sum(o do) over a step of 2 h along a unit-rms
    direction has the truncation error h^2 f''' / 6 and the rounding error of
    two sums of n terms of about 2^-22 each."""
    case = Packed(torch, 9, "f32", self_docs(21, 64, 1), 4, 2, 64, cap=6.0, bias=True,
                  prefix=[3, 0, 1])
    got = case.run(sm)
    g = torch.Generator().manual_seed(3)
    h = 2.0 ** -7
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv")):
        way = torch.randn(case.t[name].shape, generator=g).cuda()
        f = [(case.run(sm, train=False, **{name: case.t[name] + s * way})["o"].double()
              * case.t["dout"].double()).sum() for s in (h, -h)]
        want = float((got[grad].double() * way.double()).sum())
        have = float((f[0] - f[1]) / (2 * h))
        n = case.t["q"].numel()
        # f''' is of the order of n^(1/2) here; 2^-22 n^(1/2) 2 / (2 h) rounding
        bound = n ** 0.5 * (h * h + 2.0 ** -22 / h) * 4
        assert abs(want - have) <= bound, (name, want, have, bound)


def test_packed_autograd(sm):
    case = Packed(torch, 10, "bf16", self_docs(50, 20), 4, 2, 64, cap=10.0)
    want = case.run(sm)
    leaves = [case.t[n].clone().requires_grad_() for n in ("q", "k", "v")]
    o = sm.softmax_packed_attention(*leaves, *case.cu, **case.own)
    assert torch.equal(o, want["o"])
    o.backward(case.t["dout"])
    for leaf, name in zip(leaves, ("dq", "dk", "dv")):
        assert torch.equal(leaf.grad, want[name]), name
    # a gradient whose last dimension is not contiguous
    for leaf in leaves:
        leaf.grad = None
    o = sm.softmax_packed_attention(*leaves, *case.cu, **case.own)
    o.sum().backward()
    assert all(torch.isfinite(leaf.grad).all() for leaf in leaves)


def test_packed_sums_out_of_range_stay_in_bounds(sm):
    """Sums past the tensors are clamped; what comes out is not specified, but
    nothing outside of the tensors is touched."""
    case = Packed(torch, 11, "bf16", self_docs(50, 30), 2, 1, 64)
    for bad in ([0, 50, 1 << 30], [0, -5, 80], [7, 90, 80], [0, 70, 20]):
        cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        guard = torch.full((3, 80, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((3, 80, 2), 7.0, device="cuda")
        sm.softmax_packed_attention_fwd(case.t["q"], case.t["k"], case.t["v"], cu,
                                        out=guard[1], lse=lse[1], **case.own)
        torch.cuda.synchronize()
        assert (guard[::2] == 7).all() and (lse[::2] == 7).all()


# ---------------------------------------------------------------------------
# Paged

REQUESTS = {
    "single": [(1, 1), (1, 17), (1, 64), (1, 0), (1, 300)],
    "long": [(1, 2500)],
    "chunks": [(40, 40), (70, 333), (3, 65), (0, 12), (129, 130)],
    "mixed": [(1, 700), (33, 1033), (1, 5), (2, 2)],
    "before": [(9, 4), (70, 1), (1, 0), (0, 0)],   # queries before every key
    "many": [(1, 3 * i + 1) for i in range(80)],
}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("requests", REQUESTS)
@pytest.mark.parametrize("heads,kv_heads,d,size", [(8, 2, 128, 16), (4, 4, 64, 8), (5, 1, 80, 64),
                                                   (16, 1, 256, 1)])
def test_paged(sm, dtype, requests, heads, kv_heads, d, size):
    case = Paged(torch, 20, dtype, REQUESTS[requests], heads, kv_heads, d, size, spare=2)
    got = case.run(sm)
    assert_within(got, case.oracle(), ("o", "lse"))
    assert not got["o"][-2:].any() and torch.isneginf(got["lse"][-2:]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", [
    dict(cap=5.0), dict(bias=True), dict(cap=20.0, bias=True, prefix=[0, 500, 64, 7]),
    dict(causal=False), dict(scale=0.5), dict(heads_first=True), dict(width=400)])
def test_paged_scores_and_layouts(sm, dtype, how):
    case = Paged(torch, 21, dtype, [(1, 900), (50, 450), (65, 65), (7, 1300)], 8, 2, 64, 32, **how)
    assert_within(case.run(sm), case.oracle(), ("o", "lse"))


@pytest.mark.parametrize("dtype", TYPES)
def test_paged_blocks_that_are_not_there(sm, dtype):
    """Table entries outside the cache hold no keys."""
    case = Paged(torch, 22, dtype, [(1, 600), (40, 300), (2, 30)], 4, 2, 64, 16)
    case.table[0, 3], case.table[0, 20], case.table[1, 0] = -1, 1 << 30, -(1 << 31)
    case.table[2, :2] = -1
    got = case.run(sm)
    assert_within(got, case.oracle(), ("o", "lse"))
    assert torch.isneginf(got["lse"][41:]).all() and not got["o"][41:].any()


def test_paged_lengths_past_the_table_are_clamped(sm):
    case = Paged(torch, 23, "bf16", [(1, 64), (3, 128)], 4, 2, 64, 16)
    want = case.run(sm)
    case.table = case.table[:, :8]
    keys, case.keys = case.keys, [64, 1 << 30]
    got = case.run(sm)
    assert torch.equal(got["o"], want["o"]) and keys == [64, 128]
    case.keys = [-5, 128]
    got = case.run(sm)
    assert not got["o"][0].any() and torch.equal(got["o"][1:], want["o"][1:])


def test_paged_offsets_past_32_bits(sm):
    """A cache of more than 2^32 elements: the blocks at its end."""
    size, heads, d = 64, 8, 128
    blocks = (1 << 32) // (size * heads * d) + 40
    cache = torch.zeros(2, blocks, size, heads, d, dtype=torch.float16, device="cuda")
    rng = np.random.default_rng(24)
    small = Paged(torch, 24, "f16", [(1, 700), (9, 130)], 16, heads, d, size)
    spots = torch.from_numpy(rng.permutation(40)[:small.t[0].shape[0]]) + blocks - 40
    for i in range(2):
        cache[i, spots.cuda()] = small.t[i]
    held = small.table >= 0
    want = small.run(sm)
    small.table[held] = spots.numpy()[small.table[held]]
    small.t = [cache[0], cache[1]]
    got = small.run(sm)
    assert torch.equal(got["o"], want["o"]) and torch.equal(got["lse"], want["lse"])
    # and the append into them
    t = torch.randn(3, heads, d, device="cuda").half()
    at = torch.tensor([blocks * size - 1, 5, (blocks - 3) * size], device="cuda")
    sm.softmax_cache_append(t, -t, cache[0], cache[1], at)
    flat = cache.flatten(1, 2)
    assert torch.equal(flat[0, at], t) and torch.equal(flat[1, at], -t)


def test_paged_graph_replays(sm):
    """Captured once, replayed with other lengths, between eager work."""
    case = Paged(torch, 25, "bf16", [(1, 3000), (1, 40), (1, 900)], 8, 2, 128, 16)
    q, table = case.q.cuda(), torch.from_numpy(case.table).to(torch.int32).cuda()
    cu = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    keys = torch.tensor(case.keys, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    run = lambda: sm.softmax_paged_attention_fwd(q, *case.t, table, cu, keys, out=out)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens in ([3000, 40, 900], [1, 39, 0], [2999, 1, 17], [256, 40, 257]):
        keys.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        run()
        assert torch.equal(out, got)
        case.keys = lens
        assert torch.equal(case.run(sm)["o"], got)


def test_paged_agrees_with_packed(sm):
    """A prompt in chunks over the cache gives what it gives at once."""
    case = Paged(torch, 26, "f32", [(200, 200)], 4, 2, 64, 16)
    pages = torch.from_numpy(case.table[0]).cuda()
    k, v = (t[pages].flatten(0, 1)[:200] for t in case.t)
    cu = torch.tensor([0, 200], dtype=torch.int32, device="cuda")
    want, _ = sm.softmax_packed_attention_fwd(case.q.cuda(), k, v, cu)
    table = torch.from_numpy(case.table).to(torch.int32).cuda()
    parts = []
    for a, b in ((0, 37), (37, 101), (101, 200)):
        parts.append(sm.softmax_paged_attention_fwd(
            case.q.cuda()[a:b], *case.t, table,
            torch.tensor([0, b - a], dtype=torch.int32, device="cuda"),
            torch.tensor([b], dtype=torch.int32, device="cuda")))
    # two orders of fp32 sums: 200 terms of weight times value
    assert (torch.cat(parts) - want).abs().max() <= 2e-5


# ---------------------------------------------------------------------------
# Longer ones: several tiles, split keys and split rows, many documents.

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("docs,heads,kv_heads,how", [
    ([(1500, 1500)], 1, 1, dict()),
    ([(1100, 1100), (70, 70)], 4, 1, dict(cap=15.0)),
    ([(1030, 1030)], 3, 1, dict(causal=False)),
    ([(700, 1300), (40, 900)], 5, 1, dict(bias=True)),
    ([(1200, 500)], 6, 2, dict(prefix=[333])),
    ([(640, 640), (641, 641)], 8, 2, dict(bias=True, cap=9.0, prefix=[500, 0]))])
def test_packed_long_documents(sm, dtype, docs, heads, kv_heads, how):
    case = Packed(torch, 40, dtype, docs, heads, kv_heads, 64, **how)
    assert_within(case.run(sm), case.oracle(), TRAIN)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count", [62, 63, 64, 65, 200])
def test_packed_many_documents(sm, dtype, count):
    """Around the 64 documents that a wavefront's lanes hold, and more."""
    lens = np.random.default_rng(count).integers(0, 30, count)
    lens[count // 2] = 300
    case = Packed(torch, 41, dtype, self_docs(*(int(n) for n in lens)), 4, 2, 64, spare=(1, 1))
    assert_within(case.run(sm), case.oracle(), TRAIN)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cap", [256.0, 257.0, 3000.0, 1e6, 1e-3])
def test_packed_caps_of_all_sizes(sm, dtype, cap):
    case = Packed(torch, 42, dtype, self_docs(90, 40), 2, 1, 64, cap=cap, spread=4.0)
    want = case.oracle()
    # the bound's term for the cap is for caps of the scores' size
    if cap > 256.0:
        want = {**case_with_cap(case, 0.0), **{n: want[n] for n in ("o", "lse", "dq", "dk", "dv")}}
    assert_within(case.run(sm), want, TRAIN)


def case_with_cap(case, cap):
    kept = case.ref["cap"]
    case.ref["cap"] = cap
    bounds = {n: x for n, x in case.oracle().items() if n.startswith("e_")}
    case.ref["cap"] = kept
    return bounds


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_nothing_on_one_side(sm, dtype):
    """No documents, no queries, no keys: zeros, and no read of what is not
    there."""
    t = torch.randn(7, 2, 64, device="cuda").to({"f32": torch.float32, "f16": torch.float16,
                                                 "bf16": torch.bfloat16}[dtype])
    none, lse0 = t[:0], torch.empty(0, 2, device="cuda")
    zero = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    seven = torch.tensor([0, 7], dtype=torch.int32, device="cuda")
    o, lse = sm.softmax_packed_attention_fwd(t, t, t, zero[:1])
    assert not o.any() and torch.isneginf(lse).all()
    grads = sm.softmax_packed_attention_bwd(t, t, t, t, o, lse, zero[:1])
    assert not any(g.any() for g in grads)
    o, lse = sm.softmax_packed_attention_fwd(t, none, none, seven, zero)
    assert not o.any() and torch.isneginf(lse).all()
    dq, dk, dv = sm.softmax_packed_attention_bwd(t, t, none, none, o, lse, seven, zero)
    assert not dq.any() and dk.numel() == dv.numel() == 0
    o, lse = sm.softmax_packed_attention_fwd(none, t, t, zero, seven)
    assert o.numel() == lse.numel() == 0
    dq, dk, dv = sm.softmax_packed_attention_bwd(none, none, t, t, none, lse0, zero, seven)
    assert dq.numel() == 0 and not dk.any() and not dv.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_infinities_reach_their_own_rows(sm, dtype):
    case = Packed(torch, 43, dtype, self_docs(150), 2, 1, 64)
    want = case.run(sm, train=False)["o"]
    q = case.t["q"].clone()
    q[70, 1, 3] = float("inf")
    got = case.run(sm, train=False, q=q)["o"]
    assert torch.isnan(got[70, 1]).all()
    keep = torch.ones(150, 2, dtype=torch.bool, device="cuda")
    keep[70, 1] = False
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("requests,heads,kv_heads,size", [
    ([(1, 9000)], 8, 1, 16),                       # many splits
    ([(1, 5000), (1, 3), (200, 4100)], 8, 2, 64),  # splits beside chunks
    ([(1, 100)] * 130, 4, 1, 32),                  # more requests than lanes
    ([(5, 2000), (0, 700), (1, 1999)], 16, 2, 128)])
def test_paged_long(sm, dtype, requests, heads, kv_heads, size):
    case = Paged(torch, 44, dtype, requests, heads, kv_heads, 64, size)
    assert_within(case.run(sm), case.oracle(), ("o", "lse"))


def test_refusals(sm):
    q = torch.randn(10, 4, 64, device="cuda").bfloat16()
    k = torch.randn(10, 2, 64, device="cuda").bfloat16()
    cu = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    fwd = sm.softmax_packed_attention_fwd
    fwd(q, k, k, cu)
    for bad in (dict(k=k.float()), dict(k=k.cpu()), dict(cu_q=cu.long()), dict(q=q.double()),
                dict(slopes=torch.ones(4, device="cuda").half()),
                dict(out=torch.empty_like(q).float())):
        with pytest.raises((TypeError, ValueError)):
            fwd(**{**dict(q=q, k=k, v=k, cu_q=cu), **bad})
    for bad in (dict(q=q[0]), dict(q=q.transpose(1, 2)), dict(cu_q=cu[:0]), dict(k=k[:9], v=k[:9]),
                dict(slopes=torch.ones(3, device="cuda")), dict(prefix=cu),
                dict(out=torch.empty(10, 4, 63, device="cuda").bfloat16()),
                dict(lse=torch.empty(4, 10, device="cuda").t())):
        with pytest.raises(ValueError):
            fwd(**{**dict(q=q, k=k, v=k, cu_q=cu), **bad})
    for bad in (dict(scale=float("nan")), dict(cap=-2.0), dict(out=q),
                dict(q=q[..., :60], k=k[..., :60], v=k[..., :60]),
                dict(q=q.flatten()[4:4 + 9 * 256].view(9, 4, 64), k=k[:9], v=k[:9]),
                dict(causal=False, prefix=cu[:1])):
        with pytest.raises(sm.SoftmaxError) as e:
            fwd(**{**dict(q=q, k=k, v=k, cu_q=cu), **bad})
        assert e.value.code == sm.ERR_INVALID_ARG
    pinned = torch.empty(4, dtype=torch.int32)       # pageable host memory behind a pointer
    assert sm.load_library().softmax_cache_slots(
        cu.data_ptr(), cu.data_ptr(), 2, q.data_ptr(), 1, pinned.data_ptr(), 4, cu.data_ptr(), 16,
        k.data_ptr(), k.data_ptr() + 64, k.data_ptr() + 128, 1, k.data_ptr() + 256,
        k.data_ptr() + 320, None) == sm.ERR_NOT_DEVICE
    with pytest.raises(ValueError):
        sm.softmax_packed_attention(q, k, k, cu, slopes=torch.ones(4, device="cuda",
                                                                   requires_grad=True))


def test_gradients_of_any_layout(sm):
    """autograd hands the gradient on as the operation behind left it: slices
    whose rows are not whole 16-byte strips, and expanded ones."""
    case = Packed(torch, 21, "bf16", self_docs(33, 7), 4, 2, 64)
    leaves = [case.t[n].clone().requires_grad_() for n in ("q", "k", "v")]
    wide = torch.randn(40, 4 * 64 + 3, device="cuda").bfloat16()
    for dout in (wide[:, 1:257].unflatten(1, (4, 64)), wide[:, 3:].unflatten(1, (4, 64)),
                 wide[:1, :1, None].expand(40, 4, 64)):
        o = sm.softmax_packed_attention(*leaves, *case.cu, **case.own)
        got = torch.autograd.grad(o, leaves, dout)
        o, lse = sm.softmax_packed_attention_fwd(*[case.t[n] for n in ("q", "k", "v")], *case.cu,
                                                 **case.own)
        want = sm.softmax_packed_attention_bwd(
            dout.contiguous(), *[case.t[n] for n in ("q", "k", "v")], o, lse, *case.cu,
            **case.own)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_gradients_have_no_gradient_of_their_own(sm):
    case = Packed(torch, 22, "f32", self_docs(9,), 2, 2, 16)
    leaves = [case.t[n].clone().requires_grad_() for n in ("q", "k", "v")]
    o = sm.softmax_packed_attention(*leaves, *case.cu, **case.own)
    dq, = torch.autograd.grad(o.sum(), leaves[:1], create_graph=True)
    with pytest.raises(RuntimeError):
        dq.sum().backward()


def test_paged_sums_out_of_order_stay_in_bounds(sm):
    """Sums that do not ascend, in a call that is split: what comes out is not
    specified, but nothing outside of the tensors is touched."""
    case = Paged(torch, 23, "bf16", [(300, 3000), (1, 900), (2, 2000)], 2, 1, 64, 16)
    table = torch.from_numpy(case.table).to(torch.int32).cuda()
    keys = torch.tensor(case.keys, dtype=torch.int32, device="cuda")
    for bad in ([0, 300, 1, 303], [0, 303, 2, 1], [5, 0, 1 << 30, 7]):
        cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        guard = torch.full((3, 303, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        sm.softmax_paged_attention_fwd(case.q.cuda(), *case.t, table, cu, keys, out=guard[1],
                                       **case.own)
        torch.cuda.synchronize()
        assert (guard[::2] == 7).all()


def test_training_and_serving_steps_in_graphs(sm):
    """Each replay against the eager calls, with other inputs and eager work in
    between."""
    case = Packed(torch, 24, "bf16", self_docs(300, 41, 700), 8, 2, 128, cap=20.0)
    size, n = 16, 3
    caches = torch.zeros(2, 64, size, 2, 128, dtype=torch.bfloat16, device="cuda")
    table = torch.full((n, 16), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(64, device="cuda").int()
    left = torch.tensor([64], dtype=torch.int32, device="cuda")
    held = torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda")
    new = torch.tensor([5, 1, 2], dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros(8, h, 128, dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))

    def serve(caches, table, left, held):
        s = sm.softmax_cache_slots(held, new, table, free, left, 8, size)
        sm.softmax_cache_append(k, v, caches[0], caches[1], s["slots"])
        o = sm.softmax_paged_attention_fwd(q, caches[0], caches[1], table, s["cu_q"],
                                           s["key_lens"])
        held.copy_(s["key_lens"])
        left.copy_(s["free_count"])
        return o

    own = (caches.clone(), table.clone(), left.clone(), held.clone())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = case.run(sm)
        o = serve(*own)
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (q, k, v, *(case.t[name] for name in ("q", "k", "v", "dout"))):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        want, served = case.run(sm), serve(caches, table, left, held)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[name], want[name]) for name in want)
        assert torch.equal(o, served) and torch.equal(own[1], table)
        assert torch.equal(own[0], caches) and torch.equal(own[3], held)
    assert held.tolist() == [20, 4, 8]
