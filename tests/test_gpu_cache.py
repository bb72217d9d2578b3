"""The paged cache's bookkeeping and appends against the oracle."""
import numpy as np
import pytest

import oracle.heads_f64 as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sm():
    import paper_1904_12380_amd
    return paper_1904_12380_amd


def state(rng, n, context, new, size, width, spare):
    ctx = rng.integers(0, context + 1, n)
    fresh = rng.integers(0, new + 1, n)
    held = np.minimum(-(-ctx // size), width)
    ids = rng.permutation(int(held.sum()) + 4096)
    table = np.full((n, width), -1, np.int64)
    at = 0
    for b in range(n):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    return ctx, fresh, table, ids[at:at + max(spare, 1)], spare


def check(sm, ctx, fresh, table, free, count, total, size):
    want = ref.cache_slots(ctx, fresh, table, free, count, total, size)
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(torch.int32).cuda()  # noqa: E731
    got = sm.softmax_cache_slots(i32(ctx), i32(fresh), i32(table), i32(free),
                                 i32(np.array([count])), total, size)
    for name, x in want.items():
        assert np.array_equal(got[name].cpu().numpy(), x), name


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 256, 257, 700, 1500])
@pytest.mark.parametrize("size,new", [(16, 1), (8, 40), (1, 3), (64, 200)])
def test_slots(sm, n, size, new):
    rng = np.random.default_rng(n)
    args = state(rng, n, 150, new, size, -(-400 // size), 200 * n // size + n)
    total = int(args[1].sum())
    check(sm, *args, total, size)
    check(sm, *args, total + 77, size)       # padded
    check(sm, *args, total // 2, size)       # fewer slots than tokens


@pytest.mark.parametrize("spare", [0, 1, 13, 100])
def test_slots_of_a_pool_that_runs_out(sm, spare):
    rng = np.random.default_rng(spare)
    args = state(rng, 40, 100, 60, 16, 12, spare)
    check(sm, *args, int(args[1].sum()), 16)


def test_slots_past_the_table(sm):
    rng = np.random.default_rng(5)
    args = state(rng, 30, 100, 90, 16, 5, 300)   # tables of 80 tokens
    check(sm, *args, int(args[1].sum()), 16)


def test_slots_odd_inputs(sm):
    rng = np.random.default_rng(6)
    ctx, fresh, table, free, count = state(rng, 9, 50, 20, 8, 20, 60)
    fresh[:] = 0
    check(sm, ctx, fresh, table, free, count, 0, 8)        # nothing new
    check(sm, ctx, fresh, table, free, count, 5, 8)
    fresh[4] = 70
    check(sm, ctx, fresh, table, free, count, 70, 8)       # one request alone
    ctx[2], fresh[3] = -9, -4                              # count as zero
    check(sm, ctx, fresh, table, free, count, 70, 8)
    check(sm, ctx, fresh, table, free, 10 ** 6, 70, 8)     # more free than the list holds
    check(sm, ctx, fresh, table, free, -3, 70, 8)
    # no requests
    check(sm, ctx[:0], fresh[:0], table[:0], free, count, 4, 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens,heads,d,size", [(1, 1, 8, 1), (7, 3, 80, 16), (300, 8, 128, 64),
                                                 (65, 2, 256, 8), (0, 2, 64, 16)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_append(sm, dtype, tokens, heads, d, size, heads_first):
    g = torch.Generator().manual_seed(tokens)
    rows = torch.randn(tokens, 3 * heads * d, generator=g).to(dtype).cuda()
    k, v = (x.unflatten(1, (heads, d)) for x in rows.split(heads * d, 1)[:2])
    blocks = 2 * tokens // size + 3
    caches = torch.randn(2, blocks, size, heads, d, generator=g).to(dtype).cuda()
    slots = torch.randperm(blocks * size, generator=g)[:tokens]
    slots[::5] = -1
    if tokens > 8:
        slots[3], slots[6] = blocks * size, 1 << 40      # past the cache: skipped
    want = caches.clone()
    for t in range(tokens):
        if 0 <= slots[t] < blocks * size:
            want[0, slots[t] // size, slots[t] % size] = k[t]
            want[1, slots[t] // size, slots[t] % size] = v[t]
    if heads_first:
        caches = caches.transpose(2, 3).contiguous().transpose(2, 3)
    sm.softmax_cache_append(k, v, caches[0], caches[1], slots.cuda())
    assert torch.equal(caches, want)


def test_append_into_one_tensor_of_keys_and_values(sm):
    """Caches that interleave in memory: [blocks, 2, size, heads, d]."""
    both = torch.zeros(5, 2, 16, 2, 64, device="cuda")
    k = torch.randn(20, 2, 64, device="cuda")
    slots = torch.randperm(80, device="cuda")[:20]
    sm.softmax_cache_append(k, k + 1, both[:, 0], both[:, 1], slots)
    assert torch.equal(both[slots // 16, 0, slots % 16], k)
    assert torch.equal(both[slots // 16, 1, slots % 16], k + 1)
