"""Embedding rows and the table's gradient against the float64 oracle."""
import pytest
import torch

import paper_1904_12380_amd as sm
from oracle import decoder_f64 as oracle
from tests import decoder_data as data

pytestmark = pytest.mark.gpu


def tokens(kind, count, rows, g):
    if kind == "even":
        return torch.randint(rows, (count,), generator=g)
    if kind == "one":
        return torch.full((count,), rows - 1)
    if kind == "skewed":
        return ((rows ** torch.rand(count, generator=g, dtype=torch.float64)) - 1).long().clamp(0, rows - 1)
    if kind == "none":
        return torch.full((count,), -1)
    ids = torch.randint(rows, (count,), generator=g)  # "wrong": padding and ids past the table
    ids[::3] = -1
    ids[1::5] = rows
    ids[2::7] = 1 << 40
    ids[4::11] = -(1 << 50)
    return ids


def check(ids, rows, d, dtype, scale, apart=0):
    g = torch.Generator().manual_seed(rows + d)
    table = data.matrix(g, rows, d, dtype)
    dout = data.matrix(g, len(ids), d, dtype)
    gt, gd, gi = table.cuda(), dout.cuda(), ids.cuda()
    if apart:
        gt, gd = data.strided(gt, apart, apart), data.strided(gd, apart, apart)
    want = oracle.embedding(ids, table, scale)
    out = sm.softmax_embedding_fwd(gi, gt, scale=scale)
    # The scale is an fp32 number, and so is the product.
    f32 = 2.0 ** -23
    half = data.HALF[dtype] + f32
    data.close("rows", out, want, want.abs() * half + data.TINY[dtype])
    want = oracle.embedding_grad(dout, ids, rows, scale)
    size = oracle.embedding_grad(dout.abs(), ids, rows, abs(scale))
    count = torch.bincount(ids[(ids >= 0) & (ids < rows)], minlength=rows)[:, None]
    dtable = sm.softmax_embedding_bwd(gd, gi, rows, scale=scale)
    # Sums in fp32 (rounded, not cut off); one token has none.
    bound = size * ((count - 1).clamp(min=0) * 2.0 ** -24 + f32)
    data.close("dtable", dtable, want, bound + (want.abs() + bound) * half + data.TINY[dtype])
    untouched = (count[:, 0] == 0).cuda()
    assert not dtable[untouched].any()
    return dtable


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("count,rows,d", [
    (1, 1, 8), (1, 300, 64), (31, 7, 16), (32, 255, 24), (33, 256, 40), (64, 257, 128), (500, 40, 264),
    (1000, 65536, 8), (777, 1000, 520), (100, 65537, 136), (40, 90, 2056)])
def test_sizes(count, rows, d, dtype):
    g = torch.Generator().manual_seed(count)
    check(tokens("even", count, rows, g), rows, d, dtype, 1.0)


@pytest.mark.parametrize("kind", ["one", "skewed", "none", "wrong"])
@pytest.mark.parametrize("count,rows,d", [(1, 20, 8), (95, 20, 64), (1000, 400, 72), (5000, 255, 16)])
def test_tokens(kind, count, rows, d):
    g = torch.Generator().manual_seed(count)
    check(tokens(kind, count, rows, g), rows, d, "bf16", 1.0)


@pytest.mark.parametrize("kind", ["even", "one", "skewed", "wrong"])
@pytest.mark.parametrize("count,rows", [(16383, 300), (16384, 70000), (16385, 300), (20480, 255),
                                        (40000, 256), (50001, 70000), (300000, 1000)])
def test_many_tokens(kind, count, rows):
    """Around the number of tokens that one workgroup sorts, and past it."""
    g = torch.Generator().manual_seed(count)
    check(tokens(kind, count, rows, g), rows, 8, "f32", 1.0)


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("scale", [0.0, -1.0, 16.0, 0.3, 1e-30])
def test_scales(scale, dtype):
    g = torch.Generator().manual_seed(1)
    scale = float(torch.tensor(scale))  # an fp32 number, as the call takes it
    check(tokens("skewed", 300, 50, g), 50, 72, dtype, scale)


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_strides(dtype):
    g = torch.Generator().manual_seed(1)
    check(tokens("wrong", 300, 50, g), 50, 72, dtype, 1.0, apart=24)


def test_broadcast_rows():
    """A table and a gradient whose rows lie at one place."""
    ids = torch.tensor([0, 3, 3, 9, -1])
    row = torch.randn(1, 64)
    out = sm.softmax_embedding_fwd(ids.cuda(), row.cuda().expand(10, 64))
    assert torch.equal(out.cpu()[:4], row.expand(4, 64)) and not out[4].any()
    dtable = sm.softmax_embedding_bwd(row.cuda().expand(5, 64), ids.cuda(), 10).cpu()
    assert torch.equal(dtable[3], 2 * row[0]) and torch.equal(dtable[0], row[0])


def test_values_of_other_rows_stay_out():
    """NaN in rows that no token has, and in the gradient of padding."""
    table = torch.full((10, 16), torch.nan, device="cuda")
    table[4] = 2.0
    ids = torch.tensor([4, -1, 4], device="cuda")
    out = sm.softmax_embedding_fwd(ids, table)
    assert out[0].eq(2).all() and out[1].eq(0).all() and out[2].eq(2).all()
    dout = torch.ones(3, 16, device="cuda")
    dout[1] = torch.nan
    dtable = sm.softmax_embedding_bwd(dout, ids, 10)
    assert dtable[4].eq(2).all() and int(dtable.count_nonzero()) == 16
    dout[0, 3] = torch.inf
    dtable = sm.softmax_embedding_bwd(dout, ids, 10)
    assert dtable[4, 3].isinf() and int(dtable.count_nonzero()) == 16


@pytest.mark.parametrize("count", [9000, 40000])
def test_same_bits_each_time(count):
    g = torch.Generator().manual_seed(1)
    ids = tokens("skewed", count, 300, g).cuda()
    dout = torch.randn(count, 64, device="cuda")
    first = sm.softmax_embedding_bwd(dout, ids, 300)
    for _ in range(4):
        assert torch.equal(sm.softmax_embedding_bwd(dout, ids, 300), first)


def test_empty():
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.randn(5, 8, device="cuda")
    assert sm.softmax_embedding_fwd(none, table).shape == (0, 8)
    assert not sm.softmax_embedding_bwd(table[:0], none, 5).any()
    assert sm.softmax_embedding_bwd(table, torch.zeros(5, dtype=torch.int64, device="cuda"),
                                    0).shape == (0, 8)
    out = sm.softmax_embedding_fwd(torch.zeros(3, dtype=torch.int64, device="cuda"), table[:0])
    assert out.shape == (3, 8) and not out.any()


def test_differentiable():
    ids = torch.tensor([1, 1, 2, -1], device="cuda")
    table = torch.randn(4, 16, device="cuda", requires_grad=True)
    weights = torch.randn(4, 16, device="cuda")
    (sm.softmax_embedding(ids, table, scale=0.5) * weights).sum().backward()
    want = oracle.embedding_grad(weights.cpu(), ids.cpu(), 4, 0.5)
    data.close("grad", table.grad, want, want.abs() * 2.0 ** -22 + 1e-7)
    table.grad = None
    sm.softmax_embedding(ids, table, scale=0.5).sum().backward()  # a gradient of strides 0
    assert table.grad[1].eq(1.0).all() and table.grad[2].eq(0.5).all()
