"""The boundaries of what a decoder has around its attention: sizes at which another
kernel takes over, and calls that are refused."""
import pytest
import torch

import paper_1904_12380_amd as sm
from oracle import decoder_f64 as oracle
from tests import decoder_data as data
from tests import test_gpu_embedding as embedding
from tests import test_gpu_norm as norm

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# Norm: more than 1024 rows of 65 to 256 strips of 16 bytes take two or four
# strips for each lane of a wavefront, four rows a workgroup.

@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype,rows,d", [
    *((t, r, d) for t in ("f16", "bf16")
      for r, d in ((1024, 520), (1025, 520), (1026, 768), (1027, 1016), (1025, 1024), (1027, 1032),
                   (1030, 2048))),
    *(("f32", r, d) for r, d in ((1024, 264), (1027, 264), (1026, 384), (1027, 512),
                                 (1029, 520), (1025, 768), (1025, 1024), (1030, 1032)))])
def test_norm_of_many_rows_of_a_wavefront(dtype, rows, d, center):
    norm.check(*norm.inputs(rows, d, dtype), dtype, center=center)


def test_norm_of_a_broadcast_gradient():
    """y.sum() hands down one number for all rows (strides of zero)."""
    x, weight, bias, _ = norm.inputs(30, 64, "f32")
    ones = torch.ones_like(x)
    exact = oracle.layer_norm(x, weight, bias, dy=ones)
    limit = norm.bounds(x, weight, ones, 1e-5, True, "f32", exact)
    leaves = [t.cuda().requires_grad_() for t in (x, weight, bias)]
    sm.softmax_layer_norm(*leaves).sum().backward()
    for name, leaf, want, bound in zip(("dx", "dweight", "dbias"), leaves, exact[3:], limit[3:]):
        data.close(name, leaf.grad, want, bound)
    assert float(leaves[0].grad.abs().max()) > 0.1


# ---------------------------------------------------------------------------
# Embedding: a workgroup sorts 1024 tokens, up to 32 such tiles are merged, more are
# sorted digit by digit; a digit has nine bits, and a key is an id or the table's rows.

@pytest.mark.parametrize("kind", ["even", "one", "skewed", "wrong"])
@pytest.mark.parametrize("count", [1023, 1024, 1025, 2047, 2049, 31744, 32767, 32768, 32769, 36864,
                                   36865])
def test_embedding_around_the_sorts(kind, count):
    g = torch.Generator().manual_seed(count)
    embedding.check(embedding.tokens(kind, count, 700, g), 700, 8, "f32", 1.0)


@pytest.mark.parametrize("kind", ["even", "skewed", "wrong"])
@pytest.mark.parametrize("rows", [511, 512, 262143, 262144, 300000])
@pytest.mark.parametrize("count", [3000, 40000])
def test_embedding_around_the_digits(count, rows, kind):
    g = torch.Generator().manual_seed(rows)
    ids = embedding.tokens(kind, count, rows, g)
    ids[7], ids[-3] = rows - 1, 0
    embedding.check(ids, rows, 8, "bf16", 1.0)


def test_embedding_of_a_fourth_digit():
    """Rows of 2^27 and more; the last ones hit, with padding between."""
    rows, count = (1 << 27) + 5, 33000
    g = torch.Generator().manual_seed(4)
    ids = torch.randint(rows, (count,), generator=g)
    ids[::2] = rows - 1 - torch.arange(count // 2) % 9
    ids[5::6] = -1
    dout = data.matrix(g, count, 8, "bf16")
    got = sm.softmax_embedding_bwd(dout.cuda(), ids.cuda(), rows)
    hit = ids[ids >= 0].unique()
    place = torch.full((count,), -1)
    place[ids >= 0] = torch.searchsorted(hit, ids[ids >= 0])
    want = oracle.embedding_grad(dout, place, len(hit))
    size = oracle.embedding_grad(dout.abs(), place, len(hit))
    bound = size * count * 2.0 ** -24
    data.close("dtable", got[hit.cuda()], want, bound + (want.abs() + bound) * 2.0 ** -8)
    got[hit.cuda()] = 0
    assert not got.any()


# ---------------------------------------------------------------------------
# Loss: dweight from splits of the tokens, piece by piece.

@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_splits_of_dweight_in_several_pieces(dtype):
    """70001 tokens leave pieces of 3584 rows of the vocabulary (fp32: 1792), 28 tiles
    of dweight: rows of every piece against 64 bits, at the ends of pieces too."""
    rows, vocab, d = 70001, 5000, 16
    g = torch.Generator().manual_seed(6)
    x, weight = data.matrix(g, rows, d, dtype), data.matrix(g, vocab, d, dtype, 0.4)
    labels = torch.randint(vocab, (rows,), generator=g)
    dloss = torch.rand(rows, generator=g) + 0.5
    args = [t.cuda() for t in (x, weight, labels)]
    loss, lse = sm.softmax_linear_nll_fwd(*args)
    _, dweight = sm.softmax_linear_nll_bwd(dloss.cuda(), *args, loss, lse)
    pick = torch.cat([torch.arange(0, vocab, 499), torch.tensor(
        [127, 128, 1791, 1792, 1919, 3583, 3584, 3711, 4863, 4864, 4999])])
    x64, w64 = x.double(), weight.double()
    p = torch.cat([(logits := x64[i:i + 10000] @ w64.t()).sub_(logits.logsumexp(1, keepdim=True))
                   .exp_()[:, pick] for i in range(0, rows, 10000)])
    gs = (p - (labels[:, None] == pick).double()) * dloss.double()[:, None]
    want, size = gs.t() @ x64, gs.abs().t() @ x64.abs()
    # Of a g: logits of 16 terms up to 9 or so, off by 16 cuts of their terms' sizes,
    # twice, as the argument's roundings are: 6e-5 in all.  Of the sum: its terms'
    # roundings to the type, one cut each, and the last rounding; fp16's g below 2^-28
    # of the largest weight, half a denormal step of it.
    bound = size * (data.HALF[dtype] * (dtype != "f32") + 6e-5 + 2 * rows * data.CUT) + \
        want.abs() * data.HALF[dtype] + data.TINY[dtype] + x64.abs().sum(0) * (1.5 * 2.0 ** -39)
    data.close("dweight", dweight[pick.cuda()], want, bound)


# ---------------------------------------------------------------------------
# Refusals

def test_outputs_elsewhere_or_of_another_shape_are_refused():
    x, ids = torch.randn(6, 16, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda")
    f = torch.zeros(6, device="cuda")
    calls = [
        lambda out: sm.softmax_embedding_fwd(ids, x, out=out),
        lambda out: sm.softmax_embedding_bwd(x, ids, 6, dtable=out),
        lambda out: sm.softmax_layer_norm_fwd(x, out=out),
        lambda out: sm.softmax_layer_norm_bwd(x, x, None, f, f, dx=out),
        lambda out: sm.softmax_linear_nll_bwd(f, x, x, ids, f, f, dx=out),
        lambda out: sm.softmax_linear_nll_bwd(f, x, x, ids, f, f, dweight=out),
    ]
    for i, call in enumerate(calls):
        call(torch.empty(6, 16, device="cuda"))
        for bad in (torch.empty(6, 16), torch.empty(7, 16, device="cuda"),
                    torch.empty(6, 16, device="cuda").half(), torch.empty(16, 6, device="cuda").t(),
                    torch.empty(96, device="cuda")):
            with pytest.raises((ValueError, TypeError)):
                call(bad)
                print(i)


def test_inputs_of_two_devices_are_refused():
    x, ids = torch.randn(6, 16, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda")
    f = torch.zeros(6, device="cuda")
    for call in (lambda: sm.softmax_linear_nll_fwd(x, x.cpu(), ids),
                 lambda: sm.softmax_linear_nll_fwd(x, x, ids.cpu()),
                 lambda: sm.softmax_linear_nll_bwd(f.cpu(), x, x, ids, f, f),
                 lambda: sm.softmax_embedding_fwd(ids.cpu(), x),
                 lambda: sm.softmax_embedding_bwd(x, ids.cpu(), 6),
                 lambda: sm.softmax_layer_norm_fwd(x, x[0].cpu()),
                 lambda: sm.softmax_layer_norm_bwd(x.cpu(), x, None, f, f),
                 lambda: sm.softmax_layer_norm_bwd(x, x, None, f.cpu(), f)):
        with pytest.raises((ValueError, TypeError)):
            call()


RECORDED = {
    "nll": lambda x, ids: sm.softmax_linear_nll(x, x, ids),
    "embedding": lambda x, ids: sm.softmax_embedding(ids, x),
    "norm": lambda x, ids: sm.softmax_layer_norm(x),
}


@pytest.mark.parametrize("name", RECORDED)
def test_vmap_and_forward_mode_are_refused(name):
    call = RECORDED[name]
    ids = torch.zeros(6, dtype=torch.int64, device="cuda")
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda x: call(x, ids))(torch.randn(3, 6, 16, device="cuda"))
    with torch.autograd.forward_ad.dual_level():
        x = torch.randn(6, 16, device="cuda")
        dual = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises((RuntimeError, NotImplementedError)):
            call(dual, ids)
