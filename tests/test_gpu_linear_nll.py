"""The loss over a vocabulary and its gradients against the float64 oracle."""
import pytest
import torch

import paper_1904_12380_amd as sm
from oracle import decoder_f64 as oracle
from tests import decoder_data as data

pytestmark = pytest.mark.gpu

IGNORE = -100


def inputs(rows, vocab, d, dtype, seed=0, ignored=0.0, lean=3.0, spread=1.0):
    g = torch.Generator().manual_seed(seed + 7919 * rows + 31 * vocab + d)
    weight = data.matrix(g, vocab, d, dtype, 1.5 * spread / d ** 0.5)
    labels = torch.randint(vocab, (rows,), generator=g)
    x = torch.randn(rows, d, generator=g)
    x += lean * torch.rand(rows, 1, generator=g) * weight[labels].float()
    labels[torch.rand(rows, generator=g) < ignored] = IGNORE
    dloss = torch.rand(rows, generator=g) + 0.1
    return x.to(data.TYPES[dtype]), weight, labels, dloss


def check(x, weight, labels, dloss, dtype, ignore=IGNORE, apart=None, **how):
    exact = oracle.linear_nll(x, weight, labels, ignore, dloss)
    bounds = data.nll_bounds(x, weight, labels, ignore, dloss, dtype, exact)
    gx, gw = x.cuda(), weight.cuda()
    if apart:
        gx, gw = data.strided(gx, apart, apart), data.strided(gw, apart)
    loss, lse = sm.softmax_linear_nll_fwd(gx, gw, labels.cuda(), ignore=ignore)
    dx, dw = sm.softmax_linear_nll_bwd(dloss.cuda(), gx, gw, labels.cuda(), loss, lse,
                                       ignore=ignore, **how)
    names = ("loss", "lse", "dx", "dweight")
    for name, got, want, bound in zip(names, (loss, lse, dx, dw), exact, bounds):
        if got is not None:
            data.close(f"{name} {tuple(x.shape)} x {len(weight)} {dtype}", got, want, bound)
    return loss, lse, dx, dw


SIZES = [(1, 1, 8), (1, 5, 16), (2, 255, 24), (33, 256, 64), (64, 257, 72), (65, 513, 128),
         (127, 1000, 136), (129, 129, 200), (256, 640, 256), (257, 300, 264), (300, 2049, 40),
         (31, 1100, 520), (600, 77, 96)]


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("rows,vocab,d", SIZES)
def test_sizes(rows, vocab, d, dtype):
    check(*inputs(rows, vocab, d, dtype), dtype)


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("rows,vocab,d", [(3100, 300, 4096), (4000, 4001, 24), (1700, 9000, 48)])
def test_large_tiles(rows, vocab, d, dtype):
    """Sizes whose products have large tiles, whole and ragged."""
    check(*inputs(rows, vocab, d, dtype, ignored=0.05), dtype)


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_many_rows(dtype):
    """More rows than a packing workgroup takes at a time, a third of them ignored."""
    check(*inputs(70001, 130, 16, dtype, ignored=0.33), dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("live", [1, 255, 256, 257, 258])
def test_around_the_tokens_of_two_parts(live, dtype):
    """The number of tokens with a loss decides, whatever the rows."""
    x, weight, labels, dloss = inputs(400, 300, 72, dtype)
    labels[torch.randperm(400, generator=torch.Generator().manual_seed(live))[live:]] = IGNORE
    check(x, weight, labels, dloss, dtype)


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("rows,vocab,d,share", [(1, 40, 8, 1.1), (70, 300, 64, 1.1), (70, 300, 64, 0.5),
                                                (513, 260, 48, 0.9), (2000, 64, 16, 0.3)])
def test_ignored_rows_cost_and_leave_nothing(rows, vocab, d, share, dtype):
    """Their x may hold anything, and they get zeros."""
    x, weight, labels, dloss = inputs(rows, vocab, d, dtype, ignored=share)
    x[labels == IGNORE] = torch.nan
    x[labels == IGNORE, ::2] = torch.inf
    dloss[labels == IGNORE] = torch.nan
    loss, lse, dx, dw = check(x, weight, labels, dloss.nan_to_num(), dtype)
    for t in (loss, lse, dx):
        assert not t[(labels == IGNORE).cuda()].any()
    dx2, dw2 = sm.softmax_linear_nll_bwd(dloss.cuda(), x.cuda(), weight.cuda(), labels.cuda(),
                                         loss, lse)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    if share > 1:
        assert not dw.any()


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("rows,vocab,d,apart", [(40, 200, 64, 8), (100, 300, 72, 24), (3, 70, 8, 64)])
def test_strides(rows, vocab, d, apart, dtype):
    """Rows inside larger tensors, with NaN around them."""
    check(*inputs(rows, vocab, d, dtype, ignored=0.2), dtype, apart=apart)


def test_rows_at_one_place():
    """Strides of zero: the same hidden state, and the same row of the vocabulary."""
    x, weight, labels, dloss = inputs(20, 30, 64, "bf16")
    x, weight = x[:1].expand(20, 64), weight[:1].expand(30, 64)
    exact = oracle.linear_nll(x, weight, labels, IGNORE, dloss)
    bounds = data.nll_bounds(x, weight, labels, IGNORE, dloss, "bf16", exact)
    gx, gw = x[:1].cuda().expand(20, 64), weight[:1].cuda().expand(30, 64)
    loss, lse = sm.softmax_linear_nll_fwd(gx, gw, labels.cuda())
    got = (loss, lse, *sm.softmax_linear_nll_bwd(dloss.cuda(), gx, gw, labels.cuda(), loss, lse))
    for name, g, want, bound in zip(("loss", "lse", "dx", "dweight"), got, exact, bounds):
        data.close(name, g, want, bound)


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("ignore", [0, -1, 7, 1 << 40])
def test_ignore_may_be_any_label(ignore, dtype):
    x, weight, labels, dloss = inputs(90, 50, 32, dtype)
    check(x, weight, labels, dloss, dtype, ignore=ignore)


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_bad_labels_are_loud(dtype):
    x, weight, labels, dloss = inputs(90, 50, 32, dtype, ignored=0.1)
    labels[3], labels[40], labels[80] = 50, -7, 1 << 33
    loss, lse, dx, dw = (t.cpu() for t in check(x, weight, labels, dloss, dtype))
    bad = [3, 40, 80]
    assert loss[bad].isnan().all() and lse[bad].isfinite().all()
    assert dx[bad].isnan().all() and dw.isnan().all()
    rest = torch.ones(90, dtype=torch.bool)
    rest[bad] = False
    assert loss[rest].isfinite().all() and dx[rest].isfinite().all()


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_nan_and_infinity_reach_their_row(dtype):
    x, weight, labels, dloss = inputs(150, 300, 64, dtype)
    x[5, 3], x[77, 0] = torch.nan, torch.inf
    loss, lse = sm.softmax_linear_nll_fwd(x.cuda(), weight.cuda(), labels.cuda())
    dx, dw = sm.softmax_linear_nll_bwd(dloss.cuda(), x.cuda(), weight.cuda(), labels.cuda(), loss,
                                       lse)
    hit = torch.zeros(150, dtype=torch.bool)
    hit[[5, 77]] = True
    assert torch.equal(loss.isnan().cpu(), hit)
    assert torch.equal(dx.isnan().any(1).cpu(), hit)
    assert dw.isnan().any()
    good = oracle.linear_nll(torch.where(hit[:, None], 0.0, x.double()), weight, labels, IGNORE, dloss)
    assert float((loss.double().cpu() - good[0])[~hit].abs().max()) < 1e-2


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_likelihoods_near_one(dtype):
    """Where the label has nearly all of the probability: its gradient is 1 - p,
    and must not be what lse and the label's logit leave of each other."""
    rows, vocab, d = 64, 300, 64
    g = torch.Generator().manual_seed(3)
    weight = data.matrix(g, vocab, d, dtype, 0.02)
    labels = torch.arange(rows)
    weight[:rows, :] = 0
    weight[labels, labels] = 1.0
    x = torch.zeros(rows, d)
    x[labels, labels] = torch.linspace(9.0, 16.0, rows)
    x = x.to(data.TYPES[dtype])
    loss, *_, dw = check(x, weight, labels, torch.ones(rows), dtype)
    want = oracle.linear_nll(x, weight, labels, IGNORE, torch.ones(rows))
    # The sum of exponentials is 1 and a little, and its half step 2^-24 is lost in
    # every addition that takes in the 1: eight in a lane's partial sum, three of
    # its eight partial sums, two halves of a wavefront, two wavefronts, and the
    # product that brings a wavefront's sum to the tile's maximum: 15 in all.  The
    # other terms are off by 1e-6 of themselves, and they make up the loss.
    data.close("loss", loss, want[0], 1e-6 * want[0] + 15 * 2.0 ** -24)
    diag = torch.arange(rows)
    data.close("dweight of labels", dw.cpu()[diag, diag], want[3][diag, diag],
               (2 * data.HALF[dtype] + 1e-5) * want[3][diag, diag].abs() + 16 * 15 * 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_one_weight_for_all_tokens(dtype):
    """A mean's gradient, 1 / n: its rounding to 16 bits would be the same for every
    token.  Held to the bound without any rounding of the labels' entries of g."""
    rows, vocab, d = 300, 4000, 64
    x, weight, labels, _ = inputs(rows, vocab, d, dtype, lean=0.0, spread=0.01)
    dloss = torch.full((rows,), 1.0 / 1300.0)  # 0.0017 off in bf16
    exact = oracle.linear_nll(x, weight, labels, IGNORE, dloss)
    loss, lse = sm.softmax_linear_nll_fwd(x.cuda(), weight.cuda(), labels.cuda())
    _, dw = sm.softmax_linear_nll_bwd(dloss.cuda(), x.cuda(), weight.cuda(), labels.cuda(), loss,
                                      lse)
    got, want = dw.double().cpu(), exact[3]
    # Along the exact gradient errors of one sign add up, roundings of single values
    # do not.  The labels' entries are 1 - 1 / 4000 of a token's weight, at most that
    # much off where they round to 1; the results' own roundings average out over
    # 19200 values.
    along = float((got * want).sum() / want.square().sum()) - 1.0
    assert abs(along) < 1.1 / vocab + 3 * data.HALF[dtype] / 19200 ** 0.5


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_weights_of_all_sizes(dtype):
    """Tokens' weights over many powers of ten."""
    x, weight, labels, dloss = inputs(200, 150, 64, dtype)
    dloss = 10.0 ** torch.linspace(-6, 3, 200)
    dloss[::7] *= -1
    dloss[::11] = 0
    check(x, weight, labels, dloss, dtype)


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_large_logits(dtype):
    x, weight, labels, dloss = inputs(70, 260, 64, dtype, spread=60.0, lean=0.0)
    check(x, weight, labels, dloss, dtype)


def test_zero_weights():
    x, weight, labels, _ = inputs(70, 260, 64, "f16")
    _, _, dx, dw = check(x, weight, labels, torch.zeros(70), "f16")
    assert not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_pieces_of_the_vocabulary(dtype, monkeypatch):
    """A vocabulary of several pieces: tokens times vocabulary past what is kept at
    a time.  Compared with the same call on each half of the rows' gradients."""
    rows, d = (4100, 16)
    vocab = 70000 if dtype == "f32" else 140000
    g = torch.Generator(device="cuda").manual_seed(5)
    kind = data.TYPES[dtype]
    x = torch.randn(rows, d, device="cuda", generator=g).to(kind)
    weight = (torch.randn(vocab, d, device="cuda", generator=g) * 0.4).to(kind)
    labels = torch.randint(vocab, (rows,), device="cuda", generator=g)
    dloss = torch.rand(rows, device="cuda", generator=g) + 0.5
    loss, lse = sm.softmax_linear_nll_fwd(x, weight, labels)
    dx, dw = sm.softmax_linear_nll_bwd(dloss, x, weight, labels, loss, lse)
    pick = torch.arange(0, rows, 41, device="cuda")
    xs, ls, ds = (t[pick].cpu() for t in (x, labels, dloss))
    exact = oracle.linear_nll(xs, weight.cpu(), ls, IGNORE, ds)
    # The scale of g goes by the largest weight of all rows.
    bounds = data.nll_bounds(xs, weight.cpu(), ls, IGNORE, ds.clamp(min=1.6), dtype, exact)
    for name, got, want, bound in zip(("loss", "lse", "dx"), (loss[pick], lse[pick], dx[pick]),
                                      exact, bounds):
        data.close(name, got, want, bound)
    # dweight of some rows of every piece.
    logits = x.float() @ weight.float().t()
    p = (logits - lse[:, None]).exp_() * dloss[:, None]
    p[torch.arange(rows, device="cuda"), labels] -= dloss
    rows_v = torch.arange(0, vocab, 997, device="cuda")
    gs = p[:, rows_v].double().cpu()
    want = gs.t() @ x.double().cpu()
    size = gs.abs().t() @ x.double().abs().cpu()
    # p by torch in fp32: off by d cuts and the argument's roundings, 1e-5 in all.
    bound = size * (data.HALF[dtype] + rows * data.CUT + 2e-5) + want.abs() * data.HALF[dtype] + \
        data.TINY[dtype] + x.double().abs().sum(0).cpu() * (1.6 * 2.0 ** -39)
    data.close("dweight", dw[rows_v], want, bound)


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_same_bits_each_time(dtype):
    x, weight, labels, dloss = (t.cuda() for t in inputs(700, 1000, 136, dtype, ignored=0.3))
    first = None
    for _ in range(4):
        loss, lse = sm.softmax_linear_nll_fwd(x, weight, labels)
        got = [loss, lse, *sm.softmax_linear_nll_bwd(dloss, x, weight, labels, loss, lse)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("dx,dw", [(True, False), (False, True), (False, False)])
def test_one_gradient_alone(dx, dw):
    x, weight, labels, dloss = inputs(100, 300, 64, "bf16")
    both = check(x, weight, labels, dloss, "bf16")
    some = check(x, weight, labels, dloss, "bf16", need_dx=dx, need_dweight=dw)
    for need, a, b in ((dx, both[2], some[2]), (dw, both[3], some[3])):
        assert torch.equal(a, b) if need else b is None


def test_no_rows():
    weight = torch.randn(50, 64, device="cuda")
    none = torch.empty(0, 64, device="cuda")
    labels = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = sm.softmax_linear_nll_fwd(none, weight, labels)
    assert loss.shape == lse.shape == (0,)
    dx, dw = sm.softmax_linear_nll_bwd(loss, none, weight, labels, loss, lse)
    assert dx.shape == (0, 64) and dw.shape == (50, 64) and not dw.any()


def test_gradients_are_differences():
    """Against differences of the loss itself, in fp32."""
    x, weight, labels, dloss = inputs(12, 20, 16, "f32", ignored=0.2)
    gx, gw = x.cuda().requires_grad_(), weight.cuda().requires_grad_()
    (sm.softmax_linear_nll(gx, gw, labels.cuda()) * dloss.cuda()).sum().backward()
    total = lambda a, b: float((oracle.linear_nll(a, b, labels)[0] * dloss).sum())  # noqa: E731
    h = 1e-4
    for t, grad in ((x, gx.grad), (weight, gw.grad)):
        for i in range(0, t.numel(), 17):
            up, down = t.double(), t.double()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            pair = [(up, weight), (down, weight)] if t is x else [(x, up), (x, down)]
            want = (total(*pair[0]) - total(*pair[1])) / (2 * h)
            assert abs(float(grad.view(-1)[i]) - want) < 1e-6 + 1e-5 * abs(want)


def test_broadcast_gradient():
    """loss.sum() hands down one number for all tokens (a stride of zero)."""
    x, weight, labels, _ = inputs(100, 300, 64, "bf16", ignored=0.1)
    gx, gw = x.cuda().requires_grad_(), weight.cuda().requires_grad_()
    loss = sm.softmax_linear_nll(gx, gw, labels.cuda())
    loss.sum().backward()
    dx, dw = sm.softmax_linear_nll_bwd(torch.ones(100, device="cuda"), x.cuda(), weight.cuda(),
                                       labels.cuda(), *sm.softmax_linear_nll_fwd(
                                           x.cuda(), weight.cuda(), labels.cuda()))
    assert torch.equal(gx.grad, dx) and torch.equal(gw.grad, dw)


def test_only_what_is_needed():
    x, weight, labels, _ = (t.cuda() for t in inputs(50, 70, 32, "f32"))
    for need in ((True, False), (False, True)):
        a, b = x.clone().requires_grad_(need[0]), weight.clone().requires_grad_(need[1])
        sm.softmax_linear_nll(a, b, labels).mean().backward()
        assert (a.grad is not None, b.grad is not None) == need


def test_second_derivative_is_refused():
    x, weight, labels, _ = (t.cuda() for t in inputs(5, 7, 8, "f32"))
    x.requires_grad_()
    loss = sm.softmax_linear_nll(x, weight, labels).sum()
    grad, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
