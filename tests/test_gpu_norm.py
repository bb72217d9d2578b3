"""Norms of rows and their gradients against the float64 oracle."""
import pytest
import torch

import paper_1904_12380_amd as sm
from oracle import decoder_f64 as oracle
from tests import decoder_data as data

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# Roundings in a row's sum, one after the other: the strips of a lane, a tree of its
# eight columns, six levels of a wavefront, sixteen wavefronts.
CHAIN = 8 + 3 + 6 + 16


def bounds(x, weight, dy, eps, center, dtype, exact):
    """Bounds of (y, mean, rstd, dx, dweight, dbias)."""
    y, mean, rstd, dx, dw, db = exact
    x, dy = x.double(), dy.double()
    rows, d = x.shape
    half, tiny = data.HALF[dtype], data.TINY[dtype]
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double()
    b_mean = (CHAIN + 2) * U * x.abs().mean(1) if center else torch.zeros(rows, dtype=torch.float64)
    off = x - mean[:, None]
    b_off = b_mean[:, None] + U * off.abs()
    # The sum of squares: each is off by 2 |off| b_off and a rounding.
    var = off.square().mean(1) + eps
    b_var = (2 * off.abs() * b_off + b_off.square()).mean(1) + (CHAIN + 4) * U * var
    b_rstd = rstd * (b_var / var * 0.5 * (1 + b_var / var) + 4 * U)
    h = off * rstd[:, None]
    b_h = b_off * rstd[:, None] + off.abs() * b_rstd[:, None] + 2 * U * h.abs()
    b_y = b_h * w.abs() + 4 * U * (h * w).abs() + 2 * U * y.abs()
    g = dy * w
    b_c0 = (CHAIN + 2) * U * g.abs().mean(1, keepdim=True) if center else 0.0
    c1 = (g * h).mean(1, keepdim=True)
    b_c1 = (g.abs() * b_h).mean(1, keepdim=True) + (CHAIN + 4) * U * (g * h).abs().mean(1, keepdim=True)
    c0 = g.mean(1, keepdim=True).abs() if center else 0.0
    inner = g.abs() + c0 + (h * c1).abs()
    b_dx = rstd[:, None] * (b_c0 + b_h * c1.abs() + h.abs() * b_c1 + b_h * b_c1 + 6 * U * inner) + \
        b_rstd[:, None] * inner
    b_dw = (dy.abs() * b_h).sum(0) + (rows + 4) * U * (dy * h).abs().sum(0)
    b_db = (rows + 4) * U * dy.abs().sum(0)
    rounded = lambda b, want: b + (want.abs() + b) * half + tiny  # noqa: E731
    return (rounded(b_y, y), b_mean, b_rstd, rounded(b_dx, dx), rounded(b_dw, dw),
            rounded(b_db, db))


def inputs(rows, d, dtype, offset=0.3, size=1.0):
    g = torch.Generator().manual_seed(31 * rows + d)
    x = (data.matrix(g, rows, d, "f32") * size + offset).to(data.TYPES[dtype])
    return (x, (data.matrix(g, 1, d, "f32")[0] * 0.2 + 1).to(x.dtype),
            data.matrix(g, 1, d, dtype)[0], data.matrix(g, rows, d, dtype))


def check(x, weight, bias, dy, dtype, eps=1e-5, center=True, apart=0):
    exact = oracle.layer_norm(x, weight, bias, eps, center, dy)
    limit = bounds(x, weight, dy, eps, center, dtype, exact)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    gx, gy = x.cuda(), dy.cuda()
    if apart:
        gx, gy = data.strided(gx, apart, apart), data.strided(gy, apart)
    y, mean, rstd = sm.softmax_layer_norm_fwd(gx, dev(weight), dev(bias), eps=eps, center=center)
    dx, dw, db = sm.softmax_layer_norm_bwd(gy, gx, dev(weight), mean, rstd, bias=bias is not None)
    assert (mean is None) == (not center) and (dw is None) == (weight is None)
    assert (db is None) == (bias is None)
    for name, got, want, bound in zip(("y", "mean", "rstd", "dx", "dweight", "dbias"),
                                      (y, mean, rstd, dx, dw, db), exact, limit):
        if got is not None:
            data.close(f"{name} {tuple(x.shape)} {dtype}", got, want, bound)


WIDTHS = [8, 16, 40, 64, 72, 128, 200, 256, 264, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 8192,
          8200, 16384]


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, dtype):
    for rows in (1, 5):
        check(*inputs(rows, d, dtype), dtype)


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("rows,d", [(3, 8), (33, 24), (129, 200), (2000, 72), (1025, 1032), (1030, 2056),
                                    (1025, 4096), (4099, 16), (9000, 128)])
@pytest.mark.parametrize("center", [True, False])
def test_rows(rows, d, center, dtype):
    check(*inputs(rows, d, dtype), dtype, center=center)


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("has", [(True, True), (True, False), (False, True), (False, False)])
def test_without_weight_or_bias(has, center, dtype):
    x, weight, bias, dy = inputs(50, 264, dtype)
    check(x, weight if has[0] else None, bias if has[1] else None, dy, dtype, center=center)


@pytest.mark.parametrize("dtype", list(data.TYPES))
@pytest.mark.parametrize("d", [72, 4096])
def test_strides(d, dtype):
    check(*inputs(40, d, dtype), dtype, apart=24)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("offset,size", [(0.0, 1e-3), (100.0, 1.0), (1000.0, 0.5), (-3.0, 30.0)])
def test_far_means(offset, size, center):
    """Rows whose mean is large next to what they differ by."""
    check(*inputs(20, 1032, "f32", offset, size), "f32", center=center)


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_constant_rows(dtype):
    """Rows of one value: variance 0 and eps alone."""
    x, weight, bias, dy = inputs(6, 64, dtype)
    x = torch.tensor([0.0, 1.0, -2.5, 0.125, 40.0, 3.0], dtype=x.dtype)[:, None].expand(6, 64).contiguous()
    y, mean, rstd = sm.softmax_layer_norm_fwd(x.cuda(), weight.cuda(), bias.cuda())
    assert torch.equal(y.cpu(), bias.expand(6, 64))
    assert torch.equal(mean.cpu(), x[:, 0].float())
    data.close("rstd", rstd, torch.full((6,), 1e-5, dtype=torch.float64) ** -0.5, 1e-4)


def test_nan_stays_in_its_row():
    x, weight, bias, dy = inputs(40, 200, "bf16")
    x[7, 3] = torch.nan
    x[9, 0] = torch.inf
    y, mean, rstd = sm.softmax_layer_norm_fwd(x.cuda(), weight.cuda(), bias.cuda())
    dx, dw, _ = sm.softmax_layer_norm_bwd(dy.cuda(), x.cuda(), weight.cuda(), mean, rstd)
    hit = torch.zeros(40, dtype=torch.bool)
    hit[[7, 9]] = True
    for t in (y, dx):
        assert torch.equal(t.isnan().any(1).cpu(), hit)
    assert dw.isnan().all()


@pytest.mark.parametrize("rows,d", [(5000, 200), (300, 4096)])
def test_same_bits_each_time(rows, d):
    x, weight, bias, dy = (t.cuda() for t in inputs(rows, d, "bf16"))
    y, mean, rstd = sm.softmax_layer_norm_fwd(x, weight, bias)
    first = sm.softmax_layer_norm_bwd(dy, x, weight, mean, rstd, bias=True)
    for _ in range(4):
        got = sm.softmax_layer_norm_bwd(dy, x, weight, mean, rstd, bias=True)
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_no_rows():
    none, weight = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    y, mean, rstd = sm.softmax_layer_norm_fwd(none, weight)
    assert y.shape == (0, 64) and mean.shape == rstd.shape == (0,)
    dx, dw, db = sm.softmax_layer_norm_bwd(none, none, weight, mean, rstd, bias=True)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()


@pytest.mark.parametrize("need_dx,need_dw,bias", [(True, False, False), (False, True, False),
                                                  (False, False, True), (False, False, False)])
def test_one_gradient_alone(need_dx, need_dw, bias):
    x, weight, b, dy = (t.cuda() for t in inputs(100, 264, "bf16"))
    y, mean, rstd = sm.softmax_layer_norm_fwd(x, weight, b)
    every = sm.softmax_layer_norm_bwd(dy, x, weight, mean, rstd, bias=True)
    some = sm.softmax_layer_norm_bwd(dy, x, weight, mean, rstd, bias=bias, need_dx=need_dx,
                                     need_dweight=need_dw)
    for need, a, c in zip((need_dx, need_dw, bias), every, some):
        assert torch.equal(a, c) if need else c is None


@pytest.mark.parametrize("center", [True, False])
def test_gradients_are_differences(center):
    x, weight, bias, dy = inputs(3, 16, "f32")
    leaves = [t.cuda().requires_grad_() for t in (x, weight, bias)]
    (sm.softmax_layer_norm(*leaves, center=center) * dy.cuda()).sum().backward()
    h = 1e-4
    for k, t in enumerate((x, weight, bias)):
        for i in range(0, t.numel(), 5):
            total = []
            for sign in (1, -1):
                moved = [v.double() for v in (x, weight, bias)]
                moved[k] = moved[k].clone()
                moved[k].view(-1)[i] += sign * h
                total.append(float((oracle.layer_norm(*moved, center=center)[0] * dy).sum()))
            want = (total[0] - total[1]) / (2 * h)
            assert abs(float(leaves[k].grad.view(-1)[i]) - want) < 1e-5 + 1e-5 * abs(want)


def test_broadcast_gradient():
    x, weight, bias, _ = (t.cuda().requires_grad_() for t in inputs(30, 64, "f32"))
    sm.softmax_layer_norm(x, weight, bias).sum().backward()
    assert bias.grad.eq(30).all() and x.grad.abs().max() < 1e-4 * weight.abs().max() + 1
