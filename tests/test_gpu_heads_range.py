"""float16 gradients of all sizes: weights and score gradients are rounded to
float16 for the products, whose small range must not show in the results.

Errors are compared by norm.  Let e be the relative error of the float64
results rounded to the type once.  Rounding the weights or score gradients adds
terms of random signs, each e of its own, to sums whose terms have random signs
too, so e again; the rounding of o in D adds at most e.  Root sums of squares
give 1.7 e; 2.5 e is asserted."""
import numpy as np
import pytest

from tests.heads_data import Packed, types

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TRAIN = ("o", "dq", "dk", "dv")


@pytest.fixture(scope="module")
def sm():
    import paper_1904_12380_amd
    return paper_1904_12380_amd


def scaled(case, name, by):
    """The case's tensor times a power of two or any number, in the type."""
    t = (case.t[name].double() * by).to(types(torch)[case.dtype])
    case.t[name], case.f[name] = t, t.double().cpu().numpy()


def assert_norms(case, got, names=TRAIN, times=2.5):
    want = case.oracle()
    for name in names:
        ref = want[name]
        once = torch.from_numpy(ref).to(types(torch)[case.dtype]).double().numpy()
        value = got[name].double().cpu().numpy()
        assert np.isfinite(value).all(), name
        size = np.linalg.norm(ref)
        off, least = (np.linalg.norm(x - ref) / size for x in (value, once))
        assert off <= times * least, (name, off, least)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-4, 1e-5, 1e-6])
@pytest.mark.parametrize("docs,heads,d,how", [
    ([(2048, 2048)], 1, 128, {}),                       # split keys, long rows
    ([(300, 300), (41, 41), (700, 700)], 2, 64, {}),
    ([(900, 900)], 2, 64, dict(cap=20.0, bias=True)),
    ([(200, 700), (30, 30)], 2, 256, dict(causal=False))])
def test_gradients_of_small_numbers(sm, dtype, size, docs, heads, d, how):
    case = Packed(torch, 50, dtype, docs, heads, 1, d, **how)
    scaled(case, "dout", size)
    assert_norms(case, case.run(sm))


@pytest.mark.parametrize("how", [{}, dict(cap=20.0), dict(bias=True)])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_large_numbers(sm, how, d):
    """Score gradients past 65504, results below."""
    case = Packed(torch, 51, "f16", [(40, 40), (260, 260)], 2, 1, d, scale=2.0 ** -6, **how)
    scaled(case, "dout", 2.0 ** 13 * 8 / d ** 0.5)
    scaled(case, "v", 4.0)
    assert_norms(case, case.run(sm))


def test_gradients_that_grow_along_a_document(sm):
    """Rows of very different sizes meet in one key's sum, in both orders."""
    for way in (1, -1):
        case = Packed(torch, 52, "f16", [(1300, 1300)], 2, 1, 64)
        steps = np.exp2(np.linspace(-14, 6, 1300))[::way]
        scaled(case, "dout", torch.from_numpy(steps.copy()).cuda()[:, None, None])
        assert_norms(case, case.run(sm))


def test_values_of_keys_that_all_rows_see_little_of(sm):
    """Every row's weight of the last key is about 2^-26, and the sum of 32768
    of them has eight bits more than a denormal number of that size would keep."""
    rows, keys, d = 4096, 512, 64
    case = Packed(torch, 53, "f16", [(rows, keys)], 8, 1, d, causal=False, scale=1.0, spread=0.0)
    case.t["q"][..., 0] = 1.0
    case.t["k"][..., 0] = 0.0
    case.t["k"][-1, :, 0] = -11.78125      # 512 exp(11.78) is 2^26
    case.t["dout"] += 0.5
    for name in ("q", "k", "dout"):
        case.f[name] = case.t[name].double().cpu().numpy()
    got, want = case.run(sm)["dv"][-1].double().cpu().numpy(), case.oracle()["dv"][-1]
    # 2^-11 of the sum, its own denormal step, and the fp32 sum of 32768 terms
    assert np.abs(got - want).max() <= 2.0 ** -10 * np.abs(want).max() + 2.0 ** -25


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [1, 40, 130])
@pytest.mark.parametrize("gap", [9.0, 14.0, 17.5])
def test_many_keys_of_small_weight_beside_a_large_one(sm, dtype, rows, gap):
    """One key holds most of each row's weight, thousands of others e^-gap of it
    each: together they move the result by many times its rounding."""
    keys, d = 60000, 64
    case = Packed(torch, 54, dtype, [(rows, keys)], 1, 1, d, causal=False, scale=1.0)
    case.t["q"][:] = 0.0
    case.t["k"][:] = 0.0
    case.t["q"][..., 0] = 1.0
    case.t["k"][..., 0] = -gap
    case.t["k"][7, :, 0] = 0.0
    case.t["v"] += 1.0
    case.t["v"][7] = 0.0
    for name in ("q", "k", "v"):
        case.f[name] = case.t[name].double().cpu().numpy()
    got = case.run(sm, train=False)["o"].double().cpu().numpy()
    want = case.oracle(train=False)["o"]
    # the weight's and the output's rounding, and the fp32 sum of the keys: 938
    # steps of 64, each off by at most 2^-24 of the sum
    u = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    assert np.abs(got - want).max() <= (2.0 * u + 2.0 ** -14) * np.abs(want).max()
