"""Scores of 10^5 to 10^10: one key holds all of a row's weight, and the result is
its value.  What is left of a score's size in the exponent's argument (its
rounding, several powers of two here) must not scale the weights."""
import numpy as np
import pytest

from tests.heads_data import Packed, Paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sm():
    import paper_1904_12380_amd
    return paper_1904_12380_amd


def check(got, want, dtype):
    """The value's copy within two roundings: the one weight is 1 in any type."""
    o = got["o"].double().cpu().numpy()
    assert np.isfinite(o).all()
    u = {"f32": 2.0 ** -22, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}[dtype]
    assert np.abs(o - want["o"]).max() <= u * np.abs(want["o"]).max()
    lse = got["lse"].double().cpu().numpy()
    assert np.abs(lse / want["lse"] - 1).max() <= 2.0 ** -20


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** 5, 2.0 ** 9, 2.0 ** 12])
@pytest.mark.parametrize("rows,how", [(1, {}), (20, {}), (300, {}), (40, dict(bias=True)),
                                      (300, dict(scale=-0.7))])
def test_packed(sm, dtype, size, rows, how):
    case = Packed(torch, 90, dtype, [(rows, 333)], 2, 1, 64, causal=False, **{"scale": 1.0, **how})
    for name in ("q", "k"):
        case.t[name] *= size
        case.f[name] = case.t[name].double().cpu().numpy()
    # rows whose two largest scores lie within fp32's rounding are left out
    scale = case.how["scale"]
    x = np.einsum("qhd,kd->qhk", case.f["q"], case.f["k"][:, 0]) * scale
    top = np.sort(x, 2)
    clear = top[:, :, -1] - top[:, :, -2] > 2.0 ** -18 * np.abs(x).max() + 30.0
    assert clear.mean() > 0.9 or size == 2.0 ** 5
    got, want = case.run(sm, train=False), case.oracle(train=False)
    keep = torch.from_numpy(clear)
    check({n: y[keep.cuda()] for n, y in got.items()}, {n: y[clear] for n, y in want.items()},
          dtype)
    assert torch.isfinite(got["o"]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("requests", [[(1, 60)], [(1, 3000)], [(50, 900)]])
def test_paged(sm, dtype, requests):
    case = Paged(torch, 91, dtype, requests, 4, 1, 64, 16, scale=1.0, causal=False)
    case.q *= 2.0 ** 12
    case.fq = case.q.double().numpy()
    case.t[0] *= 2.0 ** 12
    case.f[0] = case.t[0].double().cpu().numpy()
    got, want = case.run(sm), case.oracle()
    keys = requests[0][1]
    rows = case.table[0, np.arange(keys) // 16]
    k = case.f[0][rows, np.arange(keys) % 16, 0]
    x = np.sort(np.einsum("qhd,kd->qhk", case.fq, k), 2)
    clear = x[:, :, -1] - x[:, :, -2] > 2.0 ** -16 * np.abs(x).max()
    assert clear.mean() > 0.9
    check({n: y.cpu()[torch.from_numpy(clear)] for n, y in got.items()},
          {n: y[clear] for n, y in want.items()}, dtype)
    assert torch.isfinite(got["o"]).all()
