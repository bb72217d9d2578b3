"""Multi-head attention against the float64 oracle by norm: instances and calls
that bounds by element leave open (split gradients of wide heads with caps and
biases, large scores, values with a common part, rows of a few keys)."""
import numpy as np
import pytest

from tests.heads_data import Packed, Paged
from tests.heads_norms import FEW, assert_norms

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = ("f32", "f16", "bf16")
TRAIN = ("o", "dq", "dk", "dv")


@pytest.fixture(scope="module")
def sm():
    import paper_1904_12380_amd
    return paper_1904_12380_amd


def values(got):
    return {n: x.double().cpu().numpy() for n, x in got.items()}


def check(case, sm, names=TRAIN, **how):
    assert_norms(torch, values(case.run(sm)), case.oracle(), case.dtype, names, **how)


SCORES = {"plain": {}, "cap": dict(cap=15.0), "bias": dict(bias=True),
          "both": dict(cap=9.0, bias=True)}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [72, 128, 136, 256])
@pytest.mark.parametrize("scores", SCORES)
@pytest.mark.parametrize("docs,heads,kv_heads,how", [
    ([(1100, 1100), (70, 70)], 4, 1, {}),              # key tiles split over heads' rows
    ([(640, 640), (641, 641)], 4, 2, dict(prefix=[500, 0])),
    ([(700, 1300)], 3, 1, dict(causal=False))])
def test_split_gradients_of_wide_heads(sm, dtype, d, scores, docs, heads, kv_heads, how):
    check(Packed(torch, 80, dtype, docs, heads, kv_heads, d, **how, **SCORES[scores]), sm)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("spread", [4.0, 30.0])
@pytest.mark.parametrize("how", [{}, dict(cap=50.0), dict(bias=True)])
def test_large_scores(sm, dtype, d, spread, how):
    check(Packed(torch, 81, dtype, [(150, 150), (333, 333)], 2, 1, d, spread=spread, **how), sm,
          spread=spread)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [range(1, 9), [8] * 70, [1, 2, 3] * 30])
def test_rows_of_a_few_keys(sm, dtype, lens):
    case = Packed(torch, 82, dtype, [(n, n) for n in lens], 4, 2, 64)
    check(case, sm, times=FEW)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [(300, 41), (1200,)])
def test_values_with_a_common_part(sm, dtype, lens):
    """D is then large beside the differences that it is taken from, and o's
    rounding would put the gradients of queries and keys off by a quarter of
    themselves."""
    case = Packed(torch, 83, dtype, [(n, n) for n in lens], 2, 1, 64)
    case.t["v"] += 60.0
    case.f["v"] = case.t["v"].double().cpu().numpy()
    # float32: D is 60 times what is left of it
    check(case, sm, spread=60.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_of_nearly_one_key(sm, dtype, d):
    """A first key that takes nearly all of every row's weight: the terms of dq
    and dk all but cancel."""
    case = Packed(torch, 86, dtype, [(500, 500), (90, 90)], 2, 1, d)
    for first in (0, 500):
        case.t["k"][first] *= 0
        case.t["k"][first, :, 0] = 8.0 * d ** 0.5
    case.t["q"][..., 0] = 1.0
    for name in ("q", "k"):
        case.f[name] = case.t[name].double().cpu().numpy()
    check(case, sm)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count", [64, 300])
def test_many_documents(sm, dtype, count):
    lens = np.random.default_rng(count).integers(0, 40, count)
    lens[count // 3] = 900
    check(Packed(torch, 84, dtype, [(int(n), int(n)) for n in lens], 4, 1, 128, cap=20.0), sm)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("scores", SCORES)
@pytest.mark.parametrize("requests,size", [
    ([(1, 4000), (1, 70), (1, 2500)], 16), ([(1, 900), (60, 2100), (200, 700)], 8)])
def test_paged(sm, dtype, d, scores, requests, size):
    case = Paged(torch, 85, dtype, requests, 4, 1, d, size, **SCORES[scores])
    assert_norms(torch, values(case.run(sm)), case.oracle(), dtype, ("o",))
