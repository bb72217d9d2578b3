"""What the bounds by norm can see: the gradients of 16-bit types as the kernels
round them, emulated in numpy, stay within them, and leaving out the second part of
large weights, the correction of D or fp16's range does not."""
import numpy as np
import pytest

import oracle.heads_f64 as ref
from tests.heads_norms import FEW, TIMES, errors, rounded

torch = pytest.importorskip("torch")


def emulate(q, k, v, do, scale, dtype, two_parts=True, correct_d=True, fit=True):
    """One causal document: {o, dq, dk, dv}, sums in float64."""
    cut = lambda x: rounded(torch, x, dtype)  # noqa: E731
    n = len(q)
    x = scale * (q @ k.T)
    x[np.triu_indices(n, 1)] = -np.inf
    p = np.exp(x - x.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)

    def parts(w):
        """w as the products take it: blocks of 32 x 32."""
        by = 2.0 ** 9 / np.abs(w).max() if fit else 1.0
        hi = cut(w * by)
        if two_parts:
            large = np.zeros_like(w, bool)
            for a in range(0, n, 32):
                for b in range(0, n, 32):
                    large[a:a + 32, b:b + 32] = (p[a:a + 32, b:b + 32] > 0.125).any()
            hi = hi + np.where(large, cut(w * by - hi), 0.0)
        return hi / by
    if two_parts and n <= 64:
        o = cut(p @ v)
    else:
        o = cut(cut(p) @ v)
    dp = do @ v.T
    delta = (do * o).sum(1, keepdims=True)
    if two_parts and n <= 64:
        delta = (p * dp).sum(1, keepdims=True)
    ds = p * (dp - delta)
    dk_delta = delta + ds.sum(1, keepdims=True) if correct_d else delta
    return {"o": o, "dq": cut(scale * parts(ds) @ k),
            "dk": cut(scale * parts(p * (dp - dk_delta)).T @ q), "dv": cut(parts(p).T @ do)}


def case(dtype, lens, offset=0.0, size=1.0, d=64, **how):
    """Relative errors over documents of these lengths, in units of rounding once."""
    rng = np.random.default_rng(5)
    got, want = ({x: [] for x in ("o", "dq", "dk", "dv")} for _ in range(2))
    for n in lens:
        q, k, v, do = (rounded(torch, rng.standard_normal((n, d)) * s + b, dtype)
                       for s, b in ((1, 0), (1, 0), (1, offset), (size, 0)))
        one = emulate(q, k, v, do, d ** -0.5, dtype, **how)
        exact = ref.head(q, k, v, dtype=dtype, scale=d ** -0.5, dout=do)
        for x in got:
            got[x].append(one[x])
            want[x].append(exact[x])
    got, want = ({x: np.concatenate(y) for x, y in z.items()} for z in (got, want))
    return {x: off / once for x, (off, once) in errors(torch, got, want, dtype, got).items()}


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_second_parts(dtype):
    lens = list(range(2, 9)) * 12
    assert max(case(dtype, lens).values()) <= FEW
    without = case(dtype, lens, two_parts=False)
    assert min(without[x] for x in ("o", "dq", "dk", "dv")) > FEW


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_correction_of_d(dtype):
    right = case(dtype, [300], offset=60.0)
    assert max(right[x] for x in ("o", "dk", "dv")) <= TIMES
    assert case(dtype, [300], offset=60.0, correct_d=False)["dk"] > 4 * TIMES


def test_range_of_f16():
    for size in (1.0, 1e-3, 1e-4):
        assert max(case("f16", [400], size=size).values()) <= TIMES
    without = case("f16", [1500], size=1e-4, fit=False)
    assert min(without["dq"], without["dk"]) > TIMES
