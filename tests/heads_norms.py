"""Errors of the multi-head attention by norm, beside the bounds by element of
the oracle, which add up absolute values and cannot see a small bias.

Let e be the relative error, by norm, of the float64 results rounded to the type
once.  Weights or score gradients rounded once add terms of random signs, each e
of its own, to sums whose terms have random signs too: e again.  D = do . o from
the rounded o, where it is not corrected, adds at most e.  Root sums of squares:
1.7 e, and TIMES = 2.5 is asserted.  Rows of at most 8 keys have a weight above
1/8, all of their blocks are taken in two parts and D from the weights, so that
only e is left: FEW = 1.05.

float32: a score is off by about 2^-23 of the largest, its weight by twice that
and by 2^-20 for the exponential, gradients by twice as much: 2^-18 times the
scores' spread."""
import numpy as np

TIMES, FEW, F32 = 2.5, 1.05, 2.0 ** -18


def rounded(torch, x, dtype):
    t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    return torch.from_numpy(np.ascontiguousarray(x)).to(t).double().numpy()


def errors(torch, got, want, dtype, names):
    """{name: (relative error, that of rounding once)}."""
    out = {}
    for name in names:
        ref, value = want[name], np.asarray(got[name], np.float64)
        assert np.isfinite(value).all(), name
        size = np.linalg.norm(ref)
        out[name] = tuple(np.linalg.norm(x - ref) / size
                          for x in (value, rounded(torch, ref, dtype)))
    return out


def assert_norms(torch, got, want, dtype, names, times=TIMES, spread=1.0):
    for name, (off, once) in errors(torch, got, want, dtype, names).items():
        bound = F32 * spread if dtype == "f32" else times * once
        assert off <= bound, (name, off, once, bound)
