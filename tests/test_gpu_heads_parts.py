"""Weights in two 16-bit parts: the first 64 keys of rows that see at most 128,
whatever tile the rows lie in.

The bound: the output's own rounding u |o|; for keys in two parts a weight's
remainder after two roundings, at most u^2, which 2^-15 covers beside the fp32
errors of the score and the exponential (2^-17 for scores of up to 30); u for
the weights of keys past the first 64."""
import numpy as np
import pytest

import oracle.heads_f64 as ref
from tests.heads_data import Packed, Paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sm():
    import paper_1904_12380_amd
    return paper_1904_12380_amd


def bound(run, v, dtype, late):
    """u |o| + 2^-15 sum P |v| + u sum of P |v| over late keys; run(v) is the
    oracle's o for values v."""
    u = ref.UNIT[dtype]
    size = np.nan_to_num(np.abs(v))
    return u * np.abs(run(v)) + 2.0 ** -15 * run(size) + u * run(size * late) + ref.TINY[dtype] * 200


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("how", [{}, dict(bias=True), dict(cap=20.0)])
@pytest.mark.parametrize("heads,kv_heads,size", [(8, 2, 16), (4, 4, 8), (5, 1, 64)])
def test_single_tokens(sm, dtype, how, heads, kv_heads, size):
    keys = [1, 20, 32, 33, 40, 47, 48, 63, 64, 65, 90, 127, 128]
    case = Paged(torch, 60, dtype, [(1, n) for n in keys], heads, kv_heads, 64, size, scale=0.5,
                 **how)
    got = case.run(sm)["o"].double().cpu().numpy()

    # 1 where a slot holds a key past its request's first 64
    late = np.zeros(case.f[1].shape)
    for row, n in zip(case.table, keys):
        j = np.arange(64, max(n, 64))
        late[row[j // size], j % size] = 1.0

    def run(v):
        return ref.paged(case.fq, case.f[0], v, case.table, case.cu_q, case.keys,
                         dtype=dtype, **case.ref)["o"]
    off = np.abs(got - run(case.f[1]))
    assert (off <= bound(run, case.f[1], dtype, late)).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (2, 2), (8, 4)])
def test_ends_of_documents(sm, dtype, heads, kv_heads):
    """Tiles of a document's last few rows beside whole ones."""
    lens = [35, 40, 50, 64, 33, 1, 100, 128]
    case = Packed(torch, 61, dtype, [(n, n) for n in lens], heads, kv_heads, 64, scale=0.5)
    got = case.run(sm, train=False)["o"].double().cpu().numpy()
    late = np.concatenate([np.arange(n) >= 64 for n in lens]).astype(float)[:, None, None]

    def run(v):
        return ref.packed(case.f["q"], case.f["k"], v, case.cu_q, case.cu_k, dtype=dtype,
                          **case.ref)["o"]
    off = np.abs(got - run(case.f["v"]))
    assert (off <= bound(run, case.f["v"], dtype, late)).all()
