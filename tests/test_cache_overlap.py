"""The append refuses caches of keys and of values that have an element in common
(both would be written there, in no order), and takes ones that interleave."""
import numpy as np
import pytest

import paper_1904_12380_amd as sm
from paper_1904_12380_amd import attention as at

BAD = sm.ERR_INVALID_ARG
FAR = 1 << 40


def append(k, v, shape, k_strides, v_strides=None, dtype=2):
    """The append into caches that start at elements k and v of one allocation."""
    blocks, size, heads, d = shape
    width = 4 if dtype == 0 else 2
    tensor = [at._Heads(i << 44, 10, heads, d, heads * d, d) for i in (2, 3)]
    caches = [at._Cache(FAR + width * base, blocks, size, heads, d, *strides)
              for base, strides in ((k, k_strides), (v, v_strides or k_strides))]
    return sm.load_library().softmax_cache_append(*tensor, *caches, 4 << 44, dtype, None)


@pytest.mark.parametrize("dtype", [0, 2])
def test_layouts_of_both(dtype):
    b, s, h, d = shape = (5, 16, 2, 64)
    row = h * d
    assert append(0, 0, shape, (s * row, row, d), dtype=dtype) == BAD           # one tensor
    assert append(0, s * row, shape, (s * row, row, d), dtype=dtype) == BAD     # a block on
    assert append(row, 0, shape, (s * row, row, d), dtype=dtype) == BAD         # a row back
    assert append(0, 8, shape, (s * row, row, d), dtype=dtype) == BAD           # within a row
    for v, strides in ((s * row, (2 * s * row, row, d)),             # [blocks, 2, size, heads, d]
                       (row, (2 * s * row, 2 * row, d)),             # [blocks, size, 2, heads, d]
                       (d, (2 * s * row, 2 * row, 2 * d)),           # [blocks, size, heads, 2, d]
                       (s * d, (2 * s * row, d, 2 * s * d)),         # [blocks, heads, 2, size, d]
                       (b * s * row, (s * row, row, d))):            # [2, blocks, ...]
        assert append(0, v, shape, strides, dtype=dtype) != BAD
        assert append(v, 0, shape, strides, dtype=dtype) != BAD
        assert append(0, v - 8, shape, strides, dtype=dtype) == BAD
        assert append(v - 8, 0, shape, strides, dtype=dtype) == BAD
    # heads before tokens in one, tokens first in the other, between each other
    assert append(0, s * row, shape, (2 * s * row, row, d), (2 * s * row, d, s * d),
                  dtype=dtype) != BAD


def test_against_sets_of_elements():
    rng = np.random.default_rng(1)
    seen = [0, 0]
    for _ in range(2000):
        blocks, size, heads = (int(rng.integers(1, 5)) for _ in range(3))
        size = 1 << (size - 1)
        d = 8 * int(rng.integers(1, 4))
        counts = {"blocks": blocks, "size": size, "heads": heads}
        strides, extent = {}, d
        for name in rng.permutation(list(counts)):
            strides[name] = extent + 8 * int(rng.choice([0, 0, 1, 2, extent // 8]))
            extent = strides[name] * (counts[name] - 1) + extent
        way = (strides["blocks"], strides["size"], strides["heads"])
        delta = 8 * int(rng.integers(0, extent // 8 + 2))
        index = np.add.outer(np.add.outer(np.add.outer(
            np.arange(blocks) * way[0], np.arange(size) * way[1]), np.arange(heads) * way[2]),
            np.arange(d)).ravel()
        meet = bool(np.isin(index, index + delta).any())
        seen[meet] += 1
        for k, v in ((0, delta), (delta, 0)):
            got = append(k, v, (blocks, size, heads, d), way)
            assert (got == BAD) == meet, (counts, d, way, delta)
    assert min(seen) > 200
