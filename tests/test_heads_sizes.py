"""Sizes past a launch's limit (2^24 workgroups) are refused before any HIP call;
sizes below it get past the checks of arguments."""
import pytest

import paper_1904_12380_amd as sm
from paper_1904_12380_amd import attention as at
from tests.test_heads_host import bwd, fwd, paged, score

BAD = sm.ERR_INVALID_ARG


def packed_docs(docs, dtype, tokens=100):
    """The forward call with that many documents of one tensor."""
    fn = sm.load_library().softmax_packed_attention_fwd
    far = [i << 44 for i in range(1, 7)]

    def of(i, n):
        return at._Heads(far[i], tokens, n, 64, n * 64, 64)
    return fn(of(0, 4), of(1, 2), of(2, 2), far[3], far[4], far[5], far[5], docs, score(), dtype,
              None)


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_documents(dtype):
    # (100 * 2 / T + docs + 1) * 2 workgroups
    per = 200 // (64 if dtype == 0 else 128)
    most = ((1 << 24) - 1) // 2 - per - 1
    assert packed_docs(most, dtype) != BAD
    assert packed_docs(most + 1, dtype) == BAD
    assert packed_docs(1 << 40, dtype) == BAD
    assert packed_docs((1 << 63) - 1, dtype) == BAD


def test_requests_and_rows():
    assert paged(requests=3) != BAD
    for requests in (1 << 23, 1 << 29, 1 << 62):
        assert paged(requests=requests) == BAD
    size = sm.load_library().softmax_paged_attention_workspace
    assert size(100, 4, 2, 64, 1 << 23, 4096) == -1
    # 2^30 rows: 2^24 tiles of fp32, 2^23 of 16 bits
    room = sm.load_library().softmax_packed_attention_bwd_workspace
    assert room(1 << 28, 100, 4, 4, 64, 0) == -1
    assert room(1 << 28, 100, 4, 4, 64, 2) > 8 << 30


def test_small_calls_get_past_the_checks():
    assert fwd() != BAD and bwd() != BAD and paged() != BAD
