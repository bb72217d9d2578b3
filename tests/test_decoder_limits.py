"""The limits that include/decoder_mi355x.h states are those of the entry points: the
largest sizes get past the checks (no device is there to run them), the next do not."""
import paper_1904_12380_amd as sm
from tests.test_decoder_host import (BAD, HEADER, embed_bwd, embed_fwd, nll_bwd, nll_fwd,
                                     norm_bwd, norm_fwd)

MOST = 1 << 29


def test_header_states_the_limits():
    for words in ("Rows and tokens are at most 2^29", "vocab is at most 2^29",
                  "fewer than 2^23 - 64 tiles of 256 x 256", "2^24 - 64 of 128 x 128",
                  "at most 2^38 - 2^14 bytes"):
        assert words in HEADER, words


def test_rows_and_tokens():
    wide = dict(rows=MOST, d=8)
    assert norm_fwd(**wide, sx=8) != BAD and norm_bwd(**wide, sx=8, sy=8) != BAD
    assert norm_fwd(rows=MOST, d=4096, sx=0) != BAD   # a workgroup for each row
    assert embed_fwd(tokens=MOST, rows=MOST, d=8, stride=8) != BAD
    assert embed_bwd(tokens=MOST, rows=MOST, d=8, stride=8) != BAD
    for call in (norm_fwd, norm_bwd, embed_fwd, embed_bwd, nll_fwd, nll_bwd):
        assert call(rows=MOST + 1, d=8) == BAD
    for call in (embed_fwd, embed_bwd):
        assert call(tokens=MOST + 1, d=8) == BAD


def test_bytes_of_looked_up_rows():
    """16-byte strips of 2^14 bytes a workgroup, fewer than 2^24 workgroups."""
    d, size = 1 << 13, 2
    most = ((1 << 38) - (1 << 14)) // (d * size)
    assert embed_fwd(tokens=most, d=d, stride=d) != BAD
    assert embed_fwd(tokens=most + 1, d=d, stride=d) == BAD


def test_tiles():
    for dtype, tile, most in ((2, 256, (1 << 23) - 64), (0, 128, (1 << 24) - 64)):
        side = 1 << 9
        for call in (nll_fwd, nll_bwd):
            fits = dict(d=8, sx=8, sw=8, dtype=dtype, vocab=side * tile)
            assert call(rows=(most // side - 1) * tile, **fits) != BAD
            assert call(rows=(most // side + 1) * tile, **fits) == BAD
    assert sm.load_library().softmax_linear_nll_fwd_workspace(MOST, 8, 8, 2) > 0
