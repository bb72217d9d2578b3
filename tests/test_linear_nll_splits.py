"""How the loss over a vocabulary shares its products out, seen by the workspaces that
it asks for, without a GPU."""
import pytest

import paper_1904_12380_amd as sm


def bytes_of(rows, vocab, d, dtype=0):
    return sm.load_library().softmax_linear_nll_bwd_workspace(rows, vocab, d, dtype)


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("rows,d", [(4768, 1144), (3000, 1024), (1496, 1280)])
def test_one_row_more_than_a_tile_keeps_the_splits_of_dweight(rows, d, dtype):
    """A vocabulary of 257 rows has a few tiles of dweight more than one of 256, not
    those of its piece of 512, and shares their sums over the tokens out as well: the
    splits' sums are most of the workspace."""
    assert bytes_of(rows, 257, d, dtype) > bytes_of(rows, 256, d, dtype)
