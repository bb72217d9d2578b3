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


@pytest.mark.parametrize("what", ["fwd", "bwd"])
@pytest.mark.parametrize("rows,vocab,d", [(1, 256, 4096), (30, 969, 4096), (4, 2500, 4096),
                                          (1121, 574, 3000), (256, 3000, 4096)])
def test_fp32_logits_of_few_tiles_are_split(rows, vocab, d, what):
    """A workgroup for each of a few tiles would run all of d alone: the workspace has
    the logits of two splits at least, beside the packed rows and g."""
    size = getattr(sm.load_library(), f"softmax_linear_nll_{what}_workspace")
    padded, logits = -(-rows // 256) * 256, -(-rows // 256) * 256 * -(-vocab // 256) * 256 * 4
    assert size(rows, vocab, d, 0) > padded * d * 4 + 2 * logits
    # One stage of d cannot be split.
    assert size(rows, vocab, 32, 0) < size(rows, vocab, d, 0) - 2 * logits


@pytest.mark.parametrize("rows", [12, 60])
def test_splits_of_dx_count_on_both_fp32_workgroups_of_a_cu(rows):
    """22 narrow tiles of dx: 21 splits nearly fill two workgroups on each of 256 CUs."""
    vocab, d = 75898, 2816
    packed, g = 256 * d * 4, 256 * -(-vocab // 256) * 256 * 4
    assert bytes_of(rows, vocab, d) > packed + g + 20 * 256 * d * 4


@pytest.mark.parametrize("rows,vocab,d", [(4096, 256, 2048), (3000, 500, 1160)])
def test_fp32_dweight_of_less_than_a_tile_for_each_cu_is_split(rows, vocab, d):
    """Beside the packed rows, g and a split of dx: the sums of two splits of dweight."""
    padded, whole = -(-rows // 256) * 256, -(-vocab // 256) * 256
    assert bytes_of(rows, vocab, d) > padded * (2 * d + whole) * 4 + 2 * whole * d * 4
