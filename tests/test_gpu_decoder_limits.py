"""Calls at the far end of what include/decoder_mi355x.h accepts, on rows that lie at
one place where their values do not matter."""
import pytest
import torch

import paper_1904_12380_amd as sm
from oracle import decoder_f64 as oracle
from tests import decoder_data as data

pytestmark = pytest.mark.gpu


def room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_loss_of_more_rows_than_one_launch_joins():
    """2^28 tokens and a few: sixteen threads for each are more than a launch takes."""
    rows, vocab, d = (1 << 28) + 21, 8, 8
    room(80)
    g = torch.Generator(device="cuda").manual_seed(3)
    few = torch.randn(1, d, device="cuda", generator=g).bfloat16()
    weight = torch.randn(vocab, d, device="cuda", generator=g).bfloat16()
    labels = torch.full((rows,), -100, device="cuda")
    labels[:9] = torch.arange(9, device="cuda") % vocab
    labels[-40:] = torch.arange(40, device="cuda") % vocab
    labels[1 << 27] = 5
    loss, lse = sm.softmax_linear_nll_fwd(few.expand(rows, d), weight, labels)
    at = (labels != -100).nonzero()[:, 0]
    assert len(at) == 50
    x, own = few.expand(len(at), d).cpu(), labels[at].cpu()
    exact = oracle.linear_nll(x, weight.cpu(), own, -100, torch.ones(len(at)))
    bounds = data.nll_bounds(x, weight.cpu(), own, -100, torch.ones(len(at)), "bf16", exact)
    for name, got, want, bound in zip(("loss", "lse"), (loss, lse), exact, bounds):
        data.close(name, got[at], want, bound)
        assert int(got.count_nonzero()) == 50


def test_norm_of_more_wide_rows_than_one_launch_takes():
    """2^24 rows and a few of a workgroup each."""
    rows, d = (1 << 24) + 3, 2056
    room(100)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(1, d, device="cuda", generator=g).bfloat16()
    y, mean, rstd = sm.softmax_layer_norm_fwd(x.expand(rows, d))
    want = oracle.layer_norm(x.cpu())
    # Sums of 2056 terms by at most 33 roundings in a row; y's own rounding on top.
    assert abs(float(mean[0]) - float(want[1])) < 40 * 2.0 ** -24 * float(x.double().abs().mean())
    data.close("y", y[:1], want[0], want[0].abs() * 2.0 ** -8 + 1e-4)
    assert torch.equal(mean, mean[:1].expand(rows)) and torch.equal(rstd, rstd[:1].expand(rows))
    for at in range(0, rows, 1 << 20):
        some = y[at:at + (1 << 20)]
        assert torch.equal(some, y[:1].expand(len(some), d)), at
