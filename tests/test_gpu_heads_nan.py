"""A row of NaN or infinite scores has no finite log of its sum: lse is NaN with
its o, not the -infinity of a row that sees no key."""
import pytest

from tests.heads_data import Packed, Paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sm():
    import paper_1904_12380_amd
    return paper_1904_12380_amd


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("how", [{}, dict(cap=10.0), dict(bias=True)])
@pytest.mark.parametrize("lens", [(1,), (20,), (150,), (40, 700)])
def test_packed(sm, dtype, how, lens):
    case = Packed(torch, 70, dtype, [(n, n) for n in lens], 2, 1, 64, **how)
    want = case.run(sm, train=False)
    q = case.t["q"].clone()
    at = len(q) - 1
    q[at, 1, 3] = float("nan")
    got = case.run(sm, train=False, q=q)
    assert torch.isnan(got["o"][at, 1]).all() and torch.isnan(got["lse"][at, 1])
    keep = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
    keep[at, 1] = False
    assert torch.equal(got["lse"][keep], want["lse"][keep])
    assert torch.equal(got["o"][keep], want["o"][keep])
    # rows that see nothing keep their -infinity
    none = Packed(torch, 70, dtype, [(5, 0), (9, 4)], 2, 1, 64, **how)
    bad = none.run(sm, train=False, q=torch.full_like(none.t["q"], float("nan")))
    assert torch.isneginf(bad["lse"][:10]).all() and torch.isnan(bad["lse"][10:]).all()
    assert not bad["o"][:10].any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("requests", [[(1, 60), (1, 3000)], [(1, 30), (50, 2000)]])
def test_paged(sm, dtype, requests):
    """Also in calls whose keys are split and joined."""
    case = Paged(torch, 71, dtype, requests, 4, 2, 64, 16)
    want = case.run(sm)
    case.q[-1, 2, 5] = float("nan")
    got = case.run(sm)
    assert torch.isnan(got["o"][-1, 2]).all() and torch.isnan(got["lse"][-1, 2])
    keep = torch.ones(got["lse"].shape, dtype=torch.bool, device="cuda")
    keep[-1, 2] = False
    assert torch.equal(got["lse"][keep], want["lse"][keep])
