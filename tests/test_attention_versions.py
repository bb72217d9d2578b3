"""Tensors that a call writes (caches, block tables, outputs that are given)
count as written for autograd: a backward pass that needs their former values is
refused, not fed with the new ones."""
import pytest

import paper_1904_12380_amd as sm
from paper_1904_12380_amd import attention as at

torch = pytest.importorskip("torch")


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


class Library:
    def __getattr__(self, name):
        return lambda *args: 0


@pytest.fixture
def calls(monkeypatch):
    at._lib()
    monkeypatch.setattr(at, "_fns", Library())
    monkeypatch.setattr(sm, "_run", lambda fn, device, stream, args: sm.OK)


def test_written_tensors_count(calls):
    i32 = lambda *shape: gpu(*shape, dtype=torch.int32)  # noqa: E731
    q, k, cu = gpu(9, 4, 64), gpu(9, 2, 64), i32(2)
    caches, table = gpu(2, 5, 16, 2, 64), i32(2, 3)
    versions = lambda *ts: [t._version for t in ts]  # noqa: E731
    sm.softmax_cache_append(k, k, caches[0], caches[1], gpu(9, dtype=torch.int64))
    assert caches._version == 2 and k._version == 0       # both views' writes
    sm.softmax_cache_slots(i32(2), i32(2), table, i32(4), i32(1), 7, 16)
    assert table._version == 1
    o, lse = gpu(9, 4, 64), gpu(9, 4)
    sm.softmax_packed_attention_fwd(q, k, k, cu, out=o, lse=lse)
    assert versions(o, lse, q, k, cu) == [1, 1, 0, 0, 0]
    grads = gpu(9, 4, 64), gpu(9, 2, 64), gpu(9, 2, 64)
    sm.softmax_packed_attention_bwd(q, q, k, k, o, lse, cu, dq=grads[0], dk=grads[1], dv=grads[2])
    assert versions(*grads, o, lse) == [1, 1, 1, 1, 1]
    sm.softmax_paged_attention_fwd(q, caches[0], caches[1], table, i32(3), i32(2), out=o)
    assert versions(o, caches, table) == [2, 2, 1]


def test_inference_tensors_are_taken(calls):
    with torch.inference_mode():
        caches = gpu(2, 5, 16, 2, 64)
    k, slots = gpu(9, 2, 64), gpu(9, dtype=torch.int64)
    sm.softmax_cache_append(k, k, caches[0], caches[1], slots)
    with torch.inference_mode():
        sm.softmax_cache_append(k, k, caches[0], caches[1], slots)


@pytest.mark.gpu
def test_a_cache_that_a_backward_pass_needs():
    caches = torch.randn(2, 5, 16, 2, 64, device="cuda")
    x = torch.randn(2, 64, device="cuda", requires_grad=True)
    y = (x * caches[0, 0, 0]).sum()
    k = torch.randn(3, 2, 64, device="cuda")
    slots = torch.tensor([0, 1, 2], device="cuda")
    sm.softmax_cache_append(k, k, caches[0], caches[1], slots)
    assert torch.equal(caches[0, 0, :3], k)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
