"""The paged call's workspace is sized for the device of its tensors (the number
of splits goes by its compute units), whatever device is current."""
import contextlib

import pytest

import paper_1904_12380_amd as sm
from paper_1904_12380_amd import attention as at

torch = pytest.importorskip("torch")


class OnThird(torch.Tensor):
    is_cuda = True
    device = property(lambda self: torch.device("cuda", 3))


@pytest.mark.parametrize("at_first", [0, 3])
def test_workspace_of_the_tensors_device(at_first, monkeypatch):
    at._lib()
    current, asked, given = [at_first], [], []

    @contextlib.contextmanager
    def device(index):
        current.append(index)
        yield
        current.pop()

    class Library:
        def softmax_paged_attention_workspace(self, *args):
            asked.append(current[-1])
            return 4096 if current[-1] == 3 else 16

        def softmax_paged_attention_fwd(self, *args):
            given.append((current[-1], args[-2]))
            return sm.OK

    monkeypatch.setattr(at, "_fns", Library())
    monkeypatch.setattr(sm, "_get_device", lambda: current[-1])
    monkeypatch.setattr(sm, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(sm, "_empty", lambda shape, dtype, device, stream, returned=True:
                        torch.empty(shape, dtype=dtype).as_subclass(OnThird))
    make = lambda *shape, dtype=torch.float32: \
        torch.zeros(*shape, dtype=dtype).as_subclass(OnThird)  # noqa: E731
    i32 = lambda *shape: make(*shape, dtype=torch.int32)  # noqa: E731
    sm.softmax_paged_attention_fwd(make(2, 4, 64), make(5, 16, 2, 64), make(5, 16, 2, 64),
                                   i32(2, 3), i32(3), i32(2))
    assert asked == [3] and given == [(3, 4096)] and current == [at_first]
