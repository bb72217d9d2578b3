"""What a decoder has around its attention, without a GPU: the entry points refuse
bad arguments before any HIP call, the binding refuses bad tensors, memory belongs
to the call's stream, and the oracle agrees with differences and closed forms."""
import contextlib
import math
import os
import re

import pytest

import paper_1904_12380_amd as sm
from oracle import decoder_f64 as oracle
from paper_1904_12380_amd import attention as at
from tests.test_stream_memory import Library, OnGpu, gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "decoder_mi355x.h")).read()
P = [i << 44 for i in range(1, 20)]      # far apart, never dereferenced
BAD = sm.ERR_INVALID_ARG
ROOM = 1 << 42


def nll_fwd(x=P[0], sx=64, w=P[1], sw=64, labels=P[2], rows=100, vocab=300, d=64, ignore=-100,
            dtype=2, loss=P[3], lse=P[4], work=P[5], room=ROOM):
    return sm.load_library().softmax_linear_nll_fwd(x, sx, w, sw, labels, rows, vocab, d, ignore,
                                                    dtype, loss, lse, work, room, None)


def nll_bwd(x=P[0], sx=64, w=P[1], sw=64, labels=P[2], rows=100, vocab=300, d=64, dtype=2,
            dloss=P[6], dx=P[7], dw=P[8], work=P[5], room=ROOM):
    return sm.load_library().softmax_linear_nll_bwd(dloss, x, sx, w, sw, labels, rows, vocab, d,
                                                    -100, dtype, P[3], P[4], dx, dw, work, room,
                                                    None)


def embed_fwd(ids=P[0], tokens=100, table=P[1], stride=64, rows=300, d=64, scale=1.0, dtype=2,
              out=P[2]):
    return sm.load_library().softmax_embedding_fwd(ids, tokens, table, stride, rows, d, scale,
                                                   dtype, out, None)


def embed_bwd(dout=P[0], stride=64, ids=P[1], tokens=100, rows=300, d=64, scale=1.0, dtype=2,
              dtable=P[2], work=P[3], room=ROOM):
    return sm.load_library().softmax_embedding_bwd(dout, stride, ids, tokens, rows, d, scale,
                                                   dtype, dtable, work, room, None)


def norm_fwd(x=P[0], sx=64, w=P[1], b=P[2], rows=100, d=64, eps=1e-5, center=1, dtype=2, y=P[3],
             mean=P[4], rstd=P[5]):
    return sm.load_library().softmax_layer_norm_fwd(x, sx, w, b, rows, d, eps, center, dtype, y,
                                                    mean, rstd, None)


def norm_bwd(dy=P[0], sy=64, x=P[1], sx=64, w=P[2], mean=P[3], rstd=P[4], rows=100, d=64, dtype=2,
             dx=P[5], dw=P[6], db=P[7], work=P[8], room=ROOM):
    return sm.load_library().softmax_layer_norm_bwd(dy, sy, x, sx, w, mean, rstd, rows, d, dtype,
                                                    dx, dw, db, work, room, None)


CALLS = [nll_fwd, nll_bwd, embed_fwd, embed_bwd, norm_fwd, norm_bwd]


def test_header_and_binding_agree():
    assert re.search(r"#define SOFTMAX_MAX_WIDTH (\d+)", HEADER).group(1) == str(sm.MAX_WIDTH)
    assert re.search(r"#define SOFTMAX_MAX_ROW_STRIDE (\d+)", HEADER).group(1) == \
        str(sm.decoder.MAX_ROW_STRIDE)
    for what in ("linear_nll", "embedding", "layer_norm"):
        for name in (f"softmax_{what}_fwd", f"softmax_{what}_bwd"):
            assert re.search(rf"SOFTMAX_API int {name}\(", HEADER) and name in sm.__all__
        assert f"softmax_{what}" in sm.__all__


def test_good_calls_get_past_the_checks():
    for call in CALLS:
        for dtype in (0, 1, 2):
            assert call(dtype=dtype) != BAD, call


@pytest.mark.parametrize("call", CALLS)
def test_sizes_and_types_are_refused(call):
    for dtype in (-1, 3, 9):
        assert call(dtype=dtype) == BAD
    for d in (0, -8, 4, 7, 12, 16392, 1 << 40):
        assert call(d=d) == BAD
    for rows in (-1, (1 << 29) + 1, 1 << 62, -(1 << 63)):
        assert call(rows=rows) == BAD


@pytest.mark.parametrize("call,names", [
    (nll_fwd, ("x", "w", "work")), (nll_bwd, ("x", "w", "dx", "dw", "work")),
    (embed_fwd, ("table", "out")), (embed_bwd, ("dout", "dtable", "work")),
    (norm_fwd, ("x", "w", "b", "y")), (norm_bwd, ("dy", "x", "w", "dx", "work"))])
def test_misaligned_data_is_refused(call, names):
    for name in names:
        assert call(**{name: P[12] + 8}) == BAD, name


@pytest.mark.parametrize("call,names", [
    (nll_fwd, ("sx", "sw")), (nll_bwd, ("sx", "sw")), (embed_fwd, ("stride",)),
    (embed_bwd, ("stride",)), (norm_fwd, ("sx",)), (norm_bwd, ("sx", "sy"))])
def test_strides_are_refused(call, names):
    for name in names:
        for stride in (-64, 68, 1 << 62):
            assert call(**{name: stride}) == BAD, (name, stride)
        assert call(**{name: 0}) != BAD      # rows at one place
    for name in ("sw", "stride"):
        if name in names and call is not embed_bwd:
            assert call(**{name: (1 << 20) + 8}) == BAD
            assert call(**{name: 1 << 20}) != BAD


@pytest.mark.parametrize("call,outputs,inputs", [
    (nll_fwd, ("loss", "lse", "work"), ("x", "w", "labels")),
    (nll_bwd, ("dx", "dw", "work"), ("x", "w", "labels", "dloss")),
    (embed_fwd, ("out",), ("ids", "table")), (embed_bwd, ("dtable", "work"), ("dout", "ids")),
    (norm_fwd, ("y", "mean", "rstd"), ("x", "w", "b")),
    (norm_bwd, ("dx", "dw", "db", "work"), ("dy", "x", "w", "mean", "rstd"))])
def test_overlaps_are_refused(call, outputs, inputs):
    for out in outputs:
        for other in (*inputs, *outputs):
            if other != out:
                assert call(**{out: P[12], other: P[12] + 16}) == BAD, (out, other)


def test_missing_pointers_are_refused():
    for call, names in ((nll_fwd, ("x", "w", "labels", "loss", "lse")),
                        (nll_bwd, ("x", "w", "labels", "dloss")), (embed_fwd, ("ids", "table", "out")),
                        (embed_bwd, ("ids", "dout", "dtable")), (norm_fwd, ("x", "y", "mean", "rstd")),
                        (norm_bwd, ("x", "dy", "rstd"))):
        for name in names:
            assert call(**{name: None}) == BAD, (call, name)


def test_workspaces():
    lib = sm.load_library()
    assert nll_fwd(room=lib.softmax_linear_nll_fwd_workspace(100, 300, 64, 2)) != BAD
    assert nll_fwd(room=lib.softmax_linear_nll_fwd_workspace(100, 300, 64, 2) - 1) == BAD
    assert embed_bwd(room=lib.softmax_embedding_bwd_workspace(100, 300, 64, 2)) != BAD
    assert embed_bwd(room=lib.softmax_embedding_bwd_workspace(100, 300, 64, 2) - 1) == BAD
    assert norm_bwd(room=lib.softmax_layer_norm_bwd_workspace(100, 64, 2)) != BAD
    assert norm_bwd(room=lib.softmax_layer_norm_bwd_workspace(100, 64, 2) - 1) == BAD
    assert norm_bwd(room=0, work=None, dw=None, db=None) != BAD
    for size in (lib.softmax_linear_nll_fwd_workspace, lib.softmax_linear_nll_bwd_workspace,
                 lib.softmax_embedding_bwd_workspace):
        for bad in ((-1, 300, 64, 2), (100, -1, 64, 2), (100, 300, 12, 2), (100, 300, 64, 3),
                    (1 << 30, 300, 64, 2), (100, 1 << 30, 64, 2)):
            assert size(*bad) == -1, bad
        assert size(0, 0, 64, 2) == 0
    for bad in ((-1, 64, 2), (100, 12, 2), (100, 64, 3), (1 << 30, 64, 2)):
        assert lib.softmax_layer_norm_bwd_workspace(*bad) == -1


def test_launch_limits():
    """Tiles past a launch's number of threads."""
    assert nll_fwd(rows=1 << 20, vocab=1 << 18) != BAD
    assert nll_fwd(rows=1 << 20, vocab=1 << 20) == BAD
    assert nll_fwd(rows=1 << 29, vocab=1 << 29) == BAD
    assert nll_bwd(rows=1 << 20, vocab=1 << 20) == BAD
    assert embed_fwd(tokens=1 << 29, d=16384) == BAD
    assert sm.load_library().softmax_linear_nll_fwd_workspace(1 << 20, 1 << 20, 64, 2) == -1


def test_numbers_are_refused():
    for scale in (math.nan, math.inf, -math.inf):
        assert embed_fwd(scale=scale) == BAD and embed_bwd(scale=scale) == BAD
    for eps in (math.nan, math.inf, -1e-5):
        assert norm_fwd(eps=eps) == BAD
    assert norm_fwd(eps=0.0) != BAD
    for center in (-1, 2):
        assert norm_fwd(center=center) == BAD
    assert norm_fwd(center=0) == BAD                     # a mean that is not written
    assert norm_fwd(center=0, mean=None) != BAD
    assert nll_fwd(vocab=0) == BAD and nll_bwd(vocab=0) == BAD


def test_nothing_to_do():
    """No rows: nothing is touched, also where pointers are null."""
    assert nll_fwd(rows=0, x=None, labels=None, loss=None, lse=None, work=None, room=0) == sm.OK
    assert nll_bwd(rows=0, x=None, labels=None, dloss=None, dx=None, dw=None, work=None,
                   room=0) == sm.OK
    assert embed_fwd(tokens=0, ids=None, out=None) == sm.OK
    assert embed_bwd(rows=0, dtable=None, work=None, room=0) == sm.OK
    assert norm_fwd(rows=0, x=None, y=None, mean=None, rstd=None) == sm.OK
    assert norm_bwd(rows=0, x=None, dy=None, rstd=None, dw=None, db=None, work=None,
                    room=0) == sm.OK


# ---------------------------------------------------------------------------
# The binding

def test_cpu_tensors_are_refused():
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: sm.softmax_linear_nll_fwd(x, x, ids),
                 lambda: sm.softmax_linear_nll_bwd(x[:, 0], x, x, ids, x[:, 0], x[:, 0]),
                 lambda: sm.softmax_linear_nll(x, x, ids),
                 lambda: sm.softmax_embedding_fwd(ids, x), lambda: sm.softmax_embedding(ids, x),
                 lambda: sm.softmax_embedding_bwd(x, ids, 3),
                 lambda: sm.softmax_layer_norm_fwd(x), lambda: sm.softmax_layer_norm(x),
                 lambda: sm.softmax_layer_norm_bwd(x, x, None, None, x[:, 0])):
        with pytest.raises(ValueError, match="GPU"):
            call()


@pytest.fixture
def calls(monkeypatch):
    """The binding's calls reach a stand-in for the library."""
    at._lib()
    monkeypatch.setattr(sm, "load_library", Library)
    monkeypatch.setattr(sm, "_run", lambda fn, device, stream, args: sm.OK)
    monkeypatch.setattr(sm, "_empty", lambda shape, dtype, device, stream, returned=True:
                        torch.empty(shape, dtype=dtype).as_subclass(OnGpu))
    monkeypatch.setattr(at, "_fns", Library())


def test_bad_tensors_are_refused(calls):
    x, w, f = gpu(6, 16), gpu(9, 16), gpu(6)
    ids = gpu(6, dtype=torch.int64)
    sm.softmax_linear_nll_fwd(x, w, ids)
    sm.softmax_linear_nll_bwd(f, x, w, ids, f, f)
    sm.softmax_embedding_fwd(ids, w)
    sm.softmax_embedding_bwd(x, ids, 9)
    sm.softmax_layer_norm_fwd(x, x[0], x[1])
    sm.softmax_layer_norm_bwd(x, x, x[0], f, f, bias=True)
    half, long, flat = x.half(), gpu(7, dtype=torch.int64), gpu(16)
    wrong = [
        lambda: sm.softmax_linear_nll_fwd(x.double(), w.double(), ids),
        lambda: sm.softmax_linear_nll_fwd(x, w.half(), ids),
        lambda: sm.softmax_linear_nll_fwd(x, w, ids.int()),
        lambda: sm.softmax_linear_nll_bwd(f.half(), x, w, ids, f, f),
        lambda: sm.softmax_embedding_fwd(ids.int(), w),
        lambda: sm.softmax_embedding_fwd(ids, w.double()),
        lambda: sm.softmax_layer_norm_fwd(x, half[0]),
        lambda: sm.softmax_layer_norm_bwd(half, x, x[0], f, f),
        lambda: sm.softmax_layer_norm_bwd(x, x, x[0], f, f.half()),
        lambda: sm.softmax_layer_norm_fwd([1.0]),
    ]
    for call in wrong:
        with pytest.raises(TypeError):
            call()
    wrong = [
        lambda: sm.softmax_linear_nll_fwd(flat, w, ids),
        lambda: sm.softmax_linear_nll_fwd(x, gpu(9, 8), ids),
        lambda: sm.softmax_linear_nll_fwd(x, w, long),
        lambda: sm.softmax_linear_nll_fwd(x, gpu(0, 16), ids),
        lambda: sm.softmax_linear_nll_fwd(x.t(), w.t(), ids),
        lambda: sm.softmax_linear_nll_fwd(x, w, ids, loss=gpu(7)),
        lambda: sm.softmax_linear_nll_fwd(x, w, ids, lse=gpu(6, dtype=torch.float64)),
        lambda: sm.softmax_linear_nll_bwd(f, x, w, ids, f, gpu(5)),
        lambda: sm.softmax_linear_nll_bwd(gpu(1).expand(6), x, w, ids, f, f),
        lambda: sm.softmax_linear_nll_bwd(f, x, w, ids, f, f, dx=gpu(6, 8)),
        lambda: sm.softmax_linear_nll_bwd(f, x, w, ids, f, f, dweight=gpu(16, 9).t()),
        lambda: sm.softmax_embedding_fwd(gpu(2, 3, dtype=torch.int64), w),
        lambda: sm.softmax_embedding_fwd(ids, w, out=gpu(5, 16)),
        lambda: sm.softmax_embedding_bwd(x, long, 9),
        lambda: sm.softmax_embedding_bwd(x, ids, 9, dtable=gpu(8, 16)),
        lambda: sm.softmax_layer_norm_fwd(x, gpu(8)),
        lambda: sm.softmax_layer_norm_fwd(x, None, gpu(32)[::2]),
        lambda: sm.softmax_layer_norm_bwd(gpu(5, 16), x, x[0], f, f),
        lambda: sm.softmax_layer_norm_bwd(x, x, x[0], gpu(5), f),
        lambda: sm.softmax_layer_norm_bwd(x, x, x[0], f, f, dx=gpu(16, 6).t()),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            print(i)


def test_returned_values(calls):
    """What is not asked for is None; tensors that are given are returned, and
    count as written."""
    x, w, f = gpu(6, 16), gpu(9, 16), gpu(6)
    ids, out = gpu(6, dtype=torch.int64), gpu(6, 16)
    before = out._version
    assert sm.softmax_embedding_fwd(ids, w, out=out) is out and out._version > before
    dx, dw = sm.softmax_linear_nll_bwd(f, x, w, ids, f, f, need_dx=False)
    assert dx is None and dw.shape == (9, 16)
    assert sm.softmax_linear_nll_bwd(f, x, w, ids, f, f, need_dx=False, need_dweight=False) == \
        (None, None)
    y, mean, rstd = sm.softmax_layer_norm_fwd(x, center=False)
    assert y.shape == (6, 16) and mean is None and rstd.shape == (6,)
    dx, dw, db = sm.softmax_layer_norm_bwd(x, x, None, None, rstd)
    assert dx.shape == (6, 16) and dw is None and db is None


def stream_calls():
    x, w, f = gpu(6, 16), gpu(9, 16), gpu(6)
    ids = gpu(6, dtype=torch.int64)
    return {
        "nll": lambda s: sm.softmax_linear_nll_fwd(x, w, ids, stream=s),
        "nll_bwd": lambda s: sm.softmax_linear_nll_bwd(f, x, w, ids, f, f, stream=s),
        "embedding": lambda s: [sm.softmax_embedding_fwd(ids, w, stream=s)],
        "embedding_bwd": lambda s: [sm.softmax_embedding_bwd(x, ids, 9, stream=s)],
        "norm": lambda s: sm.softmax_layer_norm_fwd(x, stream=s),
        "norm_bwd": lambda s: sm.softmax_layer_norm_bwd(x, x, x[0], f, f, bias=True, stream=s),
    }


@pytest.mark.parametrize("name", stream_calls())
def test_allocations_belong_to_the_stream(name, monkeypatch):
    at._lib()
    current, made, kept = ["main"], [], []

    class Stream:
        cuda_stream = 7

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    real = torch.empty

    def allocate(*args, **how):
        t = real(*args, **how).as_subclass(OnGpu)
        made.append((t.data_ptr(), current[-1]))
        return t

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: current[-1])
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(OnGpu, "record_stream", lambda t, s: kept.append((t.data_ptr(), s)))
    monkeypatch.setattr(sm, "load_library", Library)
    monkeypatch.setattr(sm, "_run", lambda fn, device, stream, args: sm.OK)
    monkeypatch.setattr(at, "_fns", Library())
    side = Stream()
    got = stream_calls()[name](side)
    assert made and all(stream is side for _, stream in made)
    assert all((t.data_ptr(), "main") in kept for t in got)
    made.clear()
    stream_calls()[name](None)
    assert made and all(stream == "main" for _, stream in made)


# ---------------------------------------------------------------------------
# The oracle

def test_oracle_nll_is_torch_autograd():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(7, 12, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(5, 12, generator=g, dtype=torch.float64, requires_grad=True)
    labels, dloss = torch.tensor([0, 4, -100, 2, 2, -100, 1]), torch.rand(7, generator=g)
    loss, lse, dx, dw, *_ = oracle.linear_nll(x.detach(), w.detach(), labels, dloss=dloss)
    want = torch.nn.functional.cross_entropy(x @ w.t(), labels, reduction="none")
    torch.testing.assert_close(loss, want.detach())
    grads = torch.autograd.grad((want * dloss).sum(), (x, w))
    torch.testing.assert_close((dx, dw), grads)
    assert oracle.linear_nll(x.detach(), w.detach(), torch.tensor([5] * 7))[0].isnan().all()


def test_oracle_of_equal_logits():
    loss, lse = oracle.linear_nll(torch.zeros(3, 8), torch.randn(10, 8), torch.tensor([0, 1, 9]))
    torch.testing.assert_close(loss, torch.full((3,), math.log(10), dtype=torch.float64))
    torch.testing.assert_close(lse, loss)


def test_oracle_embedding_is_torch_autograd():
    g = torch.Generator().manual_seed(1)
    table = torch.randn(5, 8, generator=g, dtype=torch.float64, requires_grad=True)
    ids, dout = torch.tensor([1, 1, 4, 0]), torch.randn(4, 8, generator=g, dtype=torch.float64)
    out = torch.nn.functional.embedding(ids, table) * 3.0
    torch.testing.assert_close(oracle.embedding(ids, table.detach(), 3.0), out.detach())
    grad, = torch.autograd.grad(out, table, dout)
    torch.testing.assert_close(oracle.embedding_grad(dout, ids, 5, 3.0), grad)
    wrong = torch.tensor([-1, 5, 1 << 40, 2])
    assert not oracle.embedding(wrong, table.detach())[:3].any()
    assert int(oracle.embedding_grad(dout, wrong, 5).any(1).sum()) == 1


@pytest.mark.parametrize("center", [True, False])
def test_oracle_norm_is_torch_autograd(center):
    g = torch.Generator().manual_seed(1)
    leaves = [torch.randn(*s, generator=g, dtype=torch.float64, requires_grad=True)
              for s in ((6, 8), (8,), (8,))]
    x, w, b = leaves
    dy = torch.randn(6, 8, generator=g, dtype=torch.float64)
    if center:
        y = torch.nn.functional.layer_norm(x, (8,), w, b, 1e-5)
    else:
        y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-5) * w + b
    got = oracle.layer_norm(*(t.detach() for t in leaves), 1e-5, center, dy)
    torch.testing.assert_close(got[0], y.detach())
    torch.testing.assert_close(tuple(got[3:]), torch.autograd.grad(y, leaves, dy))
