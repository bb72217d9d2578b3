"""Python binding of what a decoder has around its attention
(include/decoder_mi355x.h): the loss of hidden states against a vocabulary, rows
of an embedding table, and the norm of rows.

Argument marshalling only, as for the rest of the package, whose functions these
join: every step runs in the HIP kernels, torch supplies device memory and the
current stream, and there is no fallback.

    softmax_linear_nll(x, weight, labels, ...) -> loss, with gradients (torch.autograd)
    softmax_linear_nll_fwd(x, weight, labels, ...) -> (loss, lse)
    softmax_linear_nll_bwd(dloss, x, weight, labels, loss, lse, ...) -> (dx, dweight)
    softmax_embedding(ids, table, ...) -> rows, with gradients
    softmax_embedding_fwd(ids, table, ...) -> rows
    softmax_embedding_bwd(dout, ids, rows, ...) -> dtable
    softmax_layer_norm(x, weight=None, bias=None, ...) -> y, with gradients
    softmax_layer_norm_fwd(x, weight=None, bias=None, ...) -> (y, mean, rstd)
    softmax_layer_norm_bwd(dy, x, weight, mean, rstd, ...) -> (dx, dweight, dbias)

Only the functions without a suffix record a graph: the results of the others are
constants for torch.autograd, also where inputs require gradients.
"""
from __future__ import annotations

import ctypes

import paper_1904_12380_amd as _sm

from .attention import _checked, _dtypes, _last_dim, _lib, _output, _tensor, _vector

MAX_WIDTH = 16384
MAX_ROW_STRIDE = 1048576

_i64, _i32, _f32, _vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p


def declare(lib: ctypes.CDLL) -> None:
    """Argument types of the entry points, for the loader of the library."""
    matrix = [_vp, _i64]
    sizes = [_i64, _i64, _i64]
    work = [_vp, _i64, _vp]
    for name, args, result in (
            ("linear_nll_fwd_workspace", [*sizes, _i32], _i64),
            ("linear_nll_fwd", [*matrix, *matrix, _vp, *sizes, _i64, _i32, _vp, _vp, *work], _i32),
            ("linear_nll_bwd_workspace", [*sizes, _i32], _i64),
            ("linear_nll_bwd", [_vp, *matrix, *matrix, _vp, *sizes, _i64, _i32, _vp, _vp, _vp, _vp,
                                *work], _i32),
            ("embedding_fwd", [_vp, _i64, *matrix, _i64, _i64, _f32, _i32, _vp, _vp], _i32),
            ("embedding_bwd_workspace", [*sizes, _i32], _i64),
            ("embedding_bwd", [*matrix, _vp, *sizes, _f32, _i32, _vp, *work], _i32),
            ("layer_norm_fwd", [*matrix, _vp, _vp, _i64, _i64, _f32, _i32, _i32, _vp, _vp, _vp,
                                _vp], _i32),
            ("layer_norm_bwd_workspace", [_i64, _i64, _i32], _i64),
            ("layer_norm_bwd", [*matrix, *matrix, _vp, _vp, _vp, _i64, _i64, _i32, _vp, _vp, _vp,
                                *work], _i32)):
        fn = getattr(lib, "softmax_" + name)
        fn.argtypes, fn.restype = args, result


def _rows(t, name: str, like=None):
    """(pointer, stride of the rows, rows, d) of a matrix."""
    _tensor(t, name, 2)
    if like is None:
        if t.dtype not in _dtypes:
            raise TypeError(f"{name} must be float32, float16 or bfloat16, got {t.dtype}")
    elif t.dtype != like.dtype or t.device != like.device:
        raise TypeError(f"{name} must have the type and device of the other tensors")
    strides = t.stride()
    _last_dim(strides, t, name)
    # The stride of a dimension of one is never used, and torch leaves it odd.
    return t.data_ptr(), strides[0] if t.shape[0] > 1 else 0, *t.shape


def _work(room: int, device, stream):
    """(memory, its pointer, its bytes) of a call's workspace."""
    if room <= 0:
        return None, None, 0
    work = _sm._empty(room, _sm._torch_mod.uint8, device, stream, returned=False)
    return work, work.data_ptr(), room


def _nll_sizes(x, weight, labels):
    px, sx, rows, d = _rows(x, "x")
    pw, sw, vocab, width = _rows(weight, "weight", x)
    if width != d:
        raise ValueError(f"weight must be [vocab, {d}] as x is [rows, {d}], got {width} columns")
    if rows > 0 and vocab == 0:
        raise ValueError("weight must have a row at least")
    pl = _vector(labels, "labels", _sm._torch_mod.int64, rows, x.device)
    return px, sx, pw, sw, pl, rows, vocab, d


def softmax_linear_nll_fwd(x, weight, labels, *, ignore: int = -100, loss=None, lse=None,
                           stream=None):
    """Per-row negative log-likelihood of ``labels`` (int64 [rows]) under the
    softmax of the logits x weight^T, which are not kept: x [rows, d] and weight
    [vocab, d] in float32, float16 or bfloat16.

    Rows whose label is ``ignore`` get a loss and lse of 0; a label outside [0,
    vocab) else gives NaN.  Returns float32 (loss [rows], lse [rows])."""
    fn = _lib().softmax_linear_nll_fwd
    f32 = _sm._torch_mod.float32
    px, sx, pw, sw, pl, rows, vocab, d = _nll_sizes(x, weight, labels)
    device, dtype = x.device, _dtypes[x.dtype]
    loss = _output(loss, (rows,), f32, device, "loss", stream)
    lse = _output(lse, (rows,), f32, device, "lse", stream)
    room = _lib().softmax_linear_nll_fwd_workspace(rows, vocab, d, dtype)
    work, at, room = _work(room, device, stream)
    _checked(_sm._run(fn, device, stream,
                      (px, sx, pw, sw, pl, rows, vocab, d, ignore, dtype, loss.data_ptr(),
                       lse.data_ptr(), at, room)),
             "softmax_linear_nll_fwd")
    return loss, lse


def softmax_linear_nll_bwd(dloss, x, weight, labels, loss, lse, *, ignore: int = -100,
                           need_dx: bool = True, need_dweight: bool = True, dx=None,
                           dweight=None, stream=None):
    """Gradients (dx [rows, d], dweight [vocab, d]) of softmax_linear_nll_fwd with
    the same arguments, from its ``loss`` and ``lse`` and the gradient ``dloss``
    (float32 [rows]) of loss.  None for one that is not needed."""
    fn = _lib().softmax_linear_nll_bwd
    f32 = _sm._torch_mod.float32
    px, sx, pw, sw, pl, rows, vocab, d = _nll_sizes(x, weight, labels)
    device, dtype = x.device, _dtypes[x.dtype]
    given = [_vector(t, name, f32, rows, device)
             for t, name in ((dloss, "dloss"), (loss, "loss"), (lse, "lse"))]
    dx = _output(dx, (rows, d), x.dtype, device, "dx", stream) if need_dx else None
    dweight = _output(dweight, (vocab, d), x.dtype, device, "dweight", stream) \
        if need_dweight else None
    room = 0
    if need_dx or need_dweight:
        room = _lib().softmax_linear_nll_bwd_workspace(rows, vocab, d, dtype)
    work, at, room = _work(room, device, stream)
    if need_dx or need_dweight:
        _checked(_sm._run(fn, device, stream,
                          (given[0], px, sx, pw, sw, pl, rows, vocab, d, ignore, dtype, given[1],
                           given[2], None if dx is None else dx.data_ptr(),
                           None if dweight is None else dweight.data_ptr(), at, room)),
                 "softmax_linear_nll_bwd")
    return dx, dweight


def softmax_embedding_fwd(ids, table, *, scale: float = 1.0, out=None, stream=None):
    """Rows scale * table[ids] ([tokens, d]) of a table [rows, d] in float32,
    float16 or bfloat16; ids outside [0, rows) (int64 [tokens]), such as -1, are
    padding and get zeros."""
    fn = _lib().softmax_embedding_fwd
    pt, st, rows, d = _rows(table, "table")
    pi = _vector(ids, "ids", _sm._torch_mod.int64, None, table.device)
    out = _output(out, (len(ids), d), table.dtype, table.device, "out", stream)
    _checked(_sm._run(fn, table.device, stream,
                      (pi, len(ids), pt, st, rows, d, scale, _dtypes[table.dtype],
                       out.data_ptr())),
             "softmax_embedding_fwd")
    return out


def softmax_embedding_bwd(dout, ids, rows: int, *, scale: float = 1.0, dtable=None, stream=None):
    """Gradient [rows, d] of the table of softmax_embedding_fwd, from the gradient
    ``dout`` [tokens, d] of its rows: sums over the tokens of each id, in fp32, the
    same bits each time."""
    fn = _lib().softmax_embedding_bwd
    pd, sd, tokens, d = _rows(dout, "dout")
    device, dtype = dout.device, _dtypes[dout.dtype]
    pi = _vector(ids, "ids", _sm._torch_mod.int64, tokens, device)
    dtable = _output(dtable, (rows, d), dout.dtype, device, "dtable", stream)
    work, at, room = _work(_lib().softmax_embedding_bwd_workspace(tokens, rows, d, dtype), device,
                           stream)
    _checked(_sm._run(fn, device, stream,
                      (pd, sd, pi, tokens, rows, d, scale, dtype, dtable.data_ptr(), at, room)),
             "softmax_embedding_bwd")
    return dtable


def _columns(t, name, x, d):
    return None if t is None else _vector(t, name, x.dtype, d, x.device)


def softmax_layer_norm_fwd(x, weight=None, bias=None, *, eps: float = 1e-5, center: bool = True,
                           out=None, stream=None):
    """Rows of x [rows, d] (float32, float16 or bfloat16) brought to mean 0 and
    variance 1, or without ``center`` to mean square 1, then times ``weight`` plus
    ``bias`` ([d] of x's type; None: ones, zeros).  Returns (y, mean, rstd), the
    last two float32 [rows], mean None without ``center``."""
    fn = _lib().softmax_layer_norm_fwd
    f32 = _sm._torch_mod.float32
    px, sx, rows, d = _rows(x, "x")
    pw, pb = _columns(weight, "weight", x, d), _columns(bias, "bias", x, d)
    y = _output(out, (rows, d), x.dtype, x.device, "out", stream)
    mean = _sm._empty(rows, f32, x.device, stream) if center else None
    rstd = _sm._empty(rows, f32, x.device, stream)
    _checked(_sm._run(fn, x.device, stream,
                      (px, sx, pw, pb, rows, d, eps, 1 if center else 0, _dtypes[x.dtype],
                       y.data_ptr(), None if mean is None else mean.data_ptr(),
                       rstd.data_ptr())),
             "softmax_layer_norm_fwd")
    return y, mean, rstd


def softmax_layer_norm_bwd(dy, x, weight, mean, rstd, *, bias: bool = False,
                           need_dx: bool = True, need_dweight: bool = True, dx=None,
                           dweight=None, dbias=None, stream=None):
    """Gradients (dx, dweight, dbias) of softmax_layer_norm_fwd, from its ``mean``
    (None without center) and ``rstd`` and the gradient ``dy`` of y.  dbias only
    with ``bias``, dweight only where there is a weight; None for one that is not
    needed."""
    fn = _lib().softmax_layer_norm_bwd
    f32 = _sm._torch_mod.float32
    px, sx, rows, d = _rows(x, "x")
    py, sy, *shape = _rows(dy, "dy", x)
    if shape != [rows, d]:
        raise ValueError(f"dy must be [{rows}, {d}] as x is, got {shape}")
    pw = _columns(weight, "weight", x, d)
    pm = None if mean is None else _vector(mean, "mean", f32, rows, x.device)
    pr = _vector(rstd, "rstd", f32, rows, x.device)
    need_dweight = need_dweight and weight is not None
    dx = _output(dx, (rows, d), x.dtype, x.device, "dx", stream) if need_dx else None
    dweight = _output(dweight, (d,), x.dtype, x.device, "dweight", stream) if need_dweight else None
    dbias = _output(dbias, (d,), x.dtype, x.device, "dbias", stream) if bias else None
    room = 0
    if need_dweight or bias:
        room = _lib().softmax_layer_norm_bwd_workspace(rows, d, _dtypes[x.dtype])
    work, at, room = _work(room, x.device, stream)
    _checked(_sm._run(fn, x.device, stream,
                      (py, sy, px, sx, pw, pm, pr, rows, d, _dtypes[x.dtype],
                       None if dx is None else dx.data_ptr(),
                       None if dweight is None else dweight.data_ptr(),
                       None if dbias is None else dbias.data_ptr(), at, room)),
             "softmax_layer_norm_bwd")
    return dx, dweight, dbias


def _as_rows(t):
    """A gradient's layout is what the operation behind it left: a copy where the
    kernels do not take it."""
    strip = 16 // t.element_size()
    rows, columns = t.stride()
    if (columns == 1 or t.shape[1] == 1) and (rows % strip == 0 or t.shape[0] == 1) and \
            t.data_ptr() % 16 == 0:
        return t
    return t.clone(memory_format=_sm._torch_mod.contiguous_format)


_functions = None


def _differentiable():
    global _functions
    if _functions is not None:
        return _functions
    torch = _sm._torch()
    once = torch.autograd.function.once_differentiable

    class LinearNll(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, labels, ignore):
            loss, lse = softmax_linear_nll_fwd(x, weight, labels, ignore=ignore)
            ctx.save_for_backward(x, weight, labels, loss, lse)
            ctx.ignore = ignore
            return loss

        @staticmethod
        @once
        def backward(ctx, dloss):
            x, weight, labels, loss, lse = ctx.saved_tensors
            dx, dweight = softmax_linear_nll_bwd(
                dloss.contiguous(), x, weight, labels, loss, lse, ignore=ctx.ignore,
                need_dx=ctx.needs_input_grad[0], need_dweight=ctx.needs_input_grad[1])
            return dx, dweight, None, None

    class Embedding(torch.autograd.Function):
        @staticmethod
        def forward(ctx, ids, table, scale):
            ctx.save_for_backward(ids)
            ctx.rows, ctx.scale = table.shape[0], scale
            return softmax_embedding_fwd(ids, table, scale=scale)

        @staticmethod
        @once
        def backward(ctx, dout):
            ids, = ctx.saved_tensors
            return None, softmax_embedding_bwd(_as_rows(dout), ids, ctx.rows,
                                               scale=ctx.scale), None

    class LayerNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, eps, center):
            y, mean, rstd = softmax_layer_norm_fwd(x, weight, bias, eps=eps, center=center)
            ctx.save_for_backward(x, weight, mean, rstd)
            return y

        @staticmethod
        @once
        def backward(ctx, dy):
            x, weight, mean, rstd = ctx.saved_tensors
            needs = ctx.needs_input_grad
            grads = softmax_layer_norm_bwd(_as_rows(dy), x, weight, mean, rstd, bias=needs[2],
                                           need_dx=needs[0], need_dweight=needs[1])
            return (*grads, None, None)

    _functions = LinearNll, Embedding, LayerNorm
    return _functions


def softmax_linear_nll(x, weight, labels, *, ignore: int = -100):
    """softmax_linear_nll_fwd's loss, differentiable in x and weight."""
    return _differentiable()[0].apply(x, weight, labels, ignore)


def softmax_embedding(ids, table, *, scale: float = 1.0):
    """softmax_embedding_fwd, differentiable in the table."""
    return _differentiable()[1].apply(ids, table, scale)


def softmax_layer_norm(x, weight=None, bias=None, *, eps: float = 1e-5, center: bool = True):
    """softmax_layer_norm_fwd's y, differentiable in x, weight and bias."""
    return _differentiable()[2].apply(x, weight, bias, eps, center)
