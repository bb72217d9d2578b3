"""Python binding of the attention of language models (include/attention_mi355x.h).

Argument marshalling only, as for the rest of the package, whose functions
these join: every step runs in the HIP kernels, torch supplies device memory
and the current stream, and there is no fallback.

    softmax_packed_attention(q, k, v, cu_q, ...) -> o, with gradients (torch.autograd)
    softmax_packed_attention_fwd(q, k, v, cu_q, cu_k=None, ...) -> (o, lse)
    softmax_packed_attention_bwd(dout, q, k, v, o, lse, cu_q, cu_k=None, ...) -> (dq, dk, dv)
    softmax_paged_attention_fwd(q, k_cache, v_cache, block_table, cu_q, key_lens, ...) -> o
    softmax_cache_slots(context_lens, new_lens, block_table, free_blocks, free_count, total,
                        block_size) -> dict
    softmax_cache_append(k, v, k_cache, v_cache, slots)

Only softmax_packed_attention records a graph: the results of the other
functions are constants for torch.autograd, also where inputs require gradients.
"""
from __future__ import annotations

import ctypes

import paper_1904_12380_amd as _sm

HEADS_MAX_DIM = 256
HEADS_MAX_STRIDE = 8388608

_i64, _i32, _f32, _vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p


class _Heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("tokens", _i64), ("heads", _i64), ("d", _i64),
                ("token_stride", _i64), ("head_stride", _i64)]


class _Cache(ctypes.Structure):
    _fields_ = [("data", _vp), ("blocks", _i64), ("block_size", _i64), ("heads", _i64),
                ("d", _i64), ("block_stride", _i64), ("token_stride", _i64),
                ("head_stride", _i64)]


class _Score(ctypes.Structure):
    _fields_ = [("scale", _f32), ("cap", _f32), ("causal", _i32), ("slopes", _vp),
                ("prefix", _vp)]


_fns = None
_dtypes = {}


def declare(lib: ctypes.CDLL) -> None:
    """Argument types of the entry points, for the loader of the library."""
    heads, cache, score = map(ctypes.POINTER, (_Heads, _Cache, _Score))
    for name, args, result in (
            ("packed_attention_fwd", [heads, heads, heads, _vp, _vp, _vp, _vp, _i64, score,
                                      ctypes.c_int, _vp], ctypes.c_int),
            ("packed_attention_bwd_workspace", [_i64] * 5 + [ctypes.c_int], _i64),
            ("packed_attention_bwd", [heads] * 5 + [_vp] * 6 + [_i64, score, ctypes.c_int, _vp,
                                                                _i64, _vp], ctypes.c_int),
            ("paged_attention_workspace", [_i64] * 6, _i64),
            ("paged_attention_fwd", [heads, cache, cache, _vp, _i64, _vp, _vp, _i64, score,
                                     ctypes.c_int, _vp, _vp, _vp, _i64, _vp], ctypes.c_int),
            ("cache_slots", [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp,
                             _i64, _vp, _vp, _vp], ctypes.c_int),
            ("cache_append", [heads, heads, cache, cache, _vp, ctypes.c_int, _vp],
             ctypes.c_int)):
        fn = getattr(lib, "softmax_" + name)
        fn.argtypes, fn.restype = args, result


def _lib():
    global _fns
    if _fns is None:
        torch = _sm._torch()
        _dtypes.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
        _fns = _sm.load_library()
    return _fns


def _tensor(t, name: str, dims: int):
    torch = _sm._torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (no CPU path exists)")
    if t.dim() != dims:
        raise ValueError(f"{name} must have {dims} dimensions, got {t.dim()}")


def _last_dim(strides, t, name):
    if strides[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")


def _heads(t, name: str, like=None) -> _Heads:
    _tensor(t, name, 3)
    if like is None:
        if t.dtype not in _dtypes:
            raise TypeError(f"{name} must be float32, float16 or bfloat16, got {t.dtype}")
    elif t.dtype != like.dtype or t.device != like.device:
        raise TypeError(f"{name} must have the type and device of the other tensors")
    strides = t.stride()
    _last_dim(strides, t, name)
    tokens, heads, d = t.shape
    # The stride of a dimension of one is never used, and torch leaves it odd.
    return _Heads(t.data_ptr(), tokens, heads, d, strides[0] if tokens > 1 else 0,
                  strides[1] if heads > 1 else 0)


def _cache(t, name: str, like) -> _Cache:
    _tensor(t, name, 4)
    if t.dtype != like.dtype or t.device != like.device:
        raise TypeError(f"{name} must have the type and device of the other tensors")
    strides = t.stride()
    _last_dim(strides, t, name)
    blocks, size, heads, d = t.shape
    return _Cache(t.data_ptr(), blocks, size, heads, d, strides[0] if blocks > 1 else 0,
                  strides[1] if size > 1 else 0, strides[2] if heads > 1 else 0)


def _vector(t, name: str, dtype, count, device) -> int:
    """Pointer of a contiguous vector (count None: any length)."""
    try:
        if t.dtype is dtype and t.device == device and t.dim() == 1 and t.is_contiguous() and \
                (count is None or t.numel() == count):
            return t.data_ptr()
    except AttributeError:
        pass  # no tensor: said below
    _tensor(t, name, 1)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device or not t.is_contiguous() or (count is not None and len(t) != count):
        raise ValueError(f"{name} must be contiguous, {'' if count is None else f'[{count}], '}"
                         "on the device of the other tensors")
    return t.data_ptr()


def _score(q, docs, causal, scale, cap, slopes, prefix) -> _Score:
    torch = _sm._torch_mod
    if scale is None:
        scale = max(q.shape[2], 1) ** -0.5
    return _Score(
        scale, cap, 1 if causal else 0,
        None if slopes is None else _vector(slopes, "slopes", torch.float32, q.shape[1], q.device),
        None if prefix is None else _vector(prefix, "prefix", torch.int32, docs, q.device))


def _output(out, shape, dtype, device, name, stream):
    if out is None:
        return _sm._empty(shape, dtype, device, stream)
    _tensor(out, name, len(shape))
    if out.dtype != dtype or tuple(out.shape) != tuple(shape) or out.device != device or \
            not out.is_contiguous():
        raise ValueError(f"{name} must be contiguous {list(shape)} of {dtype} on the device of "
                         "the other tensors")
    _written(out)
    return out


def _written(*tensors) -> None:
    """Counts a write of the caller's tensors, as torch's own in-place
    operations do: a backward pass that saved their former values is refused."""
    _sm._torch_mod.autograd.graph.increment_version(tensors)


def _checked(rc: int, what: str) -> None:
    if rc != _sm.OK:
        raise _sm.SoftmaxError(rc, what)


def _docs(cu_q, cu_k, q):
    torch = _sm._torch_mod
    _tensor(cu_q, "cu_q", 1)
    docs = len(cu_q) - 1
    if docs < 0:
        raise ValueError("cu_q must have one entry more than there are documents")
    pq = _vector(cu_q, "cu_q", torch.int32, None, q.device)
    return docs, pq, pq if cu_k is None else _vector(cu_k, "cu_k", torch.int32, docs + 1,
                                                     q.device)


def softmax_packed_attention_fwd(q, k, v, cu_q, cu_k=None, *, causal=True, scale=None,
                                 cap: float = 0.0, slopes=None, prefix=None, out=None, lse=None,
                                 stream=None):
    """Attention of packed documents: q [tokens, heads, d], k and v [tokens,
    kv_heads, d] in float32, float16 or bfloat16, document b at tokens
    cu_q[b] .. cu_q[b + 1] - 1 (int32 [docs + 1]; ``cu_k`` for keys of other
    lengths than the queries).

    ``scale`` defaults to 1/sqrt(d); ``cap`` > 0 caps scores with a tanh;
    ``slopes`` (float32 [heads]) subtracts slope * distance; ``causal`` hides
    later keys but the first ``prefix`` (int32 [docs]) of each document.
    Returns (o like q, float32 lse [tokens, heads])."""
    fn = _lib().softmax_packed_attention_fwd
    aq, ak, av = _heads(q, "q"), _heads(k, "k", q), _heads(v, "v", q)
    docs, pq, pk = _docs(cu_q, cu_k, q)
    if cu_k is None and k.shape[0] != q.shape[0]:
        raise ValueError("k must have q's tokens unless cu_k is given")
    score = _score(q, docs, causal, scale, cap, slopes, prefix)
    out = _output(out, q.shape, q.dtype, q.device, "out", stream)
    lse = _output(lse, q.shape[:2], _sm._torch_mod.float32, q.device, "lse", stream)
    _checked(_sm._run(fn, q.device, stream, (aq, ak, av, out.data_ptr(), lse.data_ptr(), pq, pk,
                                             docs, score, _dtypes[q.dtype])),
             "softmax_packed_attention_fwd")
    return out, lse


def softmax_packed_attention_bwd(dout, q, k, v, o, lse, cu_q, cu_k=None, *, causal=True,
                                 scale=None, cap: float = 0.0, slopes=None, prefix=None,
                                 dq=None, dk=None, dv=None, stream=None):
    """Gradients (dq, dk, dv) of softmax_packed_attention_fwd with the same
    arguments, from its ``o`` and ``lse`` and the gradient ``dout`` of o."""
    fn = _lib().softmax_packed_attention_bwd
    torch = _sm._torch_mod
    aq, ak, av = _heads(q, "q"), _heads(k, "k", q), _heads(v, "v", q)
    ao, ad = _heads(o, "o", q), _heads(dout, "dout", q)
    docs, pq, pk = _docs(cu_q, cu_k, q)
    if cu_k is None and k.shape[0] != q.shape[0]:
        raise ValueError("k must have q's tokens unless cu_k is given")
    score = _score(q, docs, causal, scale, cap, slopes, prefix)
    _tensor(lse, "lse", 2)
    if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or \
            lse.device != q.device:
        raise ValueError("lse must be contiguous float32 [tokens, heads]")
    dq = _output(dq, q.shape, q.dtype, q.device, "dq", stream)
    dk = _output(dk, k.shape, q.dtype, q.device, "dk", stream)
    dv = _output(dv, v.shape, q.dtype, q.device, "dv", stream)
    room = _fns.softmax_packed_attention_bwd_workspace(aq.tokens, ak.tokens, aq.heads, ak.heads,
                                                       aq.d, _dtypes[q.dtype])
    work = _sm._empty(max(room, 0), torch.uint8, q.device, stream, returned=False)
    _checked(_sm._run(fn, q.device, stream,
                      (ad, aq, ak, av, ao, lse.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                       dv.data_ptr(), pq, pk, docs, score, _dtypes[q.dtype], work.data_ptr(),
                       room)),
             "softmax_packed_attention_bwd")
    return dq, dk, dv


def _fits(t) -> bool:
    """Whether a tensor [tokens, heads, d] has the layout that the kernels take
    (a gradient's layout is what the operation behind it left)."""
    strip, (ts, hs, ds) = 16 // t.element_size(), t.stride()
    return ds == 1 and ts <= HEADS_MAX_STRIDE and ts % strip == hs % strip == 0 and \
        t.data_ptr() % 16 == 0


_function = None


def softmax_packed_attention(q, k, v, cu_q, cu_k=None, *, causal=True, scale=None,
                             cap: float = 0.0, slopes=None, prefix=None):
    """softmax_packed_attention_fwd's o, differentiable in q, k and v."""
    global _function
    if _function is None:
        torch = _sm._torch()

        class Attention(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, v, cu_q, cu_k, slopes, prefix, how):
                o, lse = softmax_packed_attention_fwd(q, k, v, cu_q, cu_k, slopes=slopes,
                                                      prefix=prefix, **how)
                ctx.save_for_backward(q, k, v, o, lse, cu_q, cu_k, slopes, prefix)
                ctx.how = how
                return o

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dout):
                q, k, v, o, lse, cu_q, cu_k, slopes, prefix = ctx.saved_tensors
                if not _fits(dout):
                    dout = dout.clone(memory_format=torch.contiguous_format)
                grads = softmax_packed_attention_bwd(dout, q, k, v, o, lse, cu_q, cu_k,
                                                     slopes=slopes, prefix=prefix, **ctx.how)
                return (*grads, None, None, None, None, None)

        _function = Attention
    if slopes is not None and slopes.requires_grad:
        raise ValueError("slopes get no gradient: they are constants")
    return _function.apply(q, k, v, cu_q, cu_k, slopes, prefix,
                           {"causal": causal, "scale": scale, "cap": cap})


def softmax_paged_attention_fwd(q, k_cache, v_cache, block_table, cu_q, key_lens, *, causal=True,
                                scale=None, cap: float = 0.0, slopes=None, prefix=None, out=None,
                                lse=None, stream=None):
    """Attention of new tokens q [tokens, heads, d] over a paged cache
    [blocks, block_size, kv_heads, d] that holds their keys and values too:
    request b has the tokens cu_q[b] .. cu_q[b + 1] - 1, the last of its
    key_lens[b] keys, which lie in the blocks block_table[b] (int32
    [requests, width]).  Scores as in softmax_packed_attention_fwd.  Returns o
    like q; ``lse`` (float32 [tokens, heads]) is written where given."""
    fn = _lib().softmax_paged_attention_fwd
    torch = _sm._torch_mod
    aq = _heads(q, "q")
    ak, av = _cache(k_cache, "k_cache", q), _cache(v_cache, "v_cache", q)
    device = q.device
    _tensor(block_table, "block_table", 2)
    requests, width = block_table.shape
    if block_table.dtype != torch.int32 or block_table.device != device or \
            not block_table.is_contiguous():
        raise ValueError("block_table must be contiguous int32 on the device of the other tensors")
    pq = _vector(cu_q, "cu_q", torch.int32, requests + 1, device)
    pk = _vector(key_lens, "key_lens", torch.int32, requests, device)
    score = _score(q, requests, causal, scale, cap, slopes, prefix)
    out = _output(out, q.shape, q.dtype, device, "out", stream)
    if lse is not None:
        lse = _output(lse, q.shape[:2], torch.float32, device, "lse", stream)
    room = _sm._on_device(device, _fns.softmax_paged_attention_workspace, aq.tokens, aq.heads,
                          ak.heads, aq.d, requests, width * ak.block_size)
    work = _sm._empty(room, torch.uint8, device, stream, returned=False) if room > 0 else None
    _checked(_sm._run(fn, device, stream,
                      (aq, ak, av, block_table.data_ptr(), width, pq, pk, requests, score,
                       _dtypes[q.dtype], out.data_ptr(), None if lse is None else lse.data_ptr(),
                       None if work is None else work.data_ptr(), room)),
             "softmax_paged_attention_fwd")
    return out


def softmax_cache_slots(context_lens, new_lens, block_table, free_blocks, free_count, total: int,
                        block_size: int, *, stream=None) -> dict:
    """The bookkeeping of a serving step (int32 tensors): requests of
    context_lens [n] tokens get new_lens [n] more.  The blocks that they need
    are taken from the top of the stack free_blocks, of which free_count [1]
    are left, and written into block_table [n, width].  Returns a dict of

        table       block_table itself
        cu_q        int32 [n + 1], sums of new_lens
        key_lens    int32 [n], context_lens + new_lens
        slots       int64 [total], the cache slot of each new token, -1 past
                    the last and for tokens without a block
        free_count  int32 [1], the ids left
        missing     int32 [1], blocks that were needed but not had
    """
    fn = _lib().softmax_cache_slots
    torch = _sm._torch_mod
    _tensor(block_table, "block_table", 2)
    n, width = block_table.shape
    device, i32 = block_table.device, torch.int32
    if block_table.dtype != i32 or not block_table.is_contiguous():
        raise ValueError("block_table must be contiguous int32")
    context = _vector(context_lens, "context_lens", i32, n, device)
    new = _vector(new_lens, "new_lens", i32, n, device)
    free = _vector(free_blocks, "free_blocks", i32, None, device)
    count = _vector(free_count, "free_count", i32, 1, device)
    _written(block_table)
    slots = _sm._empty(total, torch.int64, device, stream)
    sums = _sm._empty(2 * n + 3, i32, device, stream)
    at = sums.data_ptr()
    _checked(_sm._run(fn, device, stream,
                      (context, new, n, block_table.data_ptr(), width, free, len(free_blocks),
                       count, block_size, at, at + 4 * (n + 1), slots.data_ptr(), total,
                       at + 4 * (2 * n + 1), at + 4 * (2 * n + 2))),
             "softmax_cache_slots")
    cu_q, key_lens, left, missing = torch.split_with_sizes(sums, (n + 1, n, 1, 1))
    return {"table": block_table, "cu_q": cu_q, "key_lens": key_lens, "slots": slots,
            "free_count": left, "missing": missing}


def softmax_cache_append(k, v, k_cache, v_cache, slots, *, stream=None) -> None:
    """k[t] and v[t] ([tokens, heads, d]) into row slots[t] (int64 [tokens]) of
    the caches [blocks, block_size, heads, d]; slots of -1 are skipped."""
    fn = _lib().softmax_cache_append
    ak, av = _heads(k, "k"), _heads(v, "v", k)
    ck, cv = _cache(k_cache, "k_cache", k), _cache(v_cache, "v_cache", k)
    at = _vector(slots, "slots", _sm._torch_mod.int64, ak.tokens, k.device)
    _written(k_cache, v_cache)
    _checked(_sm._run(fn, k.device, stream, (ak, av, ck, cv, at, _dtypes[k.dtype])),
             "softmax_cache_append")
