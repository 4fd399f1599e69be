"""ctypes binding of include/bpe_head.h, the operators at a model's output end: argument marshalling only.

Streams, allocation, strides and refusals are as in ``_ops.py``.  ``add_norm`` and ``adjust_logits`` are recorded by torch's automatic
differentiation where what they are given wants a gradient; what is in 8 bits carries none, and is refused for a tensor that wants one.
Forward-mode derivatives are not computed: a tensor that carries one (a dual tensor) is refused, so that it is not lost.
(A training step that is captured in a graph takes its gradients from ``add_norm_grad`` and ``adjust_logits_grad``, or from
``torch.autograd.grad``: torch's ``backward()`` adds them up on the stream on which a parameter was first used, which need not be the one
that is captured.)"""
from __future__ import annotations

import ctypes

from . import _ops
from ._ops import _enqueue, _matrix, _no_tangent, _on, _pointer, _vector, _workspace

_lib = torch = _Norm = _Adjusted = _TYPES = _written = None      # (the package can be imported without torch)


def _load():
    global _lib, torch, _Norm, _Adjusted, _TYPES, _written
    if _lib is None:
        lib = _ops._load()
        torch, _TYPES, _written = _ops.torch, _ops._TYPES, _ops._written
        vp, i, i64, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        norm = [vp, i, i64, i64, i64, vp, i64, vp, i, f, vp, i64]
        histories, masks = [vp, i64, vp, vp, vp, f], [vp, i64, i64, vp]
        for name, args in {
                "add_norm": [*norm, vp, vp, i64, vp],
                "add_norm_8bit": [*norm, vp, i64, vp, vp],
                "add_norm_grad": [vp, i, i64, i64, i64, vp, i64, vp, i, vp, vp, i64, vp, i64, vp, i, i, vp, sz, vp],
                "quantize_rows": [vp, i, i64, i64, i64, vp, i64, vp, vp],
                "project_8bit": [vp, i64, i64, i64, vp, vp, i64, i64, vp, vp, i, i64, vp],
                "adjust_logits": [vp, i, i64, i64, i64, *histories, f, f, vp, vp, i64, vp, vp, *masks, vp, i64, vp],
                "adjust_logits_grad": [vp, i, i64, i64, i64, vp, i64, *histories, *masks, vp, i64, vp],
        }.items():
            function = getattr(lib, "bpe_" + name)
            function.argtypes, function.restype = args, i
        lib.bpe_add_norm_grad_workspace_bytes.argtypes = [i64, i64]
        lib.bpe_add_norm_grad_workspace_bytes.restype = sz
        _Norm, _Adjusted = _recorded()
        _lib = lib
    return _lib


def _recorded():
    """add_norm and adjust_logits as torch's automatic differentiation knows them."""
    once = torch.autograd.function.once_differentiable

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, residual, eps):
            out, summed, rstd = add_norm(x, weight, residual, eps)
            ctx.save_for_backward(summed, weight, rstd)
            ctx.mark_non_differentiable(rstd)
            ctx.set_materialize_grads(False)
            # (without a residual the sum is x itself, whose gradient passes by this function)
            return out, (None if residual is None else summed), rstd

        @staticmethod
        @once
        def backward(ctx, grad, grad_summed, _):
            summed, weight, rstd = ctx.saved_tensors
            if grad is None:
                return grad_summed, None, grad_summed, None
            grad_summed = None if grad_summed is None else grad_summed.contiguous()
            grad_x, grad_weight = add_norm_grad(grad.contiguous(), summed, weight, rstd, grad_summed, weights=ctx.needs_input_grad[1])
            return grad_x, grad_weight, grad_x if ctx.needs_input_grad[2] else None, None

    class Adjusted(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, ids, begin, end, penalties, bias, mask, state):
            rows = penalties if isinstance(penalties, torch.Tensor) else None
            if rows is None and penalties is not None:
                penalties = tuple(penalties)                 # (a list may be another one by the backward pass)
            ctx.save_for_backward(logits, ids, begin, end, rows, mask, state)
            ctx.penalties = None if rows is not None else penalties
            return adjust_logits(logits, ids, begin, end, penalties, bias, mask, state)

        @staticmethod
        @once
        def backward(ctx, grad):
            logits, ids, begin, end, rows, mask, state = ctx.saved_tensors
            penalties = ctx.penalties if rows is None else rows
            return adjust_logits_grad(grad.contiguous(), logits, ids, begin, end, penalties, mask, state), *[None] * 7

    return Norm, Adjusted


def _wants(*tensors):
    _no_tangent(*tensors)
    if torch.is_grad_enabled():
        for t in tensors:                                    # (not a generator's: half a microsecond of a small call's ten)
            if t is not None and t.requires_grad:
                return True
    return False


def _no_gradient(what, *tensors):
    if _wants(*tensors):
        raise ValueError(f"{what} carries no gradient: give detached tensors, or call under torch.no_grad()")


def _weight(weight, dev, dim, dtype):
    """(pointer, the library's number of its type) of a norm's weights."""
    if weight.dtype not in (torch.float32, dtype):
        raise ValueError(f"weight must be float32 or {dtype}")
    return _vector(weight, "weight", dev, weight.dtype, dim), _TYPES[weight.dtype]


def _sum(x, residual, summed):
    """(residual's pointer and stride, the sum's tensor, pointer and stride)"""
    if residual is None:
        if summed is not None:
            raise ValueError("summed needs a residual")
        return None, 0, x, None, 0
    stride = _matrix(residual, "residual", x.device, tuple(x.shape), x.dtype)
    if summed is None:
        summed = torch.empty_like(x, memory_format=torch.contiguous_format)
        return residual.data_ptr(), stride, summed, summed.data_ptr(), summed.shape[1]
    summed_stride = _matrix(summed, "summed", x.device, tuple(x.shape), x.dtype)
    _written((summed,))
    return residual.data_ptr(), stride, summed, summed.data_ptr(), summed_stride


def _bytes(t, what, dev=None, columns=None):
    """The stride between the rows of a matrix of 8-bit integers."""
    if not t.is_cuda or (dev is not None and t.device != dev):
        raise ValueError(f"{what} must be on {'the GPU' if dev is None else dev}")
    if t.dim() != 2 or t.dtype != torch.int8 or t.shape[1] < 1 or (columns is not None and t.shape[1] != columns):
        raise ValueError(f"{what} must be an int8 matrix{'' if columns is None else f' of {columns} columns'}")
    row, column = t.stride()
    if t.shape[0] <= 1:
        row = t.shape[1]
    if (column != 1 and t.shape[1] > 1) or row < t.shape[1]:
        raise ValueError(f"{what}: the columns of a row must lie side by side, and rows must not overlap")
    if row > 0xfffffe:
        raise ValueError(f"{what}: there are {row} bytes from row to row, more than 0xfffffe")
    return row


def _rows_8bit(n, dim, dev):
    """Room for rows in 8 bits, each of which begins at a multiple of 16 bytes (the product reads those fastest), and their scales."""
    wide = (dim + 15) // 16 * 16
    q = torch.empty((n, wide), dtype=torch.int8, device=dev)
    return q if wide == dim else q[:, :dim], wide, torch.empty(n, dtype=torch.float32, device=dev)


def add_norm(x, weight, residual=None, eps: float = 1e-6, out=None, summed=None, stream=None):
    """(norm, sum, reciprocal roots float32 [n]): the sum of x and the residual [n, dim] in their type, and its root-mean-square
    norm ``sum * rstd * weight`` with ``rstd = 1 / sqrt(mean(sum ** 2) + eps)``.  Without a residual the sum is x itself.  ``weight``:
    float32 or x's type.  ``out`` and ``summed`` (which may be ``residual`` itself: the residual stream in place) cannot be given where
    a gradient is wanted; the sum and the norm are part of torch's backward pass."""
    if stream is not None:
        return _on(stream, add_norm, x, weight, residual, eps, out, summed)
    lib = _lib or _load()
    if _wants(x, weight, residual):
        if out is not None or summed is not None:
            raise ValueError("out and summed cannot be recorded by automatic differentiation: give detached tensors, or call under torch.no_grad()")
        y, total, rstd = _Norm.apply(x, weight, residual, eps)
        return y, x if residual is None else total, rstd
    stride, dev = _matrix(x, "x"), x.device
    n, dim = x.shape
    weight_ptr, weight_type = _weight(weight, dev, dim, x.dtype)
    if out is not None:
        out_stride = _matrix(out, "out", dev, (n, dim), x.dtype)
    residual_ptr, residual_stride, total, summed_ptr, summed_stride = _sum(x, residual, summed)
    if out is None:
        out, out_stride = x.new_empty((n, dim)), dim
    else:
        _written((out,))
    rstd = torch.empty(n, dtype=torch.float32, device=dev)
    _enqueue(lib.bpe_add_norm, dev, x.data_ptr(), _TYPES[x.dtype], n, dim, stride, residual_ptr, residual_stride, weight_ptr,
             weight_type, eps, summed_ptr, summed_stride, rstd.data_ptr(), out.data_ptr(), out_stride)
    return out, total, rstd


def add_norm_8bit(x, weight, residual=None, eps: float = 1e-6, summed=None, stream=None):
    """(norm int8 [n, dim], scales float32 [n], sum): ``add_norm`` with each row of its result in 8 bits: ``q * scales[:, None]``
    stands for it, the largest magnitude of a row is 127.  Rows of q begin at multiples of 16 bytes."""
    if stream is not None:
        return _on(stream, add_norm_8bit, x, weight, residual, eps, summed)
    lib = _lib or _load()
    _no_gradient("add_norm_8bit", x, weight, residual)
    stride, dev = _matrix(x, "x"), x.device
    n, dim = x.shape
    weight_ptr, weight_type = _weight(weight, dev, dim, x.dtype)
    residual_ptr, residual_stride, total, summed_ptr, summed_stride = _sum(x, residual, summed)
    q, q_stride, scales = _rows_8bit(n, dim, dev)
    _enqueue(lib.bpe_add_norm_8bit, dev, x.data_ptr(), _TYPES[x.dtype], n, dim, stride, residual_ptr, residual_stride, weight_ptr,
             weight_type, eps, summed_ptr, summed_stride, q.data_ptr(), q_stride, scales.data_ptr())
    return q, scales, total


def add_norm_grad(grad, summed, weight, rstd, grad_summed=None, out=None, out_weight=None, dtype=None, accumulate: bool = False,
                  workspace=None, stream=None, *, weights: bool = True):
    """(gradient of x, which is the residual's as well, gradient of the weights) from that of the norm and that of the sum, if it was
    used besides, with the sum and ``rstd`` that ``add_norm`` returned.  The weights' gradient has ``out_weight``'s type or ``dtype``:
    float32 or weight's (the default); with ``accumulate`` it is added to what ``out_weight`` holds; without ``weights`` it is not
    computed (None).  ``out`` may be ``grad`` or ``grad_summed`` itself."""
    if stream is not None:
        return _on(stream, lambda *args: add_norm_grad(*args, weights=weights), grad, summed, weight, rstd, grad_summed, out, out_weight, dtype,
                   accumulate, workspace)
    lib = _lib or _load()
    _no_tangent(grad, summed, weight, rstd, grad_summed)
    stride, dev = _matrix(grad, "grad"), grad.device
    n, dim = grad.shape
    summed_stride = _matrix(summed, "summed", dev, (n, dim), grad.dtype)
    weight_ptr, weight_type = _weight(weight, dev, dim, grad.dtype)
    rstd_ptr = _vector(rstd, "rstd", dev, torch.float32, n)
    more_stride = 0 if grad_summed is None else _matrix(grad_summed, "grad_summed", dev, (n, dim), grad.dtype)
    out_stride = dim if out is None else _matrix(out, "out", dev, (n, dim), grad.dtype)
    if not weights:
        if accumulate or any(t is not None for t in (out_weight, dtype, workspace)):
            raise ValueError("out_weight, dtype, accumulate and workspace are for the weights' gradient")
        kind = torch.float32
    else:
        if out_weight is None:
            if accumulate:
                raise ValueError("accumulate needs out_weight")
            kind = dtype or weight.dtype
        else:
            kind = out_weight.dtype
            if dtype is not None and kind != dtype:
                raise ValueError(f"out_weight is {kind}, not {dtype}")
            _vector(out_weight, "out_weight", dev, kind, dim)
        if kind not in (torch.float32, weight.dtype):
            raise ValueError(f"the weights' gradient must be float32 or {weight.dtype}")
        workspace = _workspace(workspace, lib.bpe_add_norm_grad_workspace_bytes(n, dim), dev, "add_norm_grad")
    if out is None:
        out = grad.new_empty((n, dim))
    else:
        _written((out,))
    if out_weight is not None:
        _written((out_weight,))
    elif weights:
        out_weight = torch.empty(dim, dtype=kind, device=dev)
    _enqueue(lib.bpe_add_norm_grad, dev, grad.data_ptr(), _TYPES[grad.dtype], n, dim, stride, summed.data_ptr(), summed_stride, weight_ptr,
             weight_type, rstd_ptr, _pointer(grad_summed), more_stride, out.data_ptr(), out_stride, _pointer(out_weight), _TYPES[kind],
             1 if accumulate else 0, _pointer(workspace), 0 if workspace is None else workspace.numel())
    return out, out_weight


def quantize_rows(x, stream=None):
    """(int8 [n, dim], scales float32 [n]) of a matrix's rows: ``q * scales[:, None]`` stands for x, the largest magnitude of a row is
    127.  For hidden states ahead of ``project_8bit`` and, once, for its weights.  Rows of q begin at multiples of 16 bytes."""
    if stream is not None:
        return _on(stream, quantize_rows, x)
    lib = _lib or _load()
    _no_gradient("quantize_rows", x)
    stride, dev = _matrix(x, "x"), x.device
    n, dim = x.shape
    q, q_stride, scales = _rows_8bit(n, dim, dev)
    _enqueue(lib.bpe_quantize_rows, dev, x.data_ptr(), _TYPES[x.dtype], n, dim, stride, q.data_ptr(), q_stride, scales.data_ptr())
    return q, scales


def project_8bit(q, scales, weight, weight_scales, dtype=None, out=None, stream=None):
    """Logits [n, vocab] from hidden states int8 [n, dim] and weights int8 [vocab, dim] with a scale float32 for each row of both:
    ``(q @ weight.T) * scales[:, None] * weight_scales``, the sums exact.  Their type is ``out``'s or ``dtype`` (default: bfloat16)."""
    if stream is not None:
        return _on(stream, project_8bit, q, scales, weight, weight_scales, dtype, out)
    lib = _lib or _load()
    _no_gradient("project_8bit", scales, weight_scales)
    stride, dev = _bytes(q, "q"), q.device
    n, dim = q.shape
    weight_stride = _bytes(weight, "weight", dev, dim)
    vocab = weight.shape[0]
    scales_ptr = _vector(scales, "scales", dev, torch.float32, n)
    weight_scales_ptr = _vector(weight_scales, "weight_scales", dev, torch.float32, vocab)
    if out is None:
        dtype = dtype or torch.bfloat16
        if dtype not in _TYPES:
            raise ValueError("logits must be float32, bfloat16 or float16")
        if vocab < 1 or dim > 131071:
            raise ValueError("project_8bit: sizes out of range")
        out, out_stride = torch.empty((n, vocab), dtype=dtype, device=dev), vocab
    else:
        out_stride = _matrix(out, "out", dev, (n, vocab), dtype)
        _written((out,))
    _enqueue(lib.bpe_project_8bit, dev, q.data_ptr(), n, dim, stride, scales_ptr, weight.data_ptr(), vocab, weight_stride,
             weight_scales_ptr, out.data_ptr(), _TYPES[out.dtype], out_stride)
    return out


def _history(ids, begin, end, n, dev):
    """Pointer and number of ids, pointers of the rows' bounds."""
    if ids is None and begin is None and end is None:
        return None, 0, None, None
    if ids is None or begin is None or end is None:
        raise ValueError("a history has ids, begin and end")
    return (_vector(ids, "ids", dev, torch.int32, None), ids.numel(), _vector(begin, "begin", dev, torch.int64, n),
            _vector(end, "end", dev, torch.int64, n))


def _penalties(penalties, n, dev):
    """(pointer of the rows' own, repetition, presence and frequency of all)"""
    if penalties is None:
        return None, 1.0, 0.0, 0.0
    if isinstance(penalties, torch.Tensor):
        if penalties.device != dev or penalties.dtype != torch.float32 or penalties.shape != (n, 3) or not penalties.is_contiguous():
            raise ValueError(f"penalties must be three numbers, or a contiguous float32 matrix {(n, 3)} on {dev}")
        return penalties.data_ptr(), 1.0, 0.0, 0.0
    repetition, presence, frequency = penalties
    return None, repetition, presence, frequency


def _mask(mask, state, n, vocab, dev):
    """Pointer, number and stride of the masks, pointer of the rows' choice."""
    if mask is None:
        if state is not None:
            raise ValueError("state needs a mask")
        return None, 0, 0, None
    words = (vocab + 31) // 32
    if mask.device != dev or mask.dtype != torch.int32 or mask.dim() != 2 or mask.shape[1] != words or mask.shape[0] < 1:
        raise ValueError(f"mask must be an int32 matrix of {words} words a row on {dev}")
    states, (stride, column) = mask.shape[0], mask.stride()
    if states == 1:
        stride = max(stride, words)
    if (column != 1 and words > 1) or stride < words:
        raise ValueError("mask: the words of a row must lie side by side, and rows must not overlap")
    if state is None and states not in (1, n):
        raise ValueError(f"without a state there must be one mask, or one for each of {n} rows")
    return mask.data_ptr(), states, stride, None if state is None else _vector(state, "state", dev, torch.int32, n)


def _target(source, out):
    """(out, its stride): new, or given, which may be the source itself."""
    if out is None:
        out = torch.empty_like(source, memory_format=torch.contiguous_format)
        return out, out.shape[1]
    stride = _matrix(out, "out", source.device, tuple(source.shape), source.dtype)
    _written((out,))
    return out, stride


def adjust_logits(logits, ids=None, begin=None, end=None, penalties=None, bias=None, mask=None, state=None, out=None, stream=None):
    """Logits [n, vocab] as a token is chosen from; the formulas are in include/bpe_head.h.

    ``ids`` (int32), ``begin``, ``end`` (int64 [n]): row t's history is ``ids[begin[t]:end[t]]``: ``offsets[:-1], offsets[1:]`` of a
    packed batch, or any other stretches; ids outside the vocabulary are padding.  ``penalties``: repetition (a factor), presence
    and frequency of tokens in the history, three numbers or float32 [n, 3].  ``bias``: (ids int32, values float32, begin, end int64 [n]):
    what is added to some tokens' logits, a list for each row; of a token that a list names twice the later value counts.
    ``mask``: int32 [states, ceil(vocab / 32)], where a token's bit is 0 its logit becomes -inf; ``state`` (int32 [n]) is each row's mask
    (outside [0, states): none), and may be left out with one mask for all rows or one for each.  ``out`` may be ``logits`` itself: only
    what changes is written then.  Part of torch's backward pass where logits want a gradient (``out`` cannot be given then)."""
    if bias is not None:
        bias = tuple(bias)
        if len(bias) != 4:
            raise ValueError("bias must be ids, values, begin and end")
    if stream is not None:
        return _on_all(stream, adjust_logits, logits, ids, begin, end, penalties, bias, mask, state, out)
    lib = _lib or _load()
    _no_gradient("what logits are adjusted by", penalties if isinstance(penalties, torch.Tensor) else None,
                 None if bias is None else bias[1])
    if _wants(logits):
        if out is not None:
            raise ValueError("out cannot be recorded by automatic differentiation: give logits.detach(), or call under torch.no_grad()")
        return _Adjusted.apply(logits, ids, begin, end, penalties, bias, mask, state)
    stride, dev = _matrix(logits, "logits"), logits.device
    n, vocab = logits.shape
    history = _history(ids, begin, end, n, dev)
    rows, repetition, presence, frequency = _penalties(penalties, n, dev)
    if bias is None:
        biases = None, None, 0, None, None
    else:
        bias_ids, values, bias_begin, bias_end = bias
        count = bias_ids.numel()
        biases = (_vector(bias_ids, "bias ids", dev, torch.int32, None), _vector(values, "bias values", dev, torch.float32, count), count,
                  _vector(bias_begin, "bias begin", dev, torch.int64, n), _vector(bias_end, "bias end", dev, torch.int64, n))
    masks = _mask(mask, state, n, vocab, dev)
    out, out_stride = _target(logits, out)
    _enqueue(lib.bpe_adjust_logits, dev, logits.data_ptr(), _TYPES[logits.dtype], n, vocab, stride, *history, rows, repetition, presence,
             frequency, *biases, *masks, out.data_ptr(), out_stride)
    return out


def adjust_logits_grad(grad, logits, ids=None, begin=None, end=None, penalties=None, mask=None, state=None, out=None, stream=None):
    """The gradient with respect to the logits [n, vocab] from that of what ``adjust_logits`` returned for them and these histories,
    penalties and masks.  ``logits`` are those from before.  ``out`` may be ``grad`` itself."""
    if stream is not None:
        return _on_all(stream, adjust_logits_grad, grad, logits, ids, begin, end, penalties, mask, state, out)
    lib = _lib or _load()
    _no_tangent(grad, logits, penalties if isinstance(penalties, torch.Tensor) else None)
    grad_stride, dev = _matrix(grad, "grad"), grad.device
    n, vocab = grad.shape
    stride = _matrix(logits, "logits", dev, (n, vocab), grad.dtype)
    history = _history(ids, begin, end, n, dev)
    rows, repetition, _, _ = _penalties(penalties, n, dev)
    masks = _mask(mask, state, n, vocab, dev)
    out, out_stride = _target(grad, out)
    _enqueue(lib.bpe_adjust_logits_grad, dev, grad.data_ptr(), _TYPES[grad.dtype], n, vocab, grad_stride, logits.data_ptr(), stride,
             *history, rows, repetition, *masks, out.data_ptr(), out_stride)
    return out


def _on_all(stream, function, *args):
    """_on, with the tensors of a list of biases among those that are kept for the stream."""
    result = _on(stream, function, *args)
    if stream != torch.cuda.current_stream(stream.device):
        for group in args:
            for t in group if isinstance(group, tuple) else ():
                if isinstance(t, torch.Tensor):
                    t.record_stream(stream)
    return result
