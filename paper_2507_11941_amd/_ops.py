"""ctypes binding of include/bpe_ops.h, the operators on token batches: argument marshalling only.

Every function enqueues on ``stream`` (default: torch's current stream of the tensors' device) and synchronises nothing.
Outputs and workspaces that are not given are allocated, on that stream.  Matrices may have any stride between rows, but not
between columns; vectors are contiguous.  What the kernels cannot take is refused (ValueError), never copied into shape.

``embed_tokens`` is recorded by torch's automatic differentiation where its weight wants a gradient (not in forward mode, which it
refuses).  The functions on logits are not: their gradient is an output, which ``logits.backward(grad)`` hands on, and
log-probabilities and losses carry none."""
from __future__ import annotations

import ctypes

from ._binding import _check, load_library

_TYPES = {}                                      # torch dtype -> the library's number of it
_lib = torch = _Lookup = _written = _forward = None      # (the package can be imported without torch)


def _load():
    global _lib, torch, _Lookup, _written, _forward
    if _lib is None:
        import torch as module

        torch = module
        lib = load_library()
        vp, i, i32, i64, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        for name, args in {
                "embed_tokens": [vp, i, i64, i64, i64, vp, i64, vp, f, vp, i64, vp],
                "embed_tokens_grad": [vp, i, i64, vp, i64, vp, i64, i64, f, i, vp, i, i64, vp, sz, vp],
                "next_tokens": [vp, i64, vp, i32, vp, vp, vp],
                "token_logprobs": [vp, i, i64, i64, i64, vp, vp, vp, vp, sz, vp],
                "token_logprobs_grad": [vp, i, i64, i64, i64, vp, vp, vp, vp, i64, vp],
                "token_logprobs_and_grad": [vp, i, i64, i64, i64, vp, vp, vp, vp, vp, i64, vp],
                "preference_loss": [vp, i, i64, i64, i64, vp, vp, i32, vp, f, f, f, vp, vp, vp, vp, i64, vp, sz, vp],
                "policy_loss": [vp, i, i64, i64, i64, vp, vp, i32, vp, vp, i, vp, f, f, f, i, f, vp, vp, vp, i64, vp, sz, vp],
        }.items():
            function = getattr(lib, "bpe_" + name)
            function.argtypes, function.restype = args, i
        lib.bpe_embed_tokens_grad_workspace_bytes.argtypes = [i64, i64, i64]
        lib.bpe_embed_tokens_grad_workspace_bytes.restype = sz
        lib.bpe_token_logprobs_workspace_bytes.argtypes = [i64, i64]
        lib.bpe_token_logprobs_workspace_bytes.restype = sz
        lib.bpe_loss_workspace_bytes.argtypes = [i64, i64, i32]
        lib.bpe_loss_workspace_bytes.restype = sz
        _Lookup, _forward = _lookup(), torch.autograd.forward_ad
        _written = torch._C._increment_version   # (as in _binding.py; a call's own tensors only, given as a tuple)
        _TYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
        _lib = lib
    return _lib


def _lookup():
    """embed_tokens as torch's automatic differentiation knows it."""
    class Lookup(torch.autograd.Function):
        @staticmethod
        def forward(ctx, weight, ids, scale, count):
            ctx.save_for_backward(ids, count)
            ctx.vocab, ctx.scale = weight.shape[0], scale
            return embed_tokens(weight, ids, scale, count)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad):
            ids, count = ctx.saved_tensors
            return embed_tokens_grad(grad.contiguous(), ids, ctx.vocab, ctx.scale, count), None, None, None

    return Lookup


def _no_tangent(*tensors):
    """Refuses tensors with a forward-mode derivative, which would be lost."""
    if _forward._current_level >= 0 and any(t is not None and _forward.unpack_dual(t).tangent is not None for t in tensors):
        raise ValueError("there is no forward-mode derivative here: give the primal tensors")


def _matrix(t, what, dev=None, shape=None, dtype=None):
    """The stride between the rows of a matrix that the kernels can take."""
    if not t.is_cuda or (dev is not None and t.device != dev):
        raise ValueError(f"{what} must be on {'the GPU' if dev is None else dev}")
    if t.dim() != 2 or t.dtype not in _TYPES or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{what} must be a matrix of {dtype or 'float32, bfloat16 or float16'}")
    rows, columns = t.shape
    if columns < 1 or (shape is not None and (rows, columns) != shape):
        raise ValueError(f"{what} is {tuple(t.shape)}, not {shape or 'at least one column wide'}")
    row, column = t.stride()
    if rows <= 1:
        row = max(row, columns)
    if (column != 1 and columns > 1) or row < columns:
        raise ValueError(f"{what}: the columns of a row must lie side by side, and rows must not overlap")
    return row


def _vector(t, what, dev, dtype, count):
    if t.device != dev or t.dtype != dtype or t.dim() != 1 or not t.is_contiguous() or (count is not None and t.numel() != count):
        raise ValueError(f"{what} must be a contiguous {dtype} vector{'' if count is None else f' of {count}'} on {dev}")
    return t.data_ptr()


def _enqueue(function, dev, *args):
    """function(*args, handle of the device's current stream).  (The handle without a Stream object, and the device without the
    check that torch has begun: 2 us of a small call's 11.)"""
    if dev.index != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            return _enqueue(function, dev, *args)
    code = function(*args, torch._C._cuda_getCurrentRawStream(dev.index))
    if code != 0:
        _check(code, function.__name__)


def _on(stream, function, *args):
    """function(*args) on `stream`.  What it allocates belongs to that stream: a block of the caller's could still be in use by
    work that the caller's stream has queued.  No tensor's memory is given away before both streams are done with it."""
    _load()
    if args[0].device != stream.device:
        raise ValueError(f"stream is of {stream.device}, not {args[0].device}")
    caller = torch.cuda.current_stream(stream.device)
    if stream == caller:
        return function(*args)
    with torch.cuda.stream(stream):
        results = function(*args)
    for t in args:
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
    for t in results if isinstance(results, tuple) else (results,):
        if t is not None:
            t.record_stream(caller)
    return results


def _strings(offsets, dev):
    """(pointer, number of strings) of a batch's offsets."""
    pointer, batch = _vector(offsets, "offsets", dev, torch.int64, None), offsets.numel() - 1
    if not 0 <= batch < 1 << 31:
        raise ValueError("offsets must have a beginning and an end for each string")
    return pointer, batch


def _pointer(t):
    return None if t is None else t.data_ptr()


def _workspace(given, need, dev, what):
    if need == 0:
        raise ValueError(f"{what}: sizes out of range")
    if given is None:
        return torch.empty(need, dtype=torch.uint8, device=dev)
    if given.device != dev or given.dtype != torch.uint8 or not given.is_contiguous() or given.numel() < need:
        raise ValueError(f"workspace must be {need} contiguous bytes (uint8) on {dev}")
    return given


def _count(count, dev):
    if count is not None and (count.device != dev or count.dtype != torch.int64 or count.numel() != 1):
        raise ValueError(f"count must be one int64 on {dev}")
    return _pointer(count)


def embed_tokens(weight, ids, scale: float = 1.0, count=None, out=None, stream=None):
    """``out[t] = scale * weight[ids[t]]``: rows of an embedding [vocab, dim] for int32 ids [n]; zeros for an id outside the
    vocabulary (padding).  ``count``: one int64 on the GPU, from which row on ids and out are left alone (``out_offsets[-1:]``
    of an encoded batch, whose ids need not all be in use).  A weight that wants a gradient gets it from the backward pass, in its
    own type; ``out`` cannot be given then."""
    if stream is not None:
        return _on(stream, embed_tokens, weight, ids, scale, count, out)
    lib = _lib or _load()
    _no_tangent(weight)
    if weight.requires_grad and torch.is_grad_enabled():
        if out is not None:
            raise ValueError("out cannot be recorded by automatic differentiation: give weight.detach(), or call under torch.no_grad()")
        return _Lookup.apply(weight, ids, scale, count)
    stride, dev = _matrix(weight, "weight"), weight.device
    n, dim = ids.numel(), weight.shape[1]
    ids_ptr = _vector(ids, "ids", dev, torch.int32, None)
    if out is None:
        out, out_stride = weight.new_empty((n, dim)), dim
    else:
        out_stride = _matrix(out, "out", dev, (n, dim), weight.dtype)
        _written((out,))
    _enqueue(lib.bpe_embed_tokens, dev, weight.data_ptr(), _TYPES[weight.dtype], weight.shape[0], dim, stride, ids_ptr, n,
             None if count is None else _count(count, dev), scale, out.data_ptr(), out_stride)
    return out


def embed_tokens_grad(grad, ids, vocab: int, scale: float = 1.0, count=None, out=None, dtype=None, accumulate: bool = False,
                      workspace=None, stream=None):
    """The gradient [vocab, dim] of an embedding's weights from that of its output [n, dim]: row v is ``scale`` times the sum
    of grad[t] over the t with ids[t] = v.  Its type is ``out``'s or ``dtype``: float32 or grad's (the default).  With
    ``accumulate`` it is added to what ``out`` holds."""
    if stream is not None:
        return _on(stream, embed_tokens_grad, grad, ids, vocab, scale, count, out, dtype, accumulate, workspace)
    lib = _lib or _load()
    stride, dev = _matrix(grad, "grad"), grad.device
    n, dim = grad.shape
    ids_ptr = _vector(ids, "ids", dev, torch.int32, n)
    given = out
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((vocab, dim), dtype=dtype or grad.dtype, device=dev)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError(f"out is {out.dtype}, not {dtype}")
    if out.dtype not in (torch.float32, grad.dtype):
        raise ValueError(f"the weights' gradient must be float32 or {grad.dtype}")
    out_stride = _matrix(out, "out", dev, (vocab, dim))
    count_ptr = _count(count, dev)
    workspace = _workspace(workspace, lib.bpe_embed_tokens_grad_workspace_bytes(n, vocab, dim), dev, "embed_tokens_grad")
    if given is not None:
        _written((out,))
    _enqueue(lib.bpe_embed_tokens_grad, dev, grad.data_ptr(), _TYPES[grad.dtype], stride, ids_ptr, n, count_ptr, vocab, dim, scale,
             1 if accumulate else 0, out.data_ptr(), _TYPES[out.dtype], out_stride, workspace.data_ptr(), workspace.numel())
    return out


def next_tokens(ids, offsets, first=None, out=None, stream=None):
    """What each position of a packed batch is to predict: the id after it in its string (int64 offsets [B + 1]); -1, not
    scored, at a string's end and where that id is among the string's ``first`` tokens (int32 [B]: prompts)."""
    if stream is not None:
        return _on(stream, next_tokens, ids, offsets, first, out)
    lib = _lib or _load()
    dev, n = ids.device, ids.numel()
    if not ids.is_cuda:
        raise ValueError("ids must be on the GPU")
    ids_ptr = _vector(ids, "ids", dev, torch.int32, None)
    offsets_ptr, batch = _strings(offsets, dev)
    first_ptr = None if first is None else _vector(first, "first", dev, torch.int32, batch)
    if out is None:
        out = torch.empty_like(ids)
        out_ptr = out.data_ptr()
    else:
        out_ptr = _vector(out, "out", dev, torch.int32, n)
        _written((out,))
    _enqueue(lib.bpe_next_tokens, dev, ids_ptr, n, offsets_ptr, batch, first_ptr, out_ptr)
    return out


def _grad_of(logits, out):
    """(the gradient's matrix, the stride between its rows)"""
    if out is None:
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
        return out, out.shape[1]
    stride = _matrix(out, "out", logits.device, tuple(logits.shape), logits.dtype)
    _written((out,))
    return out, stride


def token_logprobs(logits, targets, workspace=None, stream=None):
    """(log-probabilities float32 [n] of the int32 targets [n] under logits [n, vocab], logarithms float32 [n] of the rows'
    sums of exponentials).  Rows whose target is outside the vocabulary are not scored: not read, and 0 in both."""
    if stream is not None:
        return _on(stream, token_logprobs, logits, targets, workspace)
    lib = _lib or _load()
    stride, dev = _matrix(logits, "logits"), logits.device
    n, vocab = logits.shape
    targets_ptr = _vector(targets, "targets", dev, torch.int32, n)
    logprobs = torch.empty(n, dtype=torch.float32, device=dev)
    lse = torch.empty_like(logprobs)
    need = lib.bpe_token_logprobs_workspace_bytes(n, vocab)
    workspace = _workspace(workspace, need, dev, "token_logprobs") if need else None
    _enqueue(lib.bpe_token_logprobs, dev, logits.data_ptr(), _TYPES[logits.dtype], n, vocab, stride, targets_ptr,
             logprobs.data_ptr(), lse.data_ptr(), _pointer(workspace), need)
    return logprobs, lse


def token_logprobs_grad(logits, targets, lse, upstream, out=None, stream=None):
    """The gradient [n, vocab] with respect to the logits of ``(upstream * logprobs).sum()``, from the ``lse`` that
    ``token_logprobs`` returned.  ``out`` may be ``logits`` itself."""
    if stream is not None:
        return _on(stream, token_logprobs_grad, logits, targets, lse, upstream, out)
    lib = _lib or _load()
    stride, dev = _matrix(logits, "logits"), logits.device
    n, vocab = logits.shape
    targets_ptr = _vector(targets, "targets", dev, torch.int32, n)
    lse_ptr, upstream_ptr = _vector(lse, "lse", dev, torch.float32, n), _vector(upstream, "upstream", dev, torch.float32, n)
    out, out_stride = _grad_of(logits, out)
    _enqueue(lib.bpe_token_logprobs_grad, dev, logits.data_ptr(), _TYPES[logits.dtype], n, vocab, stride, targets_ptr, lse_ptr,
             upstream_ptr, out.data_ptr(), out_stride)
    return out


def token_logprobs_and_grad(logits, targets, upstream, out=None, stream=None):
    """(logprobs, lse, gradient of ``(upstream * logprobs).sum()``) in one pass over the logits, for an upstream that is known
    before: of cross entropy it is -1 / (number of scored tokens).  ``out`` may be ``logits`` itself."""
    if stream is not None:
        return _on(stream, token_logprobs_and_grad, logits, targets, upstream, out)
    lib = _lib or _load()
    stride, dev = _matrix(logits, "logits"), logits.device
    n, vocab = logits.shape
    targets_ptr = _vector(targets, "targets", dev, torch.int32, n)
    upstream_ptr = _vector(upstream, "upstream", dev, torch.float32, n)
    logprobs, lse = torch.empty_like(upstream), torch.empty_like(upstream)
    out, out_stride = _grad_of(logits, out)
    _enqueue(lib.bpe_token_logprobs_and_grad, dev, logits.data_ptr(), _TYPES[logits.dtype], n, vocab, stride, targets_ptr,
             upstream_ptr, logprobs.data_ptr(), lse.data_ptr(), out.data_ptr(), out_stride)
    return logprobs, lse, out


def preference_loss(logits, targets, offsets, reference=None, beta: float = 0.1, smoothing: float = 0.0, scale: float = 1.0,
                    out=None, workspace=None, stream=None):
    """Preference loss over pairs of strings, 2k preferred to 2k + 1: (loss, margins float32 [B / 2], logprobs float32 [n],
    ``scale`` times the gradient with respect to the logits).  ``reference``: float32 [n], the reference model's logprobs.
    ``out`` may be ``logits`` itself.  The formulas are in include/bpe_ops.h."""
    if stream is not None:
        return _on(stream, preference_loss, logits, targets, offsets, reference, beta, smoothing, scale, out, workspace)
    lib = _lib or _load()
    stride, dev = _matrix(logits, "logits"), logits.device
    n, vocab = logits.shape
    targets_ptr = _vector(targets, "targets", dev, torch.int32, n)
    offsets_ptr, batch = _strings(offsets, dev)
    if batch % 2:
        raise ValueError("preference_loss takes an even number of strings: pairs")
    reference_ptr = None if reference is None else _vector(reference, "reference", dev, torch.float32, n)
    loss, margins = torch.empty((), dtype=torch.float32, device=dev), torch.empty(batch // 2, dtype=torch.float32, device=dev)
    logprobs = torch.empty(n, dtype=torch.float32, device=dev)
    out, out_stride = _grad_of(logits, out)
    workspace = _workspace(workspace, lib.bpe_loss_workspace_bytes(n, vocab, batch), dev, "logits")
    _enqueue(lib.bpe_preference_loss, dev, logits.data_ptr(), _TYPES[logits.dtype], n, vocab, stride, targets_ptr, offsets_ptr,
             batch, reference_ptr, beta, smoothing, scale, loss.data_ptr(), margins.data_ptr(), logprobs.data_ptr(), out.data_ptr(),
             out_stride, workspace.data_ptr(), workspace.numel())
    return loss, margins, logprobs, out


def policy_loss(logits, targets, offsets, old, advantages, reference=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_weight: float = 0.0, per: str = "token", scale: float = 1.0, out=None, workspace=None, stream=None):
    """Clipped policy loss with a KL term: (loss, logprobs float32 [n], ``scale`` times the gradient with respect to the
    logits).  ``old``, ``reference``: float32 [n], the old policy's and the reference model's logprobs.  ``advantages``: float32
    [n], or [B], one for all of a string (where n = B, it is by string if ``per`` is "string").  ``per``: "token", all scored
    tokens weigh the same, or "string", all strings.  ``out`` may be ``logits`` itself.  The formulas are in
    include/bpe_ops.h."""
    if stream is not None:
        return _on(stream, policy_loss, logits, targets, offsets, old, advantages, reference, clip_low, clip_high, kl_weight, per,
                   scale, out, workspace)
    lib = _lib or _load()
    stride, dev = _matrix(logits, "logits"), logits.device
    n, vocab = logits.shape
    targets_ptr = _vector(targets, "targets", dev, torch.int32, n)
    offsets_ptr, batch = _strings(offsets, dev)
    if per not in ("token", "string"):
        raise ValueError('per must be "token" or "string"')
    by_string = per == "string"
    old_ptr = _vector(old, "old", dev, torch.float32, n)
    whole = advantages.numel() == batch and (batch != n or by_string)
    advantages_ptr = _vector(advantages, "advantages", dev, torch.float32, batch if whole else n)
    reference_ptr = None if reference is None else _vector(reference, "reference", dev, torch.float32, n)
    loss, logprobs = torch.empty((), dtype=torch.float32, device=dev), torch.empty_like(old)
    out, out_stride = _grad_of(logits, out)
    workspace = _workspace(workspace, lib.bpe_loss_workspace_bytes(n, vocab, batch), dev, "logits")
    _enqueue(lib.bpe_policy_loss, dev, logits.data_ptr(), _TYPES[logits.dtype], n, vocab, stride, targets_ptr, offsets_ptr, batch,
             old_ptr, advantages_ptr, 1 if whole else 0, reference_ptr, clip_low, clip_high, kl_weight, 1 if by_string else 0,
             scale, loss.data_ptr(), logprobs.data_ptr(), out.data_ptr(), out_stride, workspace.data_ptr(), workspace.numel())
    return loss, logprobs, out
