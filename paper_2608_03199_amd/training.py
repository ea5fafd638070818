"""Operators of libsieve around a text encoder's blocks: the table's lookup, and the cross entropy
of hidden states against a table, each with its gradient; and the orthogonalised update of the
matrices between them (``include/sieve.h``).

As in ``encoder.py``, the ``*_forward`` / ``*_backward`` functions marshal the arguments of the
library's calls, the others join them for torch's autograd, all calls are asynchronous on the
given or current stream, and there is no CPU fallback.

Into a graph, capture the ``*_forward`` / ``*_backward`` functions.  A backward pass of torch's own
is captured only where no result of an eager pass over the same parameters is alive: what
accumulates their gradients would still belong to the eager pass's stream, which ends the
process.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch
from torch.autograd.function import once_differentiable

from . import _check
from .encoder import _CODES, _code, _here, _need, _on, _ptr, _raw_stream, _rows, _workspace
from .encoder import _library as _encoder_library

__all__ = ["embed", "embed_backward", "embed_forward", "linear_cross_entropy",
           "linear_cross_entropy_backward", "linear_cross_entropy_forward", "orthogonalize"]

_ready = None


def _library():
    global _ready
    if _ready is not None:
        return _ready
    lib = _encoder_library()
    P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.sieve_embed_forward.restype = ctypes.c_int
    lib.sieve_embed_forward.argtypes = [P, i32, i64, P, i64, i32, i64, i32, f32, P, i32, P]
    lib.sieve_embed_workspace.restype = i64
    lib.sieve_embed_workspace.argtypes = [i64, i64, i32]
    lib.sieve_embed_backward.restype = ctypes.c_int
    lib.sieve_embed_backward.argtypes = [P, i64, i32, P, i32, i64, i64, i32, f32, i32, P, i32, P,
                                         i64, P]
    lib.sieve_loss_workspace.restype = i64
    lib.sieve_loss_workspace.argtypes = [i64, i64, i32, i32, i32]
    lib.sieve_loss_forward.restype = ctypes.c_int
    lib.sieve_loss_forward.argtypes = [P, i64, P, i64, i32, i64, i64, i32, P, i32, f32, P, P, P,
                                       i64, P]
    lib.sieve_loss_backward.restype = ctypes.c_int
    lib.sieve_loss_backward.argtypes = [P, P, i64, P, i64, i32, i64, i64, i32, P, i32, P, f32, P,
                                        P, P, i64, P]
    lib.sieve_orthogonalize_workspace.restype = i64
    lib.sieve_orthogonalize_workspace.argtypes = [i64, i64, i64]
    lib.sieve_orthogonalize.restype = ctypes.c_int
    lib.sieve_orthogonalize.argtypes = [P, i64, i64, i32, i64, i64, i64, i32, P, f32, P, P, i64, P]
    _ready = lib
    return lib


# ---- embedding ----------------------------------------------------------------------------

_WHOLE = {torch.int32: 4, torch.int64: 8}


def _numbers(t: torch.Tensor, name: str, device):
    """Whole numbers of 4 or 8 bytes on the device, one after another, and their size."""
    if t.dtype not in _WHOLE:
        raise TypeError(f"{name} must be int32 or int64, not {t.dtype}")
    _need(t.device == device, f"{name} must be on {device}")
    return t.contiguous(), _WHOLE[t.dtype]


def embed_forward(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0,
                  dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """``scale * table[ids]`` as ``dtype`` (the table's, unless it is float32 and another is
    asked for): [*ids.shape, n].  A number that is not in the table gives a row of zeros."""
    _need(table.is_cuda, "table must be a GPU tensor")
    if _here(table.device, stream):
        return _embed_forward(ids, table, scale, dtype)
    with _on(table.device, stream):
        return _embed_forward(ids, table, scale, dtype)


def _embed_forward(ids, table, scale, dtype):
    _need(table.dim() == 2 and table.shape[0] >= 1 and table.shape[1] >= 1,
          "table must be [vocab, n]")
    dtype = table.dtype if dtype is None else dtype
    tcode = _code(table, "table")
    _check_pair(dtype, table.dtype)
    lib = _library()
    ids, size = _numbers(ids, "ids", table.device)
    vocab, n = table.shape
    tr, stride = _rows(table, n)
    out = table.new_empty(ids.shape + (n,), dtype=dtype)
    if ids.numel():
        _check(lib, lib.sieve_embed_forward(ids.data_ptr(), size, ids.numel(), tr.data_ptr(),
                                            stride, tcode, vocab, n, scale, out.data_ptr(),
                                            _CODES[dtype], _raw_stream(table.device)))
    return out


def _check_pair(dtype, tdtype):
    if dtype not in _CODES:
        raise TypeError(f"unsupported dtype {dtype} (float32, float16 or bfloat16)")
    if tdtype not in (dtype, torch.float32):
        raise TypeError("the table must be of the rows' dtype or float32")


def embed_backward(dy: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0,
                   dtype: Optional[torch.dtype] = None, into: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The gradient [vocab, n] of ``embed_forward``'s table, of ``dtype`` (dy's, or float32).
    ``into``: a gradient of the table that this one is added to, and returned (of a tied output
    layer, say); rows that no number names are then left as they are."""
    _need(dy.is_cuda, "dy must be a GPU tensor")
    if _here(dy.device, stream):
        return _embed_backward(dy, ids, vocab, scale, dtype, into)
    with _on(dy.device, stream):
        return _embed_backward(dy, ids, vocab, scale, dtype, into)


def _embed_backward(dy, ids, vocab, scale, dtype, into):
    shape = dy.shape
    _need(len(shape) >= 1 and shape[-1] >= 1, "dy must have a last axis of at least one value")
    n, vocab = shape[-1], int(vocab)
    _need(ids.shape == shape[:-1], f"ids must be {list(shape[:-1])}")
    _need(vocab >= 1, "vocab must be at least 1")
    dtype = (dy.dtype if into is None else into.dtype) if dtype is None else dtype
    code = _code(dy, "dy")
    _check_pair(dy.dtype, dtype)
    if into is not None:
        _need(into.shape == (vocab, n) and into.dtype is dtype and into.device == dy.device and
              into.is_contiguous(), f"into must be a contiguous [{vocab}, {n}] of {dtype} on "
                                    f"dy's device")
    lib = _library()
    ids, size = _numbers(ids, "ids", dy.device)
    dr, stride = _rows(dy, n)
    count = ids.numel()
    need = lib.sieve_embed_workspace(count, vocab, n)
    space = _workspace(lib, need, dy.device)
    out = dy.new_empty((vocab, n), dtype=dtype) if into is None else into
    _check(lib, lib.sieve_embed_backward(_ptr(dr), stride, code, _ptr(ids), size, count, vocab, n,
                                         scale, int(into is not None), out.data_ptr(),
                                         _CODES[dtype], _ptr(space), need,
                                         _raw_stream(dy.device)))
    return out


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale, dtype):
        ctx.save_for_backward(ids)
        ctx.vocab, ctx.scale, ctx.dtype = table.shape[0], scale, table.dtype
        return embed_forward(ids, table, scale, dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        ids, = ctx.saved_tensors
        return None, embed_backward(dy, ids, ctx.vocab, ctx.scale, ctx.dtype), None, None


def embed(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0,
          dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """Differentiable ``embed_forward``."""
    return _Embed.apply(ids, table, scale, dtype)


# ---- cross entropy ------------------------------------------------------------------------


def linear_cross_entropy_forward(h: torch.Tensor, table: torch.Tensor, targets: torch.Tensor,
                                 scale: float = 1.0, stream=None):
    """Softmax cross entropy of the logits ``scale * h @ table.T`` without keeping them: ``h``
    [..., n] and ``table`` [vocab, n] of one dtype, ``targets`` [...] whole numbers.  Returns
    ``(loss, lse)``, fp32 of targets' shape: each row's loss, and the logarithm of its sum.  A row
    whose target is not in the table (-100, say) is left out: its loss is 0."""
    _need(h.is_cuda, "h must be a GPU tensor")
    if _here(h.device, stream):
        return _loss_forward(h, table, targets, scale)
    with _on(h.device, stream):
        return _loss_forward(h, table, targets, scale)


def _loss_inputs(h, table, targets):
    shape = h.shape
    _need(len(shape) >= 1 and shape[-1] >= 1, "h must have a last axis of at least one value")
    n = shape[-1]
    code = _code(h, "h")
    if table.dtype != h.dtype:
        raise TypeError(f"table must be {h.dtype}, not {table.dtype}")
    _need(table.dim() == 2 and table.shape[0] >= 1 and table.shape[1] == n and
          table.device == h.device, f"table must be [vocab, {n}] on h's device")
    _need(targets.shape == shape[:-1], f"targets must be {list(shape[:-1])}")
    targets, size = _numbers(targets, "targets", h.device)
    hr, h_stride = _rows(h, n)
    tr, t_stride = _rows(table, n)
    return (hr, h_stride, tr, t_stride, code, targets.numel(), table.shape[0], n, targets, size)


def _loss_forward(h, table, targets, scale):
    lib = _library()
    hr, h_stride, tr, t_stride, code, rows, vocab, n, tg, size = _loss_inputs(h, table, targets)
    # not of one allocation: a caller may change the losses where they are, and lse is kept
    loss, lse = (h.new_empty(targets.shape, dtype=torch.float32) for _ in range(2))
    need = lib.sieve_loss_workspace(rows, vocab, n, code, 0)
    space = _workspace(lib, need, h.device)
    if rows:
        _check(lib, lib.sieve_loss_forward(hr.data_ptr(), h_stride, tr.data_ptr(), t_stride, code,
                                           rows, vocab, n, tg.data_ptr(), size, scale,
                                           loss.data_ptr(), lse.data_ptr(), _ptr(space), need,
                                           _raw_stream(h.device)))
    return loss, lse


def linear_cross_entropy_backward(dloss: torch.Tensor, h: torch.Tensor, table: torch.Tensor,
                                  targets: torch.Tensor, lse: torch.Tensor, scale: float = 1.0,
                                  h_grad: bool = True, table_grad: bool = True, stream=None):
    """Gradients of ``linear_cross_entropy_forward`` from the gradient of each row's loss (fp32),
    the forward pass's inputs and its ``lse``; the logits are computed again.  Returns ``(dh,
    dtable)``, None where not asked for."""
    _need(h.is_cuda, "h must be a GPU tensor")
    args = (dloss, h, table, targets, lse, scale, h_grad, table_grad)
    if _here(h.device, stream):
        return _loss_backward(*args)
    with _on(h.device, stream):
        return _loss_backward(*args)


def _loss_backward(dloss, h, table, targets, lse, scale, h_grad, table_grad):
    lib = _library()
    hr, h_stride, tr, t_stride, code, rows, vocab, n, tg, size = _loss_inputs(h, table, targets)
    for name, t in (("dloss", dloss), ("lse", lse)):
        _need(t.shape == targets.shape and t.dtype is torch.float32 and t.device == h.device,
              f"{name} must be {list(targets.shape)} float32 on h's device")
    dloss, lse = dloss.contiguous(), lse.contiguous()
    dh = h.new_empty(h.shape) if h_grad else None
    dtable = h.new_empty((vocab, n)) if table_grad else None
    need = lib.sieve_loss_workspace(rows, vocab, n, code, 1)
    space = _workspace(lib, need, h.device)
    _check(lib, lib.sieve_loss_backward(
        _ptr(dloss), _ptr(hr), h_stride, tr.data_ptr(), t_stride, code, rows, vocab, n, _ptr(tg),
        size, _ptr(lse), scale, _ptr(dh), _ptr(dtable), _ptr(space), need, _raw_stream(h.device)))
    return dh, dtable


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, table, targets, scale):
        loss, lse = linear_cross_entropy_forward(h, table, targets, scale)
        ctx.save_for_backward(h, table, targets, lse)
        ctx.scale = scale
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        h, table, targets, lse = ctx.saved_tensors
        dh, dtable = linear_cross_entropy_backward(
            dloss, h, table, targets, lse, ctx.scale, ctx.needs_input_grad[0],
            ctx.needs_input_grad[1])
        return dh, dtable, None, None


def linear_cross_entropy(h: torch.Tensor, table: torch.Tensor, targets: torch.Tensor,
                         scale: float = 1.0) -> torch.Tensor:
    """Differentiable ``linear_cross_entropy_forward``: each row's loss."""
    return _LinearCrossEntropy.apply(h, table, targets, scale)


# ---- orthogonalised updates ---------------------------------------------------------------


def orthogonalize(g: torch.Tensor, steps: int = 5,
                  coefficients: Sequence[float] = (3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  stream=None) -> torch.Tensor:
    """Each matrix of ``g`` [..., m, n], divided by its norm (+ ``eps``), after ``steps`` times
    ``x = a x + b (x x^T) x + c (x x^T)^2 x``: its singular vectors with singular values near 1.
    Of g's shape and dtype; not differentiable."""
    _need(g.is_cuda, "g must be a GPU tensor")
    if _here(g.device, stream):
        return _orthogonalize(g, steps, coefficients, eps)
    with _on(g.device, stream):
        return _orthogonalize(g, steps, coefficients, eps)


def _orthogonalize(g, steps, coefficients, eps):
    shape = g.shape
    _need(len(shape) >= 2 and shape[-1] >= 1 and shape[-2] >= 1,
          "g must have two last axes of at least one value")
    code = _code(g, "g")
    _need(len(coefficients) == 3, "coefficients must be three numbers")
    lib = _library()
    m, n = shape[-2:]
    x = g.detach().reshape(-1, m, n)
    batch = x.shape[0]
    if not ((x.stride(2) == 1 or n == 1) and (x.stride(1) >= n or m == 1) and x.stride(0) >= 0):
        x = x.contiguous()
    out = g.new_empty(shape, requires_grad=False)
    need = lib.sieve_orthogonalize_workspace(batch, m, n)
    space = _workspace(lib, need, g.device)
    _check(lib, lib.sieve_orthogonalize(
        _ptr(x), x.stride(0), max(x.stride(1), n), code, batch, m, n, int(steps),
        (ctypes.c_float * 3)(*coefficients), eps, _ptr(out), _ptr(space), need,
        _raw_stream(g.device)))
    return out
