"""Text-encoder operators of libsieve: layer norm and packed attention with a learned
relative position bias, forward and backward (``include/sieve.h``).

The ``*_forward`` / ``*_backward`` functions and ``AttentionPlan``'s methods marshal arguments
of single kernels' calls; ``layer_norm`` and ``attention`` join them for torch's autograd.  All
calls are asynchronous on the given or current stream.  Outputs and workspace come from torch's
allocator on that stream; there is no CPU fallback.
"""
from __future__ import annotations

import array
import contextlib
import ctypes
import math
from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import F16, F32, SieveError, _check, load_library

__all__ = ["AttentionPlan", "BF16", "attention", "layer_norm", "layer_norm_backward",
           "layer_norm_forward"]

BF16 = 2
_CODES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}


class _Desc(ctypes.Structure):
    """Mirror of ``sieve_attn_desc``."""
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("num_buckets", ctypes.c_int32),
                ("max_distance", ctypes.c_int32), ("scale", ctypes.c_float),
                ("nseq", ctypes.c_int64), ("q_offsets", ctypes.c_void_p),
                ("k_offsets", ctypes.c_void_p)]


class _Heads(ctypes.Structure):
    """Mirror of ``sieve_heads``."""
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


_ready = None


def _library():
    global _ready
    if _ready is not None:
        return _ready
    lib = load_library()
    P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.sieve_norm_forward.restype = ctypes.c_int
    lib.sieve_norm_forward.argtypes = [P, i64, P, i64, P, P, i32, i32, i64, i32, f32, P, P, P, P, P]
    lib.sieve_norm_backward.restype = ctypes.c_int
    lib.sieve_norm_backward.argtypes = [P, i64, P, i64, P, P, P, P, i32, i32, i64, i32, P, P, P, P,
                                        i64, P]
    lib.sieve_norm_workspace.restype = i64
    lib.sieve_norm_workspace.argtypes = [i64, i32]
    lib.sieve_attn_create.restype = ctypes.c_int
    lib.sieve_attn_create.argtypes = [ctypes.POINTER(_Desc), P, ctypes.POINTER(P)]
    lib.sieve_attn_free.restype = None
    lib.sieve_attn_free.argtypes = [P]
    lib.sieve_attn_workspace.restype = i64
    lib.sieve_attn_workspace.argtypes = [P, i32]
    lib.sieve_attn_forward.restype = ctypes.c_int
    lib.sieve_attn_forward.argtypes = [P, P, P, P, P, P, P, P, P, i64, P]
    lib.sieve_attn_backward.restype = ctypes.c_int
    lib.sieve_attn_backward.argtypes = [P] * 14 + [i64, P]
    _ready = lib
    return lib


@contextlib.contextmanager
def _on(device: torch.device, stream):
    """The device and the stream that the call's allocations and kernels belong to."""
    with torch.cuda.device(device):
        if stream is None:
            yield
        else:
            with torch.cuda.stream(stream):
                yield


def _here(device: torch.device, stream) -> bool:
    """Whether a call is to run on the current device and stream: the short way."""
    return stream is None and device.index == torch.cuda.current_device()


# the current stream's handle without a Stream object around it, where torch has that
_current_handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _raw_stream(device: torch.device) -> int:
    if _current_handle is not None:
        return _current_handle(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _workspace(lib, size: int, device):
    if size < 0:
        _check(lib, int(size))
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _code(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _CODES:
        raise TypeError(f"unsupported dtype {t.dtype} of {name} (float32, float16 or bfloat16)")
    return _CODES[t.dtype]


def _rows(t: torch.Tensor, n: int):
    """``t`` as rows of n values side by side, at least n apart, and how far apart; copied only
    where that is not a view."""
    if t.is_contiguous():
        return t, n
    t = t.reshape(-1, n)
    if t.shape[0] > 1 and t.stride(0) >= n and (n == 1 or t.stride(1) == 1):
        return t, t.stride(0)
    return t.contiguous(), n


# ---- layer norm ---------------------------------------------------------------------------


def layer_norm_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                       eps: float = 1e-5, residual: Optional[torch.Tensor] = None, stream=None):
    """Layer norm over the last axis of ``x`` (+ ``residual``).  Returns ``(y, h, mean, rstd)``:
    ``h`` is the sum that was normed (``x`` itself without a residual), ``mean`` and ``rstd`` are
    fp32, one a row.  ``weight`` and ``bias`` are of x's dtype or float32."""
    _need(x.is_cuda, "x must be a GPU tensor")
    if _here(x.device, stream):
        return _norm_forward(x, weight, bias, eps, residual)
    with _on(x.device, stream):
        return _norm_forward(x, weight, bias, eps, residual)


def _norm_forward(x, weight, bias, eps, residual):
    shape = x.shape
    _need(len(shape) >= 1 and shape[-1] >= 1, "x must have a last axis of at least one value")
    n = shape[-1]
    code = _code(x, "x")
    _check_affine(x, weight, bias, n)
    lib = _library()
    xr, x_stride = _rows(x, n)
    rr, r_stride, h = None, 0, None
    y = x.new_empty(shape)
    if residual is not None:
        _need(residual.shape == shape and residual.dtype is x.dtype and
              residual.device == x.device, "residual must match x")
        rr, r_stride = _rows(residual, n)
        h = x.new_empty(shape)
    w = weight.contiguous()
    b = None if bias is None else bias.contiguous()
    rows = x.numel() // n
    stats = x.new_empty((2,) + shape[:-1], dtype=torch.float32)
    if rows:
        at = stats.data_ptr()
        _check(lib, lib.sieve_norm_forward(
            xr.data_ptr(), x_stride, None if rr is None else rr.data_ptr(), r_stride,
            w.data_ptr(), None if b is None else b.data_ptr(), code, _CODES[w.dtype], rows, n, eps,
            y.data_ptr(), None if h is None else h.data_ptr(), at, at + 4 * rows,
            _raw_stream(x.device)))
    return y, x if h is None else h, stats[0], stats[1]


def _check_affine(x, weight, bias, n):
    for name, t in (("weight", weight), ("bias", bias)):
        if t is None:
            continue
        _need(t.shape == (n,) and t.device == x.device, f"{name} must be [{n}] on x's device")
        if t.dtype not in (x.dtype, torch.float32):
            raise TypeError(f"{name} must be of x's dtype or float32")
    if bias is not None and bias.dtype != weight.dtype:
        raise TypeError("weight and bias must share a dtype")


def layer_norm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor,
                        mean: torch.Tensor, rstd: torch.Tensor,
                        dh: Optional[torch.Tensor] = None, weight_grad: bool = True,
                        bias_grad: bool = True, stream=None):
    """Gradients of ``layer_norm_forward`` from its ``h``, ``mean`` and ``rstd``.  ``dh`` is the
    gradient that reaches ``h`` by another way.  Returns ``(dx, dweight, dbias)``; ``dx`` is the
    gradient of x and of the residual alike, the other two are None where not asked for."""
    _need(h.is_cuda, "h must be a GPU tensor")
    args = (dy, h, weight, mean, rstd, dh, weight_grad, bias_grad)
    if _here(h.device, stream):
        return _norm_backward(*args)
    with _on(h.device, stream):
        return _norm_backward(*args)


def _norm_backward(dy, h, weight, mean, rstd, dh, weight_grad, bias_grad):
    shape = h.shape
    _need(len(shape) >= 1 and shape[-1] >= 1, "h must have a last axis of at least one value")
    n = shape[-1]
    code = _code(h, "h")
    _check_affine(h, weight, None, n)
    rows = h.numel() // n
    for name, t in (("dy", dy), ("dh", dh)):
        if t is not None:
            _need(t.shape == shape and t.dtype is h.dtype and t.device == h.device,
                  f"{name} must match h")
    for name, t in (("mean", mean), ("rstd", rstd)):
        _need(t.numel() == rows and t.dtype is torch.float32 and t.device == h.device and
              t.is_contiguous(), f"{name} must be the forward pass's, one float32 a row")
    lib = _library()
    hr, h_stride = _rows(h, n)
    dr, dy_stride = _rows(dy, n)
    er = None if dh is None else dh.contiguous()
    w = weight.contiguous()
    dx = h.new_empty(shape)
    dw = w.new_empty(n) if weight_grad else None
    db = w.new_empty(n) if bias_grad else None
    size = lib.sieve_norm_workspace(rows, n)
    space = _workspace(lib, size, h.device)
    _check(lib, lib.sieve_norm_backward(
        _ptr(dr), dy_stride, _ptr(hr), h_stride, w.data_ptr(), _ptr(mean), _ptr(rstd), _ptr(er),
        code, _CODES[w.dtype], rows, n, _ptr(dx), _ptr(dw), _ptr(db), _ptr(space), size,
        _raw_stream(h.device)))
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, residual):
        y, h, mean, rstd = layer_norm_forward(x, weight, bias, eps, residual)
        ctx.set_materialize_grads(False)  # an output that nothing uses has no gradient
        ctx.save_for_backward(h, weight, mean, rstd)
        ctx.has_bias, ctx.has_residual = bias is not None, residual is not None
        if ctx.has_residual:
            return y, h
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh=None):
        h, weight, mean, rstd = ctx.saved_tensors
        want_w, want_b = ctx.needs_input_grad[1], ctx.has_bias and ctx.needs_input_grad[2]
        if dy is None:  # only the sum was used
            dx = dh
            dw = torch.zeros_like(weight) if want_w else None
            db = torch.zeros_like(weight) if want_b else None
        else:
            dx, dw, db = layer_norm_backward(dy, h, weight, mean, rstd, dh, want_w, want_b)
        return dx, dw, db, None, dx if ctx.has_residual else None


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5, residual: Optional[torch.Tensor] = None):
    """Differentiable layer norm.  Returns ``y``, or ``(y, x + residual)`` with a residual."""
    return _LayerNorm.apply(x, weight, bias, eps, residual)


# ---- attention ----------------------------------------------------------------------------


def _offsets(t, name: str) -> torch.Tensor:
    t = torch.as_tensor(t)
    _need(t.dim() == 1 and t.numel() >= 1 and not t.is_floating_point(),
          f"{name} must be whole numbers, one more than the sequences")
    return t.to(device="cpu", dtype=torch.int64).contiguous()


class AttentionPlan:
    """The attention of one packed batch (``sieve_attn_create``): sequence ``s`` has the queries
    ``q_offsets[s] .. q_offsets[s+1]-1`` and the keys ``k_offsets[s] .. k_offsets[s+1]-1``
    (``q_offsets`` where that is not given).  Queries fewer than the keys are the sequence's last.
    Every layer and both passes over the batch share the plan.  ``num_buckets`` > 0 adds a
    learned bias ``[num_buckets, heads]`` by buckets of the relative position."""

    def __init__(self, q_offsets, k_offsets=None, *, heads: int, kv_heads: Optional[int] = None,
                 head_dim: int, dtype: torch.dtype, causal: bool = False,
                 scale: Optional[float] = None, num_buckets: int = 0, max_distance: int = 0,
                 device=None):
        self._h = None
        lib = _library()
        if dtype not in _CODES:
            raise TypeError(f"unsupported dtype {dtype} (float32, float16 or bfloat16)")
        qo = _offsets(q_offsets, "q_offsets")
        ko = qo if k_offsets is None else _offsets(k_offsets, "k_offsets")
        _need(qo.numel() == ko.numel(), "q_offsets and k_offsets must have as many sequences")
        self.heads, self.kv_heads = int(heads), int(heads if kv_heads is None else kv_heads)
        self.head_dim, self.dtype, self.causal = int(head_dim), dtype, bool(causal)
        self.num_buckets, self.max_distance = int(num_buckets), int(max_distance)
        self.queries, self.keys = int(qo[-1]), int(ko[-1])
        _need(self.head_dim >= 1, "head_dim must be at least 1")
        self.scale = 1.0 / math.sqrt(self.head_dim) if scale is None else float(scale)
        device = torch.device("cuda" if device is None else device)
        _need(device.type == "cuda", "a plan needs a GPU")
        self.device = device if device.index is not None else \
            torch.device("cuda", torch.cuda.current_device())
        self._q_shape = torch.Size((self.queries, self.heads, self.head_dim))
        self._k_shape = torch.Size((self.keys, self.kv_heads, self.head_dim))
        self._lse_shape = self._q_shape[:2]
        desc = _Desc(_CODES[dtype], self.heads, self.kv_heads, self.head_dim, int(self.causal),
                     self.num_buckets, self.max_distance, self.scale, qo.numel() - 1,
                     qo.data_ptr(), ko.data_ptr())
        handle = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib, lib.sieve_attn_create(ctypes.byref(desc),
                                              _raw_stream(self.device),
                                              ctypes.byref(handle)))
        self._h, self._lib = handle, lib
        self._space = [int(lib.sieve_attn_workspace(handle, b)) for b in (0, 1)]

    def close(self):
        if self._h is not None and self._h.value:
            self._lib.sieve_attn_free(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _tensor(self, t: torch.Tensor, name: str, shape) -> torch.Tensor:
        if t.dtype is self.dtype and t.shape == shape and t.device == self.device and \
                t.stride(2) == 1:
            return t
        if t.dtype != self.dtype:
            raise TypeError(f"{name} must be {self.dtype}, not {t.dtype}")
        if t.shape != shape or t.device != self.device:
            raise ValueError(f"{name} must be {list(shape)} on {self.device}, "
                             f"not {list(t.shape)} on {t.device}")
        return _side_by_side(t)

    def _inputs(self, q, k, v, key_mask, bias):
        if self._h is None:
            raise SieveError(-1, "the plan is closed")
        q = self._tensor(q, "q", self._q_shape)
        k = self._tensor(k, "k", self._k_shape)
        v = self._tensor(v, "v", self._k_shape)
        if key_mask is not None:
            _need(key_mask.dtype in (torch.bool, torch.uint8) and
                  key_mask.shape == (self.keys,) and key_mask.device == self.device,
                  f"key_mask must be [{self.keys}] bool on the plan's device")
            key_mask = key_mask.contiguous()
        _need((bias is not None) == (self.num_buckets > 0),
              "bias is given with a plan that has buckets, and only then")
        if bias is not None:
            if bias.dtype != self.dtype:
                raise TypeError(f"bias must be {self.dtype}, not {bias.dtype}")
            _need(bias.shape == (self.num_buckets, self.heads) and bias.device == self.device,
                  f"bias must be [{self.num_buckets}, {self.heads}] on the plan's device")
            bias = bias.contiguous()
        return q, k, v, key_mask, bias

    def forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                key_mask: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """``q`` [queries, heads, head_dim], ``k`` and ``v`` [keys, kv_heads, head_dim], any
        strides with neighbouring values side by side; ``key_mask`` [keys], False: not seen.
        Returns ``(out, lse)``: the output and the fp32 logarithm of each row's sum."""
        if _here(self.device, stream):
            return self._forward(q, k, v, key_mask, bias)
        with _on(self.device, stream):
            return self._forward(q, k, v, key_mask, bias)

    def _forward(self, q, k, v, key_mask, bias):
        q, k, v, key_mask, bias = self._inputs(q, k, v, key_mask, bias)
        out = q.new_empty(self._q_shape)
        lse = q.new_empty(self._lse_shape, dtype=torch.float32)
        size = self._space[0]
        space = _workspace(self._lib, size, self.device) if size else None
        held, (hq, hk, hv, ho) = _heads(q, k, v, out)
        _check(self._lib, self._lib.sieve_attn_forward(
            self._h, hq, hk, hv, _ptr(key_mask), _ptr(bias), ho, lse.data_ptr(), _ptr(space),
            size, _raw_stream(self.device)))
        return out, lse

    def backward(self, dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                 out: torch.Tensor, lse: torch.Tensor, key_mask: Optional[torch.Tensor] = None,
                 bias: Optional[torch.Tensor] = None, bias_grad: Optional[bool] = None,
                 stream=None):
        """Gradients from the output's, and the forward pass's inputs and results.  Returns
        ``(dq, dk, dv, dbias)``; ``dbias`` is None without a bias (or with ``bias_grad=False``)."""
        args = (dout, q, k, v, out, lse, key_mask, bias, bias_grad)
        if _here(self.device, stream):
            return self._backward(*args)
        with _on(self.device, stream):
            return self._backward(*args)

    def _backward(self, dout, q, k, v, out, lse, key_mask, bias, bias_grad):
        q, k, v, key_mask, bias = self._inputs(q, k, v, key_mask, bias)
        dout = self._tensor(dout, "dout", self._q_shape)
        out = self._tensor(out, "out", self._q_shape)
        _need(lse.shape == self._lse_shape and lse.dtype is torch.float32 and
              lse.is_contiguous() and lse.device == self.device, "lse must be the forward pass's")
        dq = q.new_empty(self._q_shape)
        dk, dv = k.new_empty(self._k_shape), v.new_empty(self._k_shape)
        dbias = bias.new_empty(bias.shape) if bias is not None and bias_grad is not False else None
        size = self._space[1]
        space = _workspace(self._lib, size, self.device) if size else None
        held, (hdo, hq, hk, hv, ho, hdq, hdk, hdv) = _heads(dout, q, k, v, out, dq, dk, dv)
        _check(self._lib, self._lib.sieve_attn_backward(
            self._h, hdo, hq, hk, hv, ho, _ptr(lse), _ptr(key_mask), _ptr(bias), hdq, hdk, hdv,
            _ptr(dbias), _ptr(space), size, _raw_stream(self.device)))
        return dq, dk, dv, dbias


def _side_by_side(t: torch.Tensor) -> torch.Tensor:
    """A view that the kernels take (a head's values side by side), else a copy."""
    return t if t.stride(2) == 1 or t.shape[2] == 1 or t.numel() == 0 else t.contiguous()


_HEADS_SIZE = ctypes.sizeof(_Heads)


def _heads(*tensors: torch.Tensor):
    """The tensors' ``sieve_heads`` one after another: what holds them, and their addresses.
    (One array of whole numbers: a ctypes structure each costs a microsecond each.)"""
    fields = []
    for t in tensors:
        token, head, _ = t.stride()
        fields += (t.data_ptr(), token, head)
    held = array.array("q", fields)
    first = held.buffer_info()[0]
    return held, range(first, first + len(tensors) * _HEADS_SIZE, _HEADS_SIZE)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, plan, key_mask, bias):
        out, lse = plan.forward(q, k, v, key_mask, bias)
        ctx.save_for_backward(q, k, v, out, lse, key_mask, bias)
        ctx.plan = plan
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, key_mask, bias = ctx.saved_tensors
        dq, dk, dv, dbias = ctx.plan.backward(dout, q, k, v, out, lse, key_mask, bias,
                                              bias_grad=ctx.needs_input_grad[5])
        return dq, dk, dv, None, None, dbias


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: AttentionPlan,
              key_mask: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None):
    """Differentiable attention over ``plan``'s packed batch (see ``AttentionPlan.forward``)."""
    return _Attention.apply(q, k, v, plan, key_mask, bias)
