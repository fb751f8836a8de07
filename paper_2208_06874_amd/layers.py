"""Binding of the layers next to the projection (include/vp.h): embedding and its gradient, the norm with the
residual's addition and its gradient, the 8-bit product, beam search's selection over whole rows and the
reordering of states.  Argument marshalling only, as in vp.py; every step runs in the library's HIP kernels.

All calls run on `stream` (default: torch's current stream); what they allocate belongs to that stream.  Inputs
are tensors with contiguous rows, at any stride between rows, on the current device.
"""
from __future__ import annotations

import contextlib
import ctypes
from collections import namedtuple
from typing import Optional, Sequence, Tuple

from .vp import VP_ERR_UNSUPPORTED, VpError, _check, _ptr, _want, last_error, lib

TYPE_NAMES = ("float16", "bfloat16", "float32")     # vp_type
SCALE_BLOCK = 128
MAX_STATES = 8


class _Torch:
    """torch, imported on the first call, and what the calls below ask it for every time."""
    torch = None

    @classmethod
    def load(cls):
        import torch
        cls.types = {getattr(torch, n): i for i, n in enumerate(TYPE_NAMES)}
        # (a raw stream's handle costs 0.1 us, torch.cuda.current_stream() with its device look-ups 2)
        cls.raw_stream = staticmethod(getattr(torch._C, "_cuda_getCurrentRawStream", None) or
                                      (lambda index: torch.cuda.current_stream(index).cuda_stream))
        cls.current_device = staticmethod(getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device)
        cls.torch = torch
        return torch


def _torch():
    return _Torch.torch or _Torch.load()


def _type_code(t, name: str) -> int:
    """vp_type of a torch dtype."""
    _torch()
    code = _Torch.types.get(t)
    if code is None:
        raise ValueError("%s must be one of %s, got %s" % (name, ", ".join(TYPE_NAMES), t))
    return code


def _rows(t, name: str, d: Optional[int] = None, n: Optional[int] = None, dtype=None, device=None):
    """A [n, d] tensor on the GPU with contiguous rows -> (n, d, elements from row to row).  Without a `device`, the
    current one."""
    if not isinstance(t, _torch().Tensor):
        raise TypeError("%s must be a torch.Tensor, got %s" % (name, type(t).__name__))
    if t.dim() != 2:
        raise ValueError("%s must have two dimensions, got shape %s" % (name, tuple(t.shape)))
    rows, cols = t.shape
    if (d is not None and cols != d) or (n is not None and rows != n):
        raise ValueError("%s must have shape (%s, %s), got %s" % (name, "n" if n is None else n, "d" if d is None else d, (rows, cols)))
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must live in GPU memory (got a %s tensor)" % (name, t.device))
    _same_device(t, name, device)
    stride, inner = t.stride()
    if (cols > 1 and inner != 1) or (rows > 1 and stride < cols):
        raise ValueError("%s must have contiguous rows that do not overlap, got strides %s" % (name, (stride, inner)))
    return rows, cols, max(stride, cols)


def _same_device(t, name: str, device=None):
    if device is not None:
        if t.device != device:
            raise ValueError("%s is on %s, the others on %s" % (name, t.device, device))
    elif t.get_device() != _Torch.current_device():
        raise ValueError("%s is on %s, the current device is %d" % (name, t.device, _Torch.current_device()))


_NOWHERE = contextlib.nullcontext()


def _on(stream):
    """Allocations belong to the stream that the call runs on."""
    return _NOWHERE if stream is None else _torch().cuda.stream(stream)


def _handle(stream, device) -> int:
    return _Torch.raw_stream(device.index) if stream is None else stream.cuda_stream


def _like(t):
    """An uninitialised [n, d] of t's type (0.5 us less than by shape, where t itself is contiguous)."""
    return _torch().empty_like(t) if t.is_contiguous() else _torch().empty(t.shape, dtype=t.dtype, device=t.device)


def _bytes(need: int, device):
    torch = _torch()
    if need == 0:
        raise VpError(VP_ERR_UNSUPPORTED, last_error())
    return torch.empty(need, dtype=torch.uint8, device=device)


def vp_embed(table, ids, scale: float = 1.0, out_dtype=None, out=None, stream=None):
    """scale * table[ids] -> [*ids.shape, d] of out_dtype (default: the table's); ids (int32) outside the table give
    rows of zeros."""
    torch = _torch()
    V, d, stride = _rows(table, "table")
    table_type = _type_code(table.dtype, "table's type")
    _want(ids, "ids", torch.int32, None, table.device)
    out_dtype = (table.dtype if out is None else out.dtype) if out_dtype is None else out_dtype
    out_type = _type_code(out_dtype, "out_dtype")
    if out is None:
        with _on(stream):
            out = torch.empty((*ids.shape, d), dtype=out_dtype, device=table.device)
    else:
        _want(out, "out", out_dtype, (*ids.shape, d), table.device)
    _check(lib().vp_embed(table.data_ptr(), table_type, stride, V, d, ids.data_ptr(), ids.numel(), scale,
                          out.data_ptr(), out_type, _handle(stream, table.device)))
    return out


def vp_embed_grad(dout, ids, V: int, scale: float = 1.0, padding_id: int = -1, grad_dtype=None, out=None, stream=None):
    """The gradient of vp_embed with respect to its table: dout [n, d], ids int32 [n] -> grad [V, d] of grad_dtype
    (default: float32), every row written; padding_id's row is zero."""
    torch = _torch()
    n, d, stride = _rows(dout, "dout")
    dout_type = _type_code(dout.dtype, "dout's type")
    _want(ids, "ids", torch.int32, (n,), dout.device)
    grad_dtype = (torch.float32 if out is None else out.dtype) if grad_dtype is None else grad_dtype
    grad_type = _type_code(grad_dtype, "grad_dtype")
    need = lib().vp_embed_grad_workspace_bytes(n, V, d)
    with _on(stream):
        ws = _bytes(need, dout.device)
        if out is None:
            out = torch.empty((V, d), dtype=grad_dtype, device=dout.device)
        else:
            _want(out, "out", grad_dtype, (V, d), dout.device)
        _check(lib().vp_embed_grad(dout.data_ptr(), dout_type, stride, ids.data_ptr(), n, V, d, scale, padding_id,
                                   out.data_ptr(), grad_type, ws.data_ptr(), need, _handle(stream, dout.device)))
    return out


NormResult = namedtuple("NormResult", "sum norm q scales rstd")


def vp_add_norm(x, weight, residual=None, eps: float = 1e-6, norm_dtype=None, quantize: bool = False, rstd: bool = False,
                inplace: bool = False, stream=None) -> NormResult:
    """Root-mean-square norm of x + residual: NormResult(sum, norm, q, scales, rstd).
    sum is x + residual in their type (x itself without a residual; written over the residual if `inplace`); norm is
    in norm_dtype (default: x's type unless `quantize`; None otherwise); q (float8_e4m3fn [n, d], rows 128-byte
    multiples apart) and scales (fp32 [n, ceil(d / 128)]) are there if `quantize`; rstd (fp32 [n]) if `rstd`."""
    torch = _torch()
    n, d, x_stride = _rows(x, "x")
    code = _type_code(x.dtype, "x's type")
    dev = x.device
    r_stride = d
    if residual is not None:
        r_stride = _rows(residual, "residual", d, n, x.dtype, dev)[2]
    weight_type = _type_code(getattr(weight, "dtype", None), "weight's type")
    _want(weight, "weight", weight.dtype, (d,), dev)
    if norm_dtype is None and not quantize:
        norm_dtype = x.dtype
    norm_type = 0 if norm_dtype is None else _type_code(norm_dtype, "norm_dtype")
    if inplace and (residual is None or not residual.is_contiguous()):
        raise ValueError("inplace needs a contiguous residual")
    blocks = -(-d // SCALE_BLOCK)
    total, norm, q, scales, r = x, None, None, None, None
    with _on(stream):
        if residual is not None:
            total = residual if inplace else _like(x)
        if norm_dtype is not None:
            norm = _like(x) if norm_dtype is x.dtype else torch.empty((n, d), dtype=norm_dtype, device=dev)
        if quantize:
            q = torch.empty((n, blocks * SCALE_BLOCK), dtype=torch.float8_e4m3fn, device=dev)
            scales = torch.empty((n, blocks), dtype=torch.float32, device=dev)
        if rstd:
            r = torch.empty((n,), dtype=torch.float32, device=dev)
    _check(lib().vp_add_norm(x.data_ptr(), x_stride, _ptr(residual), r_stride, code, weight.data_ptr(), weight_type, n, d,
                             eps, None if residual is None else total.data_ptr(), _ptr(norm), norm_type, _ptr(q),
                             _ptr(scales), _ptr(r), _handle(stream, dev)))
    return NormResult(total, norm, q if q is None or d % SCALE_BLOCK == 0 else q[:, :d], scales, r)


def vp_add_norm_grad(dnorm, s, weight, rstd, dsum=None, stream=None):
    """The gradient of vp_add_norm's (sum, norm): (dx [n, d] in s's type, the same for x and residual; dweight fp32 [d])."""
    torch = _torch()
    n, d, s_stride = _rows(s, "s")
    code = _type_code(s.dtype, "s's type")
    dev = s.device
    dn_stride = _rows(dnorm, "dnorm", d, n, s.dtype, dev)[2]
    ds_stride = d if dsum is None else _rows(dsum, "dsum", d, n, s.dtype, dev)[2]
    weight_type = _type_code(getattr(weight, "dtype", None), "weight's type")
    _want(weight, "weight", weight.dtype, (d,), dev)
    _want(rstd, "rstd", torch.float32, (n,), dev)
    need = lib().vp_add_norm_grad_workspace_bytes(n, d)
    with _on(stream):
        ws = _bytes(need, dev)
        dx = _like(s)
        dweight = torch.empty((d,), dtype=torch.float32, device=dev)
        _check(lib().vp_add_norm_grad(dnorm.data_ptr(), dn_stride, s.data_ptr(), s_stride, _ptr(dsum), ds_stride, code,
                                      weight.data_ptr(), weight_type, rstd.data_ptr(), n, d, dx.data_ptr(),
                                      dweight.data_ptr(), ws.data_ptr(), need, _handle(stream, dev)))
    return dx, dweight


class ScaledWeight:
    """An 8-bit weight [M, d] with its scales, laid out for vp_scaled_matmul."""

    def __init__(self, packed, M: int, d: int):
        self.packed, self.M, self.d, self.device = packed, M, d, packed.device


def vp_scaled_pack(wq, ws, stream=None) -> ScaledWeight:
    """wq float8_e4m3fn [M, d] and ws fp32 [ceil(M / 128), ceil(d / 128)] -> a ScaledWeight with its own copy."""
    torch = _torch()
    M, d, stride = _rows(wq, "wq", dtype=torch.float8_e4m3fn)
    _want(ws, "ws", torch.float32, (-(-M // SCALE_BLOCK), -(-d // SCALE_BLOCK)), wq.device)
    need = lib().vp_scaled_pack_bytes(M, d)
    with _on(stream):
        packed = _bytes(need, wq.device)
    _check(lib().vp_scaled_pack(wq.data_ptr(), stride, ws.data_ptr(), M, d, packed.data_ptr(), need, _handle(stream, wq.device)))
    return ScaledWeight(packed, M, d)


def vp_scaled_matmul(weight: ScaledWeight, xq, xs, bias=None, out_dtype=None, out=None, stream=None):
    """xq float8_e4m3fn [n, d] with scales xs fp32 [n, ceil(d / 128)], times the weight, plus bias [M]
    -> [n, M] of out_dtype (default: float16).  float32 outputs are summed in 32 bits throughout; for 16-bit ones the sums
    of eight neighbouring columns are made in 13 bits below their largest product, at up to twice the rate."""
    torch = _torch()
    if not isinstance(weight, ScaledWeight):
        raise TypeError("weight must be a ScaledWeight (vp_scaled_pack), got %s" % type(weight).__name__)
    M, d, dev = weight.M, weight.d, weight.device
    n, _, stride = _rows(xq, "xq", d, None, torch.float8_e4m3fn, dev)
    _same_device(xq, "xq")
    _want(xs, "xs", torch.float32, (n, -(-d // SCALE_BLOCK)), dev)
    bias_type = 0
    if bias is not None:
        bias_type = _type_code(getattr(bias, "dtype", None), "bias's type")
        _want(bias, "bias", bias.dtype, (M,), dev)
    out_dtype = (torch.float16 if out is None else out.dtype) if out_dtype is None else out_dtype
    out_type = _type_code(out_dtype, "out_dtype")
    need = lib().vp_scaled_matmul_workspace_bytes(n, d)
    with _on(stream):
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        if out is None:
            out = torch.empty((n, M), dtype=out_dtype, device=dev)
        else:
            _want(out, "out", out_dtype, (n, M), dev)
        _check(lib().vp_scaled_matmul(weight.packed.data_ptr(), M, d, xq.data_ptr(), stride, xs.data_ptr(), n, _ptr(bias),
                                      bias_type, out.data_ptr(), out_type, ws.data_ptr(), need, _handle(stream, dev)))
    return out


def vp_beam_select(logits, scores, B: int, allowed=None, done=None, eos: int = -1, out=None, stream=None):
    """The B best continuations of every sentence over whole rows of logits [S * B, V]: (scores fp32, parent int32,
    token int32, done uint8), each [S * B]; missing ones are (-inf, -1, -1, 0).
    allowed: int32 [S * B, ceil(V / 32)], bit t % 32 of word t / 32 set where token t may follow; done: uint8 or bool
    [S * B], hypotheses that have ended and go on with eos alone."""
    torch = _torch()
    n, V, stride = _rows(logits, "logits")
    code = _type_code(logits.dtype, "logits' type")
    dev = logits.device
    if B < 1 or n % B != 0:
        raise ValueError("the %d rows are not a whole number of sentences of %d hypotheses" % (n, B))
    _want(scores, "scores", torch.float32, (n,), dev)
    bits_stride = 0
    if allowed is not None:
        bits_stride = _rows(allowed, "allowed", -(-V // 32), n, torch.int32, dev)[2]
    if done is not None:
        _want(done, "done", torch.bool if done.dtype == torch.bool else torch.uint8, (n,), dev)
        if not 0 <= eos < V:
            raise ValueError("eos = %d is no token of %d: ended hypotheses need one" % (eos, V))
    need = lib().vp_beam_select_workspace_bytes(n // B, B, V)
    with _on(stream):
        ws = _bytes(need, dev)
        if out is None:
            parent = torch.empty(n, dtype=torch.int32, device=dev)
            out = (torch.empty_like(scores), parent, torch.empty_like(parent), torch.empty(n, dtype=torch.uint8, device=dev))
        else:
            for t, name, dtype in zip(out, ("scores", "parent", "token", "done"), (torch.float32, torch.int32, torch.int32, torch.uint8)):
                _want(t, "out's " + name, dtype, (n,), dev)
        _check(lib().vp_beam_select(logits.data_ptr(), code, stride, scores.data_ptr(), n // B, B, V, _ptr(allowed),
                                    bits_stride, _ptr(done), eos, out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(),
                                    out[3].data_ptr(), ws.data_ptr(), need, _handle(stream, dev)))
    return out


STATE_DIMS = 8


class State(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("elem_bytes", ctypes.c_int32), ("dims", ctypes.c_int32),
                ("row_dim", ctypes.c_int32), ("sizes", ctypes.c_int64 * STATE_DIMS), ("strides", ctypes.c_int64 * STATE_DIMS)]


def vp_beam_reorder(states: Sequence[Tuple], parent, B: int, stream=None):
    """Moves what belongs to the hypotheses, in place: along dimension `dim` of every (tensor, dim), row s * B + b
    becomes what row s * B + parent[s * B + b] was; rows with a parent outside [0, B) stay.  Tensors may be views
    with any strides that do not overlap themselves (nor each other).  Where one of them is refused, none has moved."""
    torch = _torch()
    _want(parent, "parent", torch.int32)
    _same_device(parent, "parent")
    n = parent.numel()
    if parent.dim() != 1 or B < 1 or n % B != 0:
        raise ValueError("parent must hold a whole number of sentences of %d hypotheses, got shape %s" % (B, tuple(parent.shape)))
    described = []
    for i, (t, dim) in enumerate(states):
        name = "state %d" % i
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor, got %s" % (name, type(t).__name__))
        if not 1 <= t.dim() <= STATE_DIMS or not -t.dim() <= dim < t.dim():
            raise ValueError("%s has %d dimensions, rows along %d" % (name, t.dim(), dim))
        if not t.is_cuda:
            raise ValueError("%s must live in GPU memory (got a %s tensor)" % (name, t.device))
        _same_device(t, name, parent.device)
        if t.shape[dim] != n:
            raise ValueError("%s has %d rows along %d, parent %d" % (name, t.shape[dim], dim, n))
        k = t.dim()
        described.append(State(t.data_ptr(), t.element_size(), k, dim % k, (ctypes.c_int64 * STATE_DIMS)(*t.shape),
                               (ctypes.c_int64 * STATE_DIMS)(*t.stride())))
    parts = [described[at:at + MAX_STATES] for at in range(0, len(described), MAX_STATES)]
    parts = [((State * len(part))(*part), len(part)) for part in parts]
    if len(parts) > 1:      # (nothing moves before all of them are known to be taken)
        for part, k in parts:
            _check(lib().vp_beam_reorder_check(part, k, n // B, B))
    for part, k in parts:
        _check(lib().vp_beam_reorder(part, k, parent.data_ptr(), n // B, B, _handle(stream, parent.device)))
