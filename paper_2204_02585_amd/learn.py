"""Operators on learned tables and layers (include/sqn.h, "learned tables and
layers") over torch device tensors: rows of a table by index with the table's
gradient, updates orthogonalised by Newton-Schulz products, and layers held in
4-bit blocks.

Like `binding`, argument marshalling only: every value is computed by the
HIP library.  Calls run on torch's current stream unless `stream` is given,
which then waits for the work queued on the current stream; scratch and
outputs come from torch's allocator.  Tensors and `stream` must belong to
torch's current device (`with torch.cuda.device(x.device):`); a call on
another's is refused.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch
from torch.autograd import forward_ad

from . import binding
from .binding import Matrix, _check, _current_stream, _order_after_current, lib

BLOCK = 32                                      # elements of a 4-bit block
MUON = (3.4445, -4.7750, 2.0315)                # the Muon optimiser's coefficients

_CODES = {torch.float32: binding.SQN_F32, torch.float16: binding.SQN_F16, torch.bfloat16: binding.SQN_BF16}
_IDS = {torch.int32: binding.SQN_I32, torch.int64: binding.SQN_I64}


def _code(dtype: torch.dtype, name: str) -> int:
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, got {dtype}")
    return code


def _on_gpu(t: torch.Tensor, name: str, beside: Optional[torch.Tensor] = None) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must live on a CUDA device")
    if beside is not None and t.get_device() != beside.get_device():
        raise ValueError(f"{name} must live on {beside.device}, not {t.device}")


def _rows(t: torch.Tensor) -> torch.Tensor:
    """`t` as [rows, cols] with consecutive elements in a row; a copy only where
    the layout needs one."""
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1])
    if t.shape[1] != 1 and t.stride(1) != 1:
        t = t.contiguous()
    return t


def _matrix(t: torch.Tensor, name: str) -> Matrix:
    """`t` is of _rows()'s form."""
    rows, cols = t.shape
    code = _CODES.get(t.dtype)
    if code is None:
        code = _code(t.dtype, name)
    return Matrix(t.data_ptr(), rows, cols, t.stride(0) if rows > 1 else cols, code, 0)


def _out(out: Optional[torch.Tensor], shape, dtype, beside: torch.Tensor, name: str = "out") -> torch.Tensor:
    """A new tensor beside another, or the caller's, whose rows must lie apart."""
    if out is None:
        if type(beside) is torch.Tensor:
            return beside.new_empty(shape, dtype=dtype)
        return torch.empty(shape, dtype=dtype, device=beside.device)
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype or out.device != beside.device:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {beside.device}")
    if not out.is_contiguous() and not (out.dim() == 2 and out.stride(1) == 1 and out.stride(0) >= out.shape[1]):
        raise ValueError(f"{name} must be contiguous, or a matrix of contiguous rows")
    return out


def _workspace(size: int, beside: torch.Tensor) -> Optional[torch.Tensor]:
    return torch.empty(size, dtype=torch.uint8, device=beside.device) if size else None


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _on(stream, *tensors) -> int:
    """The stream's address, ordered after the current stream's work."""
    if stream is None:
        return _current_stream()
    _order_after_current(stream, *tensors)
    return stream.cuda_stream


def _tangent(t: torch.Tensor) -> Optional[torch.Tensor]:
    """The tangent of a dual tensor of forward-mode differentiation, None of others."""
    if getattr(forward_ad, "_current_level", 0) < 0:        # none is open: spares a call the look
        return None
    return forward_ad.unpack_dual(t).tangent


def _no_tangent(what: str, *tensors) -> None:
    """A raw pointer would drop it without a word."""
    if any(t is not None and _tangent(t) is not None for t in tensors):
        raise RuntimeError(f"{what} has no forward-mode derivative")


# ---------------------------------------------------------------- rows of a table

def _ids(ids: torch.Tensor, beside: torch.Tensor) -> torch.Tensor:
    if ids.dtype not in _IDS:
        raise TypeError(f"ids must be int32 or int64, got {ids.dtype}")
    _on_gpu(ids, "ids", beside)
    return ids if ids.is_contiguous() else ids.contiguous()


def _lookup(table, ids, scale, out, stream):
    # a few rows take less time on the GPU (3 us for 32 of 2 KB) than this call
    # takes to issue (8 us), so what is known here is not looked up again
    _on_gpu(table, "table")
    if table.dim() != 2:
        raise ValueError(f"table must be a matrix, got shape {tuple(table.shape)}")
    source, ids = _rows(table), _ids(ids, table)
    of = _matrix(source, "table")
    if out is None:
        out = _out(None, (*ids.shape, of.cols), table.dtype, table)
        into = Matrix(out.data_ptr(), ids.numel(), of.cols, of.cols, of.dtype, 0)
    else:
        out = _out(out, (*ids.shape, of.cols), table.dtype, table)
        into = _matrix(_rows(out), "out")
    _check(lib.sqn_lookup(of, ids.data_ptr(), _IDS[ids.dtype], scale, into, _on(stream, source, ids, out)))
    return out


class _Lookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale):
        ctx.save_for_backward(ids)
        ctx.save_for_forward(ids)
        ctx.rows, ctx.scale, ctx.dtype = table.shape[0], scale, table.dtype
        return _lookup(table.detach(), ids, scale, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        (ids,) = ctx.saved_tensors
        if ctx.rows == 0:             # every index was outside; the library's gradient has a row
            return grad.new_zeros((0, grad.shape[-1]), dtype=ctx.dtype), None, None
        return lookup_gradient(grad, ids, ctx.rows, scale=ctx.scale, dtype=ctx.dtype), None, None

    @staticmethod
    def jvp(ctx, table, _ids, _scale):
        (ids,) = ctx.saved_tensors
        return lookup(table, ids, scale=ctx.scale)


def lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
           stream=None) -> torch.Tensor:
    """sqn_lookup: scale * table[ids], [*ids.shape, D]; an index outside the
    table (a padding mark) gives zeros.  Differentiable in a table that
    requires a gradient (without `out` and `stream`), by lookup_gradient, and
    in forward mode."""
    if out is None and stream is None:
        if (table.requires_grad and torch.is_grad_enabled()) or _tangent(table) is not None:
            return _Lookup.apply(table, ids, float(scale))
    else:
        _no_tangent("lookup with out or stream", table)
    return _lookup(table, ids, float(scale), out, stream)


def lookup_gradient(grad: torch.Tensor, ids: torch.Tensor, rows: int, scale: float = 1.0,
                    out: Optional[torch.Tensor] = None, accumulate: bool = False,
                    dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """sqn_lookup_gradient: the gradient [rows, D] of lookup's table, from grad
    [*ids.shape, D].  `dtype` (grad's own by default) is the result's;
    `accumulate` adds to `out` instead of writing all of it.  It is linear in
    grad, and so are its forward-mode derivatives (without `out` and `stream`);
    no gradient passes back through it."""
    tangent = _tangent(grad)
    if tangent is not None:
        if out is not None or stream is not None:
            _no_tangent("lookup_gradient with out or stream", grad)
        both = (forward_ad.unpack_dual(grad).primal, tangent)
        return forward_ad.make_dual(*(lookup_gradient(g, ids, rows, scale, dtype=dtype or grad.dtype) for g in both))
    _on_gpu(grad, "grad")
    if tuple(grad.shape[:-1]) != tuple(ids.shape) or grad.dim() == 0:
        raise ValueError(f"grad of shape {tuple(grad.shape)} does not go with ids of shape {tuple(ids.shape)}")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    ids = _ids(ids, grad)
    if out is not None and dtype is None:
        dtype = out.dtype
    out = _out(out, (int(rows), grad.shape[-1]), dtype or grad.dtype, grad)
    source = _rows(grad)
    size = lib.sqn_lookup_gradient_workspace(ids.numel(), out.shape[0], out.shape[1])
    work = _workspace(size, grad)
    _check(lib.sqn_lookup_gradient(_matrix(source, "grad"), ids.data_ptr(), _IDS[ids.dtype], float(scale),
                                   1 if accumulate else 0, _matrix(out, "out"), _ptr(work), size,
                                   _on(stream, source, ids, out, work)))
    return out


# ---------------------------------------------------------------- updates

def _batch(t: torch.Tensor, name: str) -> binding.Batch:
    b, m, n = t.shape
    return binding.Batch(t.data_ptr(), b, m, n, _code(t.dtype, name), *t.stride())


def orthogonalise(updates: torch.Tensor, steps: int = 5, coefficients=MUON, eps: float = 1e-7,
                  dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """sqn_orthogonalise: [m, n] or a batch [B, m, n] of updates, any strides,
    orthogonalised by `steps` Newton-Schulz products.  A bfloat16 result
    takes one product per factor pair, a float16 or float32 one three.  The
    first is off by 1.1 times its rounding (Gaussian updates: 1.83e-3 of the
    norm, 1.66e-3 the rounding alone); `dtype=torch.float32` and then
    `.to(torch.bfloat16)` has the rounding alone, in 1.4 to 3.1 times the
    time.  The same coefficients apply to every step.  No gradient passes
    through it."""
    _no_tangent("orthogonalise", updates)
    _on_gpu(updates, "updates")
    if updates.dim() not in (2, 3):
        raise ValueError(f"updates must be [m, n] or [B, m, n], got shape {tuple(updates.shape)}")
    if len(coefficients) != 3:
        raise ValueError("three coefficients are needed")
    if out is None:
        _code(dtype, "dtype")
        out = torch.empty(updates.shape, dtype=dtype, device=updates.device)
    elif out.shape != updates.shape or out.device != updates.device:
        raise ValueError(f"out must have shape {tuple(updates.shape)} on {updates.device}")
    source, target = (updates, out) if updates.dim() == 3 else (updates.unsqueeze(0), out.unsqueeze(0))
    if updates.numel() == 0:
        return out
    into = _batch(target, "out")
    size = lib.sqn_orthogonalise_workspace(into.batch, into.rows, into.cols, into.dtype)
    work = _workspace(size, updates)
    k = (ctypes.c_float * 3)(*coefficients)
    _check(lib.sqn_orthogonalise(_batch(source, "updates"), int(steps), k, float(eps), into, _ptr(work), size,
                                 _on(stream, updates, out, work)))
    return out


# ---------------------------------------------------------------- 4-bit blocks

class Quantised:
    """A matrix in 4-bit blocks: codes uint8 [rows, blocks * 16] and scales uint8
    [rows, blocks] of `cols` columns, blocks = ceil(cols / 32)."""

    __slots__ = ("codes", "scales", "cols")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int):
        blocks = (cols + BLOCK - 1) // BLOCK
        if (codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() != 2 or cols < 1
                or codes.shape[1] != 16 * blocks or scales.shape != (codes.shape[0], blocks)):
            raise ValueError(f"codes uint8 [rows, {16 * blocks}] and scales uint8 [rows, {blocks}] hold {cols} columns, "
                             f"got {codes.dtype} {tuple(codes.shape)} and {scales.dtype} {tuple(scales.shape)}")
        _on_gpu(codes, "codes")
        _on_gpu(scales, "scales", codes)
        if not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be contiguous")
        self.codes, self.scales, self.cols = codes, scales, int(cols)

    @property
    def shape(self):
        return (self.codes.shape[0], self.cols)

    @property
    def device(self):
        return self.codes.device

    def _arg(self) -> binding.QuantisedMatrix:
        return binding.QuantisedMatrix(self.codes.data_ptr(), self.scales.data_ptr(), self.codes.shape[0], self.cols)

    def values(self, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """sqn_quantised_values: what the blocks stand for, [rows, cols]."""
        _code(dtype, "dtype")
        out = _out(out, self.shape, dtype, self.codes)
        _check(lib.sqn_quantised_values(self._arg(), _matrix(out, "out"), _on(stream, self.codes, self.scales, out)))
        return out


def quantise(x: torch.Tensor, stream=None) -> Quantised:
    """sqn_quantise: x [rows, cols] in 4-bit blocks along its rows.  Codes and
    scales are whole numbers: no gradient passes through them."""
    _on_gpu(x, "x")
    if x.dim() != 2 or x.shape[1] < 1:
        raise ValueError(f"x must be a matrix, got shape {tuple(x.shape)}")
    source = _rows(x)
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    codes = torch.empty((rows, 16 * blocks), dtype=torch.uint8, device=x.device)
    scales = torch.empty((rows, blocks), dtype=torch.uint8, device=x.device)
    q = Quantised(codes, scales, cols)
    _check(lib.sqn_quantise(_matrix(source, "x"), q._arg(), _on(stream, source, codes, scales)))
    return q


def product(x, w: Quantised, bias: Optional[torch.Tensor] = None, relu: bool = False,
            dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """A layer on 4-bit blocks, act(x w^T + bias): x is Quantised [points, cols]
    (sqn_quantised_product) or a tensor [..., cols] that is quantised in the
    call (sqn_quantised_layer); w Quantised [units, cols]; bias float32
    [units].  `dtype` is the result's: x's own, float32 for a Quantised x.
    No gradient passes through it: it is the form for evaluation."""
    blocks = isinstance(x, Quantised)
    if not isinstance(w, Quantised):
        raise TypeError("w must be Quantised")
    _no_tangent("product", None if blocks else x, bias)
    _on_gpu(x.codes if blocks else x, "x", w.codes)
    shape = x.shape
    if len(shape) < 1 or shape[-1] != w.cols:
        raise ValueError(f"x must have w's {w.cols} columns, got shape {tuple(shape)}")
    units = w.codes.shape[0]
    if bias is not None:
        _on_gpu(bias, "bias", w.codes)
        if bias.dtype != torch.float32 or bias.shape != (units,) or not bias.is_contiguous():
            raise ValueError(f"bias must be a contiguous float32 tensor of shape {(units,)}")
    if dtype is None:
        dtype = out.dtype if out is not None else torch.float32 if blocks else x.dtype
    _code(dtype, "dtype")
    out = _out(out, (*shape[:-1], units), dtype, w.codes)
    if out.numel() == 0:
        return out
    into = _matrix(_rows(out), "out")
    if blocks:
        size = lib.sqn_quantised_product_workspace(shape[0], units, w.cols)
        work = _workspace(size, out)
        _check(lib.sqn_quantised_product(x._arg(), w._arg(), _ptr(bias), 1 if relu else 0, into, _ptr(work), size,
                                         _on(stream, x.codes, x.scales, w.codes, w.scales, bias, out, work)))
        return out
    source = _rows(x)
    size = lib.sqn_quantised_layer_workspace(source.shape[0], units, w.cols)
    work = _workspace(size, out)
    _check(lib.sqn_quantised_layer(_matrix(source, "x"), w._arg(), _ptr(bias), 1 if relu else 0, into, _ptr(work), size,
                                   _on(stream, source, w.codes, w.scales, bias, out, work)))
    return out
