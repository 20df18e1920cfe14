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
_ACTIVATIONS = {None: binding.SQN_ACT_NONE, "relu": binding.SQN_ACT_RELU, "gelu": binding.SQN_ACT_GELU,
                "silu": binding.SQN_ACT_SILU}
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


def _operand(t: torch.Tensor, name: str):
    """(_rows(t), _matrix() of it), looked at once: most of a small call is such looks."""
    if t.dim() != 2 or t.dtype not in _CODES:
        rows = _rows(t)
        return rows, _matrix(rows, name)
    rows, cols = t.shape
    pitch, step = t.stride()
    if step != 1 and cols != 1:
        t = t.contiguous()
        pitch = cols
    return t, Matrix(t.data_ptr(), rows, cols, pitch if rows > 1 else cols, _CODES[t.dtype], 0)


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


def _out_like(t: torch.Tensor) -> torch.Tensor:
    """A new contiguous tensor of t's shape and type."""
    return torch.empty_like(t) if type(t) is torch.Tensor and t.is_contiguous() else _out(None, t.shape, t.dtype, t)


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
    if getattr(forward_ad, "_current_level", 0) < 0:
        return
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


# ---------------------------------------------------------------- dropout

def _probability(p) -> float:
    p = float(p)
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p must lie in [0, 1], got {p}")
    return p


def _mask(p: float, seed: int, step: Optional[torch.Tensor], beside: torch.Tensor) -> Optional[binding.DropoutMask]:
    if step is not None:
        if step.dtype != torch.int64 or step.numel() != 1:
            raise ValueError(f"step must be an int64 tensor of one element, got {step.dtype} {tuple(step.shape)}")
        _on_gpu(step, "step", beside)
    return binding.DropoutMask(p, int(seed) & 0xFFFFFFFFFFFFFFFF, _ptr(step))


def _beside(t: torch.Tensor, shape, dtype, beside: torch.Tensor, name: str) -> None:
    _on_gpu(t, name, beside)
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _wants_gradient(*tensors) -> bool:
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _dropout(x, p, seed, step, residual, out, stream):
    _on_gpu(x, "x")
    if x.dim() == 0:
        raise ValueError("x must have a dimension")
    if residual is not None:
        _beside(residual, x.shape, x.dtype, x, "residual")
    mask = _mask(p, seed, step, x)
    out = _out_like(x) if out is None else _out(out, x.shape, x.dtype, x)
    if out.numel() == 0:
        return out
    source, of_x = _operand(x, "x")
    of_residual = None
    if residual is not None:
        residual, of_residual = _operand(residual, "residual")
    _check(lib.sqn_dropout(of_x, mask, of_residual, _operand(out, "out")[1], _on(stream, source, residual, step, out)))
    return out


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, step, p, seed):
        # saved, so that a step that is changed before the backward pass is noticed
        ctx.save_for_backward(step)
        ctx.save_for_forward(step)
        ctx.p, ctx.seed = p, seed
        return _dropout(x.detach(), p, seed, step, None if residual is None else residual.detach(), None, None)

    @staticmethod
    def backward(ctx, grad):
        (step,) = ctx.saved_tensors
        grad_x = dropout(grad, ctx.p, ctx.seed, step) if ctx.needs_input_grad[0] else None
        return grad_x, grad if ctx.needs_input_grad[1] else None, None, None, None

    @staticmethod
    def jvp(ctx, x, residual, _step, _p, _seed):
        (step,) = ctx.saved_tensors
        if x is None:
            return residual
        return dropout(x, ctx.p, ctx.seed, step, residual)


def dropout(x: torch.Tensor, p: float, seed: int = 0, step: Optional[torch.Tensor] = None,
            residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """sqn_dropout: x [..., cols] with a share p of its elements zeros and the
    rest times 1 / (1 - p), plus `residual` if there is one.  The mask is made
    from `seed` (an int) plus `step` (an int64 tensor of one element on the
    device, for captured graphs; None: nothing) and each element's place; it is
    never stored, and the same arguments give the same mask.  `out` may be x or
    the residual.  Differentiable in x and the residual (without `out` and
    `stream`), also twice, and in forward mode; the gradient makes the mask
    again, so `step` must hold its value until then."""
    p = _probability(p)
    if out is None and stream is None:
        if (_wants_gradient(x, residual) or _tangent(x) is not None
                or (residual is not None and _tangent(residual) is not None)):
            return _Dropout.apply(x, residual, step, p, int(seed))
    else:
        _no_tangent("dropout with out or stream", x, residual)
    return _dropout(x, p, seed, step, residual, out, stream)


# ---------------------------------------------------------------- layers

def _activation(name) -> int:
    if name not in _ACTIVATIONS:
        raise ValueError(f"activation must be None, 'relu', 'gelu' or 'silu', got {name!r}")
    return _ACTIVATIONS[name]


def _factors(x: torch.Tensor, w: torch.Tensor) -> None:
    _on_gpu(x, "x")
    _on_gpu(w, "w", x)
    if w.dim() != 2 or x.dim() == 0 or x.shape[-1] != w.shape[1]:
        raise ValueError(f"x [..., cols] and w [units, cols] are needed, got {tuple(x.shape)} and {tuple(w.shape)}")
    if w.numel() == 0:
        raise ValueError(f"w must have units and columns, got {tuple(w.shape)}")
    if x.dtype != w.dtype:
        raise TypeError(f"x and w must have one dtype, got {x.dtype} and {w.dtype}")


def _bias(bias: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    _on_gpu(bias, "bias", w)
    if bias.dtype not in (torch.float32, w.dtype) or bias.dim() != 1 or bias.shape[0] != w.shape[0]:
        raise ValueError(f"bias must be a float32 or {w.dtype} tensor of shape {(w.shape[0],)}, got {bias.dtype} {tuple(bias.shape)}")
    return bias if bias.is_contiguous() else bias.contiguous()


def _layer(x, w, bias, activation, residual, p, seed, step, dtype, out, pre, stream):
    # one token's layer takes less time on the GPU (7 us for 4096 x 4096) than this
    # call takes to issue, so only what is there is looked at
    _factors(x, w)
    epilogue = binding.Epilogue()
    if activation is not None:
        epilogue.activation = _activation(activation)
    shape = (*x.shape[:-1], w.shape[0])
    if dtype is None:
        dtype = x.dtype if out is None else out.dtype
    if dtype != x.dtype and dtype != torch.float32:
        raise TypeError(f"dtype must be float32 or x's {x.dtype}, got {dtype}")
    if bias is not None:
        bias = _bias(bias, w)
        epilogue.bias, epilogue.bias_dtype = bias.data_ptr(), _CODES[bias.dtype]
    if residual is not None:
        _beside(residual, shape, dtype, x, "residual")
    if pre is not None:
        _out(pre, shape, x.dtype, x, "pre")
    if p or step is not None:
        mask = _mask(p, seed, step, x)
        epilogue.dropout = ctypes.addressof(mask)
    out = _out(out, shape, dtype, x)
    if x.numel() == 0:
        return out
    a, of_x = _operand(x, "x")
    b, of_w = _operand(w, "w")
    if residual is not None:
        residual, of_residual = _operand(residual, "residual")
        epilogue.residual = ctypes.addressof(of_residual)
    if pre is not None:
        of_pre = _operand(pre, "pre")[1]
        epilogue.pre = ctypes.addressof(of_pre)
    size = lib.sqn_layer_workspace(of_x, of_w)
    work = _workspace(size, x)
    _check(lib.sqn_layer(of_x, of_w, epilogue, _operand(out, "out")[1], _ptr(work), size,
                         _on(stream, a, b, bias, residual, pre, step, out, work)))
    return out


class _Layer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, residual, step, activation, p, seed, dtype):
        plain = [None if t is None else t.detach() for t in (x, w, bias, residual)]
        pre = None
        if activation is not None and any(ctx.needs_input_grad[:3]):
            _factors(x, w)
            pre = _out(None, (*x.shape[:-1], w.shape[0]), x.dtype, plain[0])
        ctx.save_for_backward(x, w, pre, step)
        ctx.options = activation, p, seed
        ctx.bias = None if bias is None else bias.dtype
        ctx.residual = None if residual is None else residual.dtype
        return _layer(*plain[:3], activation, plain[3], p, seed, step, dtype, None, pre, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, w, pre, step = ctx.saved_tensors
        activation, p, seed = ctx.options
        for_x, for_w, for_bias, for_residual = ctx.needs_input_grad[:4]
        grads = (None, None, None)
        if for_x or for_w or for_bias:
            grads = layer_gradient(grad, x, w, pre, activation, p, seed, step, for_x=for_x, for_w=for_w,
                                   for_bias=for_bias, bias_dtype=ctx.bias or torch.float32)
        return (*grads, grad if for_residual else None, None, None, None, None, None)


def layer(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: Optional[str] = None,
          residual: Optional[torch.Tensor] = None, dropout: float = 0.0, seed: int = 0,
          step: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None,
          out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """sqn_layer: D(act(x w^T + bias)) + residual, [..., units], of x [..., cols]
    and w [units, cols] (one dtype), bias [units] (float32 or theirs), residual
    [..., units] of the result's dtype, which is x's or float32.  `activation`
    is None, "relu", "gelu" (with the normal distribution itself) or "silu"; D
    is the mask of `dropout`(..., p=dropout, seed=seed, step=step).  Sums and the
    epilogue are float32, rounded once.  Differentiable in x, w, bias and
    residual (without `out`, `pre` and `stream`), by layer_gradient, which takes
    what `pre` holds: x w^T + bias in x's dtype.  `out` may be the residual; else
    `out` and `pre` share no memory with each other and the inputs.  No
    forward-mode derivative."""
    p = _probability(dropout) if dropout else 0.0
    _no_tangent("layer", x, w, bias, residual)
    if out is None and pre is None and stream is None and _wants_gradient(x, w, bias, residual):
        return _Layer.apply(x, w, bias, residual, step, activation, p, int(seed), dtype)
    return _layer(x, w, bias, activation, residual, p, seed, step, dtype, out, pre, stream)


def layer_gradient(grad: torch.Tensor, x: torch.Tensor, w: torch.Tensor, pre: Optional[torch.Tensor] = None,
                   activation: Optional[str] = None, dropout: float = 0.0, seed: int = 0,
                   step: Optional[torch.Tensor] = None, for_x: bool = True, for_w: bool = True, for_bias: bool = True,
                   bias_dtype: torch.dtype = torch.float32, stream=None):
    """sqn_layer_gradient: the gradients (of x, of w, of the bias) of layer from
    grad [..., units], that of its result (x's dtype or float32); None where one
    is not wanted.  `pre` is what layer wrote there, needed with an activation
    and only then; the residual's gradient is grad.  No gradient passes through
    it."""
    p = _probability(dropout) if dropout else 0.0
    _no_tangent("layer_gradient", grad, x, w, pre)
    _factors(x, w)
    act = _activation(activation)
    shape = (*x.shape[:-1], w.shape[0])
    _on_gpu(grad, "grad", x)
    if grad.shape != shape or (grad.dtype != x.dtype and grad.dtype != torch.float32):
        raise ValueError(f"grad must be a float32 or {x.dtype} tensor of shape {shape}, got {grad.dtype} {tuple(grad.shape)}")
    if (pre is None) != (act == 0):
        raise ValueError("pre goes with an activation, and an activation needs it")
    if pre is not None:
        _beside(pre, shape, x.dtype, x, "pre")
    if bias_dtype != torch.float32 and bias_dtype != x.dtype:
        raise TypeError(f"bias_dtype must be float32 or x's {x.dtype}, got {bias_dtype}")
    mask = _mask(p, seed, step, x) if p or step is not None else None
    grad_x = _out_like(x) if for_x else None
    grad_w = _out_like(w) if for_w else None
    grad_bias = _out(None, (w.shape[0],), bias_dtype, x) if for_bias else None
    g, of_g = _operand(grad, "grad")
    a, of_x = _operand(x, "x")
    b, of_w = _operand(w, "w")
    of_pre = None
    if pre is not None:
        pre, of_pre = _operand(pre, "pre")
    size = lib.sqn_layer_gradient_workspace(of_g, of_x, of_w, act, mask, for_x, for_w, for_bias)
    work = _workspace(size, x)
    _check(lib.sqn_layer_gradient(of_g, of_x, of_w, of_pre, act, mask, _operand(grad_x, "grad_x")[1] if for_x else None,
                                  _operand(grad_w, "grad_w")[1] if for_w else None, _ptr(grad_bias), _CODES[bias_dtype],
                                  _ptr(work), size, _on(stream, g, a, b, pre, step, grad_x, grad_w, grad_bias, work)))
    return grad_x, grad_w, grad_bias
