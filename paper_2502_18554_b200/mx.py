"""Microscaled 4-bit floating point (MXFP4: E2M1 elements, one power of two for 32 of them): the fixed-rate sibling of the
error-bounded codec, for the operands of products.  Format, rounding and errors are those of ``zccl_mx4_*`` in
``include/zccl.h``; like them, every call only enqueues on the stream (the current one of the tensors' device unless
``stream`` names another), and there is no CPU fallback.
"""
from __future__ import annotations

import contextlib
from typing import NamedTuple

import torch

from . import zccl as z


class Mx4(NamedTuple):
    """A matrix [rows, cols] in microscaled form: `codes` (uint8, code_bytes) and `scales` (uint8, scale_bytes), any shape, laid out as
    ``include/zccl.h`` says (zeros behind the last row and block of the scales)."""

    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int


def code_bytes(rows: int, cols: int) -> int:
    return int(z.lib().zccl_mx4_code_bytes(rows, cols))


def scale_bytes(rows: int, cols: int) -> int:
    return int(z.lib().zccl_mx4_scale_bytes(rows, cols))


def _allocating(stream):
    """Outputs of a call on `stream` are that stream's memory, so that it is not handed out again while the call runs."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def empty(rows: int, cols: int, device, stream=None) -> Mx4:
    """Memory for a matrix [rows, cols] in microscaled form."""
    codes, scales = z.native().mx4_sizes(rows, cols)
    with _allocating(stream):
        return Mx4(torch.empty(codes, dtype=torch.uint8, device=device), torch.empty(scales, dtype=torch.uint8, device=device), rows, cols)


def _value(r, what: str):
    """What a native call returned: its result, or a status to raise."""
    if type(r) is int:
        z._check(r, what)
    return r


def quantize(x: torch.Tensor, transpose: bool = False, out: Mx4 | None = None, stream=None) -> Mx4:
    """x (float32, bfloat16 or float16 [rows, cols], rows contiguous) in microscaled form, blocks along its rows; with
    `transpose` the form of x's transpose, blocks along x's columns."""
    if out is None:
        return Mx4._make(_value(z.native().mx4_quantize(x, transpose, None, None, stream), "zccl_mx4_quantize"))
    rows, cols = reversed(x.shape) if transpose else x.shape
    if (out.rows, out.cols) != (rows, cols):
        raise ValueError(f"expected the form of a matrix [{rows}, {cols}], got one of [{out.rows}, {out.cols}]")
    _value(z.native().mx4_quantize(x, transpose, out.codes, out.scales, stream), "zccl_mx4_quantize")
    return out


def quantize_all(matrices, transpose=None, stream=None) -> list[Mx4]:
    """quantize of several matrices of one type, in as few launches as they fit; `transpose`: whether, for each (default: none)."""
    matrices = list(matrices)
    transpose = [False] * len(matrices) if transpose is None else list(transpose)
    forms = _value(z.native().mx4_quantize_all(matrices, transpose, stream), "zccl_mx4_quantize_all")
    return [Mx4(codes, scales, *(reversed(x.shape) if t else x.shape)) for (codes, scales), x, t in zip(forms, matrices, transpose)]


def dequantize(q: Mx4, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The values of `q`, each rounded once to `dtype` (or to the type of `out`)."""
    return _value(z.native().mx4_dequantize(q.codes, q.scales, q.rows, q.cols, dtype, out, stream), "zccl_mx4_dequantize")


def matmul(a: Mx4, b: Mx4, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """A B^T of two operands that are quantised along the contraction: a [m, k] and b [n, k] to [m, n], sums in binary32, each
    rounded once to `dtype` (float32, bfloat16 or float16), or to the type of `out`."""
    if a.cols != b.cols:
        raise ValueError(f"operands are contracted over {a.cols} and {b.cols} elements")
    return _value(z.native().mx4_matmul(a.codes, a.scales, a.rows, b.codes, b.scales, b.rows, a.cols, dtype, out, stream), "zccl_mx4_matmul")


def status(stream=None) -> int:
    """zccl_mx4_status of the current device: waits for `stream`; z.OK, or z.E_TIMEOUT where a wait inside a product has run out since it was last asked.  Until
    it is asked, products and layers on that device raise ZcclError with that code."""
    return int(z.lib().zccl_mx4_status(z._stream_ptr(stream)))


def debug_wait(stream=None) -> None:
    """Test hook: a wait that runs out (zccl_debug_mx4_wait)."""
    z._check(z.lib().zccl_debug_mx4_wait(z._stream_ptr(stream)), "zccl_debug_mx4_wait")


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return _value(z.native().mx4_linear(x, w), "zccl_mx4_matmul")

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        return linear_backward(dy.contiguous(), x, w, ctx.needs_input_grad)


def linear(x: torch.Tensor, w: torch.Tensor | Mx4) -> torch.Tensor:
    """x W^T with both sides in microscaled form, in x's type, on the current stream.  x is [..., k], rows contiguous; `w` is [n, k] of x's type, or already
    quantised (weights that are laid out once; no gradient then).  With a tensor for `w` this is differentiable, by linear_backward, once and backwards: tensors with
    a forward-mode tangent are refused."""
    rows = x if x.dim() == 2 else x.reshape(x.shape[:-1].numel(), x.shape[-1])
    if isinstance(w, Mx4):
        if x.requires_grad and torch.is_grad_enabled():
            raise ValueError("quantised weights are for inference: pass the weights themselves to train, or detach x")
        if w.cols != rows.shape[1]:
            raise ValueError(f"x has rows of {rows.shape[1]}, the weights of {w.cols}")
        y = _value(z.native().mx4_linear(rows, w.codes, w.scales, w.rows), "zccl_mx4_matmul")
    elif torch.is_grad_enabled() and (x.requires_grad or w.requires_grad):
        y = _Linear.apply(rows, w)
    else:
        y = _value(z.native().mx4_linear(rows, w), "zccl_mx4_matmul")
    return y if x.dim() == 2 else y.view(*x.shape[:-1], y.shape[-1])


def linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, needed=(True, True)):
    """The gradients of linear(x, w) for matrices, from dy [m, n]: dx = Q(dy) Q(w^T)^T, contracted and quantised along n, and
    dw = Q(dy^T) Q(x^T)^T along m, each in its operand's type (quantisation itself passes gradients on unchanged)."""
    return _value(z.native().mx4_linear_backward(dy, x, w, needed[0], needed[1]), "zccl_mx4_matmul")
