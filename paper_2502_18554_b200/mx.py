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
    """A matrix [rows, cols] in microscaled form: `codes` (uint8, code_bytes) and `scales` (uint8, scale_bytes), any shape."""

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


def quantize(x: torch.Tensor, transpose: bool = False, out: Mx4 | None = None, stream=None) -> Mx4:
    """x (float32, bfloat16 or float16 [rows, cols], rows contiguous) in microscaled form, blocks along its rows; with
    `transpose` the form of x's transpose, blocks along x's columns."""
    if x.dim() != 2:
        raise ValueError("expected a matrix")
    rows, cols = (x.shape[1], x.shape[0]) if transpose else (x.shape[0], x.shape[1])
    if out is None:
        out = empty(rows, cols, x.device, stream)
    elif (out.rows, out.cols) != (rows, cols):
        raise ValueError(f"expected the form of a matrix [{rows}, {cols}], got one of [{out.rows}, {out.cols}]")
    z._check(z.native().mx4_quantize(x, transpose, out.codes, out.scales, stream), "zccl_mx4_quantize")
    return out


def dequantize(q: Mx4, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The values of `q`, each rounded once to `dtype`."""
    if out is None:
        with _allocating(stream):
            out = torch.empty(q.rows, q.cols, dtype=dtype, device=q.codes.device)
    elif tuple(out.shape) != (q.rows, q.cols):
        raise ValueError(f"expected an output [{q.rows}, {q.cols}], got {list(out.shape)}")
    z._check(z.native().mx4_dequantize(q.codes, q.scales, out, stream), "zccl_mx4_dequantize")
    return out


def matmul(a: Mx4, b: Mx4, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """A B^T of two operands that are quantised along the contraction: a [m, k] and b [n, k] to [m, n], sums in binary32, each
    rounded once to `dtype` (float32, bfloat16 or float16)."""
    if a.cols != b.cols:
        raise ValueError(f"operands are contracted over {a.cols} and {b.cols} elements")
    if out is None:
        with _allocating(stream):
            out = torch.empty(a.rows, b.rows, dtype=dtype, device=a.codes.device)
    elif tuple(out.shape) != (a.rows, b.rows):
        raise ValueError(f"expected an output [{a.rows}, {b.rows}], got {list(out.shape)}")
    z._check(z.native().mx4_matmul(a.codes, a.scales, b.codes, b.scales, a.cols, out, stream), "zccl_mx4_matmul")
    return out


def status(stream=None) -> int:
    """zccl_mx4_status of the current device: waits for `stream`; z.OK or z.E_TIMEOUT."""
    return int(z.lib().zccl_mx4_status(z._stream_ptr(stream)))


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return matmul(quantize(x), quantize(w), x.dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        return linear_backward(dy.contiguous(), x, w, ctx.needs_input_grad)


def linear(x: torch.Tensor, w: torch.Tensor | Mx4) -> torch.Tensor:
    """x W^T with both sides in microscaled form, in x's type.  x is [..., k]; `w` is [n, k], or already quantised (weights that
    are laid out once; no gradient then).  With a tensor for `w` this is differentiable, by linear_backward."""
    rows = x.reshape(-1, x.shape[-1])
    if isinstance(w, Mx4):
        if torch.is_grad_enabled() and x.requires_grad:
            raise ValueError("quantised weights are for inference: pass the weights themselves to train, or detach x")
        y = matmul(quantize(rows), w, x.dtype)
    else:
        if w.dtype != x.dtype:
            raise ValueError(f"x is {x.dtype}, the weights are {w.dtype}")
        y = _Linear.apply(rows, w)
    return y.view(*x.shape[:-1], y.shape[-1])


def linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, needed=(True, True)):
    """The gradients of linear(x, w) for matrices, from dy [m, n]: dx = Q(dy) Q(w^T)^T, contracted and quantised along n, and
    dw = Q(dy^T) Q(x^T)^T along m, each in its operand's type (quantisation itself passes gradients on unchanged)."""
    dx = matmul(quantize(dy), quantize(w, transpose=True), x.dtype) if needed[0] else None
    dw = matmul(quantize(dy, transpose=True), quantize(x, transpose=True), w.dtype) if needed[1] else None
    return dx, dw
