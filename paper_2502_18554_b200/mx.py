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
