"""What a data-parallel program does with the gradient that the ring has reduced: the norm over all tensors and the AdamW
step over all of them at once, states in 32 or in 8 bits (``zccl_grad_norm`` and ``zccl_adamw`` in ``include/zccl.h``, which
state the arithmetic).  Calls only enqueue on the stream; there is no CPU fallback.
"""
from __future__ import annotations

import torch

from . import zccl as z
from .mx import _value


def grad_norm(grads, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """sqrt(sum of g^2) over all of `grads` (CUDA tensors of one type), as a float32 [1] on their device."""
    return _value(z.native().grad_norm(grads, out, stream), "zccl_grad_norm")


def adamw(params, grads, exp_avg, exp_avg_sq, exp_avg_scale=None, exp_avg_sq_scale=None, *, step, lr, betas=(0.9, 0.999), eps=1e-8,
          weight_decay=0.01, copies=None, norm=None, max_norm=1.0, seed=0, stream=None) -> None:
    """One step over lists of contiguous CUDA tensors, in place.

    States in 32 bits are float32 tensors of the parameters' sizes.  In 8 bits `exp_avg` and `exp_avg_sq` are float8_e4m3fn (the
    latter holding the ROOT of the second moment) with a uint8 scale per 32 elements in `exp_avg_scale` and `exp_avg_sq_scale`.
    `copies` (float32 parameters only): bfloat16 or float16 tensors that receive the new parameters.  `step` (from 1 on) and `lr` are numbers, or an
    int64 and a float32 CUDA tensor of one element that are read when the call runs, which a captured call needs.  With `norm` (see
    grad_norm) gradients are scaled to `max_norm` at most, and a norm that is not finite leaves everything as it was."""
    z._check(z.native().adamw(params, grads, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale, copies, lr, betas[0], betas[1], eps,
                              weight_decay, step, seed, norm, max_norm, stream), "zccl_adamw")
