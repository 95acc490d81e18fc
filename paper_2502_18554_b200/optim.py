"""What a data-parallel program does with the gradient that the ring has reduced: the norm over all tensors and the AdamW
step over all of them at once, states in 32 or in 8 bits (``zccl_grad_norm`` and ``zccl_adamw`` in ``include/zccl.h``, which
state the arithmetic).  Calls only enqueue on the stream, but for an exchange, which waits; there is no CPU fallback.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import zccl as z
from .mx import _value
from .ring import DegenerateRange

BLOCK = 32


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


def exchange(ring, grads, eb_mode: int, eb: float) -> list[torch.Tensor]:
    """The gradients' average over the ranks of `ring` (a `ring.Ring` for at least exchange_elems(grads) elements), compressed on the way: one Allreduce of all of
    them, as float32, in which every rank ends with the same values (ZCCL_CONSISTENT_OWNER).  Returns tensors of the gradients' shapes, views of one array in which
    each begins at a multiple of 32 elements; the gaps hold zeros, which count into the range that a relative bound refers to.

    The codec takes finite values only, so the ranks agree on the smallest and largest value of all gradients first (the host waits for it).  Where a gradient of any
    rank is not finite, what is returned is NaN throughout, on every rank.  Where all values of all ranks are the same number, that is returned as it is.  An exchange that a rank has to
    refuse (values beyond 2^30 steps of the bound, a range that is not finite) raises on every rank."""
    return _exchange(ring, list(grads), eb_mode, eb)[0]


def exchange_elems(grads) -> int:
    """Elements of the array that `exchange` sends: what its ring has to be made for."""
    return sum(-(-g.numel() // BLOCK) * BLOCK for g in grads)


@torch.no_grad()
def _exchange(ring, grads: list, eb_mode: int, eb: float):
    """(exchange's tensors, whether all gradients of all ranks are finite)."""
    at, spans = 0, []
    for g in grads:
        spans.append((at, g.numel()))
        at += -(-g.numel() // BLOCK) * BLOCK
    views = lambda t: [t[o:o + n].view(g.shape) for (o, n), g in zip(spans, grads)]  # noqa: E731
    flat = torch.zeros(at, dtype=torch.float32, device=ring.codec.device)
    if at == 0:
        return views(flat), True
    torch._foreach_copy_(views(flat), grads)
    # what is not finite on any rank ends as infinity: a maximum over the ranks could drop a NaN
    low, high = torch.aminmax(flat)
    ends = torch.where(torch.isfinite(low) & torch.isfinite(high), torch.stack([-low, high]), float("inf"))
    if ring.N > 1:
        ends = ring.link.all_max(ends)
    low, high = ends.tolist()
    low = -low
    if not math.isfinite(low):
        return views(flat.fill_(float("nan"))), False
    bound = _bound(low, high, eb_mode, eb, ring.N)
    if bound is None:
        return views(flat), True
    reduced, failed = torch.empty_like(flat), None
    try:
        ring.allreduce(flat, reduced, z.EB_ABS, bound, flags=z.OP_AVG | z.CONSISTENT_OWNER)
    except (z.ZcclError, DegenerateRange) as exc:
        failed = exc
    if ring.N > 1:      # a rank's codec tells it alone of what has gone wrong there
        worst = int(ring.link.all_max(torch.tensor([-getattr(failed, "code", z.E_DEGENERATE) if failed else 0], dtype=torch.int32)).item())
        if worst and not failed:
            failed = z.ZcclError(-worst, "exchange, on another rank")
    if failed:
        raise failed
    return views(reduced), True


def _bound(low: float, high: float, eb_mode: int, eb: float, ranks: int) -> float | None:
    """The absolute bound for values from `low` to `high` on all ranks; None where there is nothing to compress.  Refuses what the codec would refuse on the rank that
    has the largest value, with the codec's arithmetic."""
    if not (eb > 0) or not math.isfinite(eb):
        raise ValueError("the error bound must be a positive finite number")
    f32 = np.float32
    if eb_mode == z.EB_ABS:
        bound = f32(eb)
        with np.errstate(all="ignore"):
            reciprocal = f32(1) / (bound * f32(0.984375) * f32(2))
    elif eb_mode == z.EB_REL:
        if low == high:
            return None
        rc, bound, _, reciprocal = z.resolve_range_host(low, high, float(f32(eb)))
        if rc != z.OK:
            raise DegenerateRange("relative bound over gradients whose range is too small or not finite")
    else:
        raise ValueError("eb_mode")
    with np.errstate(all="ignore"):
        if ranks > 1 and not f32(max(-low, high)) * f32(reciprocal) < f32(2.0 ** 30):
            raise z.ZcclError(z.E_RANGE, "exchange")
    return float(bound)


class AdamW:
    """AdamW over the contiguous CUDA tensors `params` (all of one type), with its states in 32 or 8 bits.

    step() takes the gradients from the parameters' `.grad`, or those it is given; `exchange` makes the ranks of a data-parallel job
    agree on them first.  `copies` receive the new parameters as in adamw()."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, state_bits: int = 32, copies=None, seed: int = 0):
        if state_bits not in (32, 8):
            raise ValueError("state_bits is 32 or 8")
        self.params, self.copies = list(params), None if copies is None else list(copies)
        self.lr, self.betas, self.eps, self.weight_decay, self.seed = lr, betas, eps, weight_decay, seed
        self.steps = 0
        dtype = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        state = lambda: [torch.zeros(p.shape, dtype=dtype, device=p.device) for p in self.params]  # noqa: E731
        scale = lambda: [torch.zeros(-(-p.numel() // BLOCK), dtype=torch.uint8, device=p.device) for p in self.params]  # noqa: E731
        self.exp_avg, self.exp_avg_sq = state(), state()
        self.exp_avg_scale, self.exp_avg_sq_scale = (scale(), scale()) if state_bits == 8 else (None, None)

    def step(self, grads=None, max_norm: float | None = None, ring=None, eb_mode: int = z.EB_REL, eb: float = 1e-3, stream=None) -> torch.Tensor | None:
        """One step.  `ring`: exchange the gradients over its ranks first, with this error bound (then on the current stream).  `max_norm`: scale them to
        that norm at most; returns the norm (float32 [1], on the device).  A step whose norm is not finite changes nothing but `steps`; nor does one whose
        gradients are not finite on some rank of `ring`, on any of its ranks, with `max_norm` or without."""
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        if any(g is None for g in grads):
            raise ValueError("every parameter needs a gradient")
        if ring is not None:
            if stream is not None:
                raise ValueError("an exchange runs on the current stream")
            grads, finite = _exchange(ring, grads, eb_mode, eb)
            if not finite:
                self.steps += 1
                return None if max_norm is None else torch.full((1,), float("nan"), device=ring.codec.device)
        norm = None if max_norm is None else grad_norm(grads, stream=stream)
        adamw(self.params, grads, self.exp_avg, self.exp_avg_sq, self.exp_avg_scale, self.exp_avg_sq_scale, step=self.steps + 1, lr=self.lr, betas=self.betas, eps=self.eps,
              weight_decay=self.weight_decay, copies=self.copies, norm=norm, max_norm=1.0 if max_norm is None else max_norm, seed=self.seed, stream=stream)
        self.steps += 1     # not before: a step that is refused has not been
        return norm

    def state_dict(self) -> dict:
        """Steps so far, the seed of the roundings and the states (the tensors themselves)."""
        return {"steps": self.steps, "seed": self.seed, "exp_avg": self.exp_avg, "exp_avg_sq": self.exp_avg_sq, "exp_avg_scale": self.exp_avg_scale, "exp_avg_sq_scale": self.exp_avg_sq_scale}

    def load_state_dict(self, state: dict) -> None:
        """Takes over what state_dict gave, the seed included (where there is none in it, this optimizer's stays): the steps that follow are those that would have followed there."""
        steps, seed = state["steps"], state.get("seed", self.seed)
        for key in ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"):
            mine, theirs = getattr(self, key), state[key]
            if (mine is None) != (theirs is None) or (mine is not None and [(t.shape, t.dtype) for t in mine] != [(t.shape, t.dtype) for t in theirs]):
                raise ValueError(f"{key} does not fit these parameters and this state_bits")
        for key in ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"):
            for m, t in zip(getattr(self, key) or (), state[key] or ()):
                m.copy_(t)
        self.steps, self.seed = steps, seed
