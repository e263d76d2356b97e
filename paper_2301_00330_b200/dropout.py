"""Dropout whose mask is never stored, on the library's kernels (include/gf_block.h).

The mask is a function of two 64-bit words and the element's index, computed again in the backward pass: what is kept
for it are 16 bytes, whatever the tensor's size.  Only marshalling happens here.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .norm import _dense


def dropout_seed(device) -> torch.Tensor:
    """Two random 64-bit words from torch's generator of `device`: they follow torch.manual_seed, and are drawn anew by every
    replay of a captured graph."""
    return torch.randint(-(1 << 63), (1 << 63) - 1, (2,), dtype=torch.int64, device=device)


def _check_p(p: float) -> float:
    p = float(p)
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"the probability of dropping lies in 0 .. 1, got {p}")
    return p


def _seed_for(x: torch.Tensor, p: float, seed):
    """The words to use, checked, or None where nothing is dropped (p is taken to a multiple of 2^-16)."""
    if round(p * 65536.0) == 0:
        return None
    if seed is None:
        return dropout_seed(x.device)
    if seed.dtype != torch.int64 or seed.numel() != 2 or seed.device != x.device:
        raise ValueError("seed has two int64 values on the device of x")
    return seed.contiguous()


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, seed, p: float):
        ctx.in_dtype, ctx.p = x.dtype, p
        out_dtype = x.dtype if residual is None else residual.dtype
        fmt = torch.contiguous_format
        if not x.is_contiguous() and x.dim() == 4 and x.is_contiguous(memory_format=torch.channels_last):
            fmt = torch.channels_last            # the index of an element is its place in memory
        ctx.fmt = fmt
        x = _dense(x, fmt)
        y = torch.empty_like(x, dtype=out_dtype, memory_format=fmt)
        desc = B.make_dropout_desc(x.numel(), dtype=x.dtype, out_dtype=out_dtype, p=p)
        with torch.cuda.device(x.device):
            B.gf_dropout_forward(desc, x, None if residual is None else _dense(residual, fmt), seed, y,
                                 torch.cuda.current_stream(x.device))
        ctx.desc = desc
        ctx.save_for_backward(seed)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, g_y):
        g_x = None
        if ctx.needs_input_grad[0]:
            g = _dense(g_y, ctx.fmt)
            g_x = torch.empty_like(g, dtype=ctx.in_dtype, memory_format=ctx.fmt)
            with torch.cuda.device(g.device):
                B.gf_dropout_backward(ctx.desc, g, ctx.saved_tensors[0], g_x, torch.cuda.current_stream(g.device))
        return g_x, g_y if ctx.needs_input_grad[1] else None, None, None


def dropout(x: torch.Tensor, p: float = 0.5, training: bool = True, residual: torch.Tensor | None = None,
            seed: torch.Tensor | None = None) -> torch.Tensor:
    """residual + dropout(x) (residual None: dropout(x)), in one pass.

    x and residual are float32 or bfloat16 of one shape; the result has the residual's dtype.  Each element of x
    is dropped with probability p (rounded to a multiple of 2^-16) and scaled by 1 / (1 - p) otherwise; with training
    false nothing is.  seed: two int64 words on x's device that the mask follows from (dropout_seed); None: new
    ones.  A map in torch's channels_last memory format keeps it, and its elements count in memory order."""
    p = _check_p(p)
    if not x.is_cuda or (residual is not None and not residual.is_cuda):
        raise RuntimeError("dropout needs CUDA tensors: there is no CPU path")
    B._dt(x.dtype)
    if residual is not None:
        B._dt(residual.dtype)
        if residual.shape != x.shape or residual.device != x.device:
            raise ValueError(f"residual has the shape and device of x, {tuple(x.shape)} on {x.device}")
    if not training:
        p = 0.0
    if p == 0.0 and residual is None:
        return x
    return _DropoutFn.apply(x, residual, _seed_for(x, p, seed), p)


class Dropout(torch.nn.Module):
    """dropout(x, p) while training; forward(x, residual) adds the residual in the same pass."""

    def __init__(self, p: float = 0.5):
        super().__init__()
        self.p = _check_p(p)

    def forward(self, x, residual=None):
        return dropout(x, self.p, self.training, residual)

    def extra_repr(self):
        return f"p={self.p}"
