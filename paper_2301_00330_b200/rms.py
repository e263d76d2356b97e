"""Root-mean-square norm of a residual sum, on the library's kernels (include/gf_block.h).

`rms_norm` adds a residual (and drops elements of the branch that is added to it) in the pass that norms the sum.
Only marshalling happens here.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .dropout import _check_p, _seed_for
from .norm import _dense


def _check_args(x, weight, residual, what: str):
    if not x.is_cuda or any(t is not None and not t.is_cuda for t in (weight, residual)):
        raise RuntimeError(f"{what} needs CUDA tensors: there is no CPU path")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x has rows of at least one value")
    B._dt(x.dtype)
    for t in (weight, residual):
        if t is not None:
            B._dt(t.dtype)
            if t.device != x.device:
                raise ValueError(f"all tensors lie on the device of x, {x.device}, got {t.device}")
    if weight is not None and weight.shape != x.shape[-1:]:
        raise ValueError(f"weight has the shape ({x.shape[-1]},), got {tuple(weight.shape)}")
    if residual is not None:
        if residual.shape != x.shape:
            raise ValueError(f"residual has the shape of x, {tuple(x.shape)}, got {tuple(residual.shape)}")
        if x.dtype == torch.float32 and residual.dtype != torch.float32:
            raise TypeError("a float32 x needs a float32 residual")


def _norm_desc(x, weight, residual, eps: float, p: float):
    C = x.shape[-1]
    return B.make_rms_desc(x.numel() // C, C, dtype=x.dtype, residual_dtype=x.dtype if residual is None else residual.dtype,
                           param_dtype=torch.float32 if weight is None else weight.dtype, eps=eps, p=p)


def _norm_backward(desc, g_y, g_h, h, rstd, weight, seed, need_x: bool, need_w: bool, need_res: bool, x_dtype):
    """(g_x, g_weight, g_residual) as the library gives them; those not needed are None."""
    dev = h.device
    with torch.cuda.device(dev):
        g_res = g_x = None
        if need_res or (need_x and seed is None and desc.dtype == desc.residual_dtype):
            g_res = torch.empty_like(h)
        if need_x and not (seed is None and desc.dtype == desc.residual_dtype):
            g_x = torch.empty(h.shape, dtype=x_dtype, device=dev)
        g_w = torch.empty(desc.cols, dtype=torch.float32, device=dev) if need_w else None
        ws = torch.empty(B.gf_rms_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device=dev)
        B.gf_rms_norm_backward(desc, _dense(g_y), None if g_h is None else _dense(g_h), h, rstd, weight, seed, g_res, g_x, g_w, ws, None,
                               torch.cuda.current_stream(dev))
    if need_x and g_x is None:
        g_x = g_res
    return g_x, None if g_w is None else g_w if weight.dtype == torch.float32 else g_w.to(weight.dtype), g_res if need_res else None


class _RmsNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, seed, eps: float, p: float):
        ctx.set_materialize_grads(False)
        desc = _norm_desc(x, weight, residual, eps, p)
        x = _dense(x)
        weight = None if weight is None else _dense(weight)
        residual = None if residual is None else _dense(residual)
        y = torch.empty_like(x)
        plain = residual is None and seed is None
        h = None if plain else torch.empty_like(x if residual is None else residual)
        rstd = torch.empty(max(desc.rows, 1), dtype=torch.float32, device=x.device)
        with torch.cuda.device(x.device):
            B.gf_rms_norm_forward(desc, x, residual, seed, weight, h, y, rstd, torch.cuda.current_stream(x.device))
        ctx.desc, ctx.x_dtype = desc, x.dtype
        ctx.save_for_backward(x if plain else h, rstd, weight, seed)
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, g_y, g_h):
        h, rstd, weight, seed = ctx.saved_tensors
        need_x, need_w, need_res = ctx.needs_input_grad[:3]
        if g_y is None:
            g_y = torch.zeros(h.shape, dtype=ctx.x_dtype, device=h.device)
        g_x, g_w, g_res = _norm_backward(ctx.desc, g_y, g_h, h, rstd, weight, seed, need_x, need_w, need_res, ctx.x_dtype)
        return g_x, g_w, g_res, None, None, None


def rms_norm(x: torch.Tensor, weight: torch.Tensor | None = None, eps: float = 1e-5, residual: torch.Tensor | None = None,
             p: float = 0.0, training: bool = True, seed: torch.Tensor | None = None):
    """Root-mean-square norm over the last dimension: y = h weight / sqrt(mean(h^2) + eps).

    Without a residual h = x and y is returned.  With one, h = residual + dropout(x, p) (gf.dropout's, of the same seed) is
    formed in the same pass, and (y, h) is returned: h is the residual of what follows.  x is float32 or
    bfloat16, as is y; a bfloat16 x may have a float32 residual, which h then is too.  Gradients come back in the
    dtypes of their tensors (the sum over rows is fp32)."""
    _check_args(x, weight, residual, "rms_norm")
    p = _check_p(p) if training else 0.0
    if residual is None and p > 0:
        raise ValueError("p > 0 drops elements of a branch that is added to a residual: there is none")
    y, h = _RmsNormFn.apply(x, weight, residual, _seed_for(x, p, seed), float(eps), p)
    return y if residual is None else (y, h)


class RMSNorm(torch.nn.Module):
    """Root-mean-square norm over the last dimension; forward(x, residual) gives (y, h) with h = residual + dropout(x, p)."""

    def __init__(self, channels: int, eps: float = 1e-5, p: float = 0.0, device=None, dtype=None):
        super().__init__()
        self.eps, self.p = eps, _check_p(p)
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device, dtype=dtype))

    def forward(self, x, residual=None):
        if residual is None:
            return rms_norm(x, self.weight, self.eps)
        return rms_norm(x, self.weight, self.eps, residual, self.p, self.training)
