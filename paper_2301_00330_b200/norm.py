"""Layer normalisation over the channels, with its backward pass, on the library's kernels (include/gf_train.h).

`layer_norm` takes rows (channels last in memory) and feature maps with the channels in dimension 1;
a map in torch's channels_last memory format takes the row kernels, as its memory is rows of
channels.  Only marshalling happens here.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


def _dense(t: torch.Tensor, fmt=torch.contiguous_format) -> torch.Tensor:
    """Dense and on a 16-byte boundary (a view may be neither)."""
    t = t.contiguous(memory_format=fmt)
    return t if t.data_ptr() % 16 == 0 else t.clone(memory_format=fmt)


class _LayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps: float, channel_dim: int):
        if not x.is_cuda or any(p is not None and not p.is_cuda for p in (weight, bias)):
            raise RuntimeError("layer_norm needs CUDA tensors: there is no CPU path")
        C = x.shape[channel_dim]
        for p in (weight, bias):
            if p is not None and p.device != x.device:
                raise ValueError(f"weight and bias lie on the device of x, {x.device}, got {p.device}")
            if p is not None and p.shape != (C,):
                raise ValueError(f"weight and bias have the shape ({C},), got {tuple(p.shape)}")
        if weight is not None and bias is not None and weight.dtype != bias.dtype:
            raise TypeError("weight and bias have one dtype")
        fmt = torch.contiguous_format
        if channel_dim == 1:
            N, _, H, W = x.shape
            layout = B.GF_NCHW
            if not x.is_contiguous() and x.is_contiguous(memory_format=torch.channels_last):
                fmt, layout = torch.channels_last, B.GF_NHWC
        else:
            N, H, W, layout = x.numel() // max(C, 1), 1, 1, B.GF_NHWC
        param = weight if weight is not None else bias
        ctx.had_grad = x.requires_grad, weight is not None and weight.requires_grad, bias is not None and bias.requires_grad
        x = _dense(x, fmt)
        weight = None if weight is None else _dense(weight)
        bias = None if bias is None else _dense(bias)
        y = torch.empty_like(x, memory_format=fmt)
        if x.numel() == 0 and N > 0 and H * W == 0:
            N, H, W = 0, 1, 1                     # maps without pixels
        desc = B.make_norm_desc(N, C, H, W, dtype=x.dtype, param_dtype=torch.float32 if param is None else param.dtype,
                                layout=layout, eps=eps)
        stats = torch.empty((2, -(-max(N * H * W, 1) // 4) * 4), dtype=torch.float32, device=x.device)
        with torch.cuda.device(x.device):
            B.gf_layer_norm_forward(desc, x, weight, bias, y, stats[0], stats[1], torch.cuda.current_stream(x.device))
        ctx.desc, ctx.fmt = desc, fmt
        ctx.param_dtypes = (None if weight is None else weight.dtype), (None if bias is None else bias.dtype)
        ctx.save_for_backward(x, weight, stats)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, g_y):
        x, weight, stats = ctx.saved_tensors
        desc, (need_x, need_w, need_b) = ctx.desc, ctx.had_grad
        g_y = _dense(g_y, ctx.fmt)
        dev = g_y.device
        g_x = torch.empty_like(x, memory_format=ctx.fmt) if need_x else None
        g_w = torch.empty(desc.C, dtype=torch.float32, device=dev) if need_w else None
        g_b = torch.empty(desc.C, dtype=torch.float32, device=dev) if need_b else None
        with torch.cuda.device(dev):
            ws = torch.empty(B.gf_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device=dev)
            B.gf_layer_norm_backward(desc, g_y, x, weight, stats[0], stats[1], g_x, g_w, g_b, ws, None,
                                     torch.cuda.current_stream(dev))
        g_w = None if g_w is None else g_w.to(ctx.param_dtypes[0])
        g_b = None if g_b is None else g_b.to(ctx.param_dtypes[1])
        return g_x, g_w, g_b, None, None


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, eps: float = 1e-5,
               channel_dim: int = -1) -> torch.Tensor:
    """Layer norm of x over one dimension: the last one (any number of dimensions), or dimension 1 of
    a map [N, C, H, W].  x is float32 or bfloat16; weight and bias share a dtype, either of the two.
    Gradients come back in the dtypes of their tensors (the sums over pixels are fp32)."""
    if x.dim() < 1 or channel_dim not in (-1, 1, x.dim() - 1):
        raise ValueError("channel_dim is the last dimension, or 1 for a map [N, C, H, W]")
    last = channel_dim in (-1, x.dim() - 1)
    if not last and x.dim() != 4:
        raise ValueError("channel_dim = 1 needs a map [N, C, H, W]")
    return _LayerNormFn.apply(x, weight, bias, float(eps), -1 if last else 1)


class LayerNorm(torch.nn.Module):
    """Layer norm over `channels`: of the last dimension, or with channel_dim = 1 of the channels of
    maps [N, C, H, W] -- the norm between the convolutions of a block."""

    def __init__(self, channels: int, eps: float = 1e-5, channel_dim: int = -1, bias: bool = True, device=None, dtype=None):
        super().__init__()
        self.eps, self.channel_dim = eps, channel_dim
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(channels, device=device, dtype=dtype)) if bias else None

    def forward(self, x):
        return layer_norm(x, self.weight, self.bias, self.eps, self.channel_dim)
