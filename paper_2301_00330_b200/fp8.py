"""Frozen layers in 8 bits, on the library's kernels (include/gf_block.h).

A fine-tuning step runs the layers that are not trained forward, and takes the gradient of their inputs.  `Fp8Linear` keeps
such a layer's weight as e4m3 codes with a scale for each 128 x 128 block, half the bytes of 16 bits, and multiplies rows
quantised the same way (a scale for each 128 columns) in both directions with the one stored weight; nothing of its input is
kept for the backward pass.  `rms_norm_linear` leads a norm straight into such layers, its rows never stored in 16 bits.
Only marshalling happens here.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .autograd import FilteredConv2d
from .dropout import _check_p, _seed_for
from .norm import _dense
from .rms import _check_args, _norm_backward, _norm_desc

_INT32 = (1 << 31) - 1


@dataclass
class Fp8Matrix:
    """rows x cols values: codes [rows, fp8_pitch(cols)] (uint8) times scales, for each 128 columns of a row
    [ceil(cols / 128), fp8_scale_pitch(rows)], or for each 128 x 128 block [ceil(rows / 128), ceil(cols / 128)] (blocks true)."""
    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int
    blocks: bool

    def check(self) -> None:
        """The tensors have the sizes and types that the library reads."""
        codes = (self.rows, B.fp8_pitch(self.cols))
        scales = (-(-self.rows // 128), -(-self.cols // 128)) if self.blocks else (-(-self.cols // 128), B.fp8_scale_pitch(self.rows))
        if tuple(self.codes.shape) != codes or self.codes.element_size() != 1:
            raise ValueError(f"codes of one byte and shape {codes} expected, got {self.codes.dtype} {tuple(self.codes.shape)}")
        if tuple(self.scales.shape) != scales or self.scales.dtype != torch.float32 or self.scales.device != self.codes.device:
            raise ValueError(f"float32 scales of shape {scales} beside the codes expected, got {self.scales.dtype} {tuple(self.scales.shape)}")

    def dequantize(self) -> torch.Tensor:
        """The values as float32 [rows, cols]."""
        self.check()
        v = self.codes.view(torch.float8_e4m3fn)[:, :self.cols].float()
        if self.blocks:
            s = self.scales.repeat_interleave(128, 0)[:self.rows]
        else:
            s = self.scales[:, :self.rows].t()
        return v * s.repeat_interleave(128, 1)[:, :self.cols]


def _rows_of(x: torch.Tensor) -> int:
    return x.numel() // x.shape[-1]


def _empty_rows(rows: int, cols: int, device) -> Fp8Matrix:
    if rows > _INT32:
        raise ValueError(f"an 8-bit matrix has at most {_INT32} rows, got {rows}")
    return Fp8Matrix(torch.empty((rows, B.fp8_pitch(cols)), dtype=torch.uint8, device=device),
                     torch.empty((-(-cols // 128), B.fp8_scale_pitch(rows)), dtype=torch.float32, device=device), rows, cols, False)


def quantize_rows(x: torch.Tensor) -> Fp8Matrix:
    """x [..., cols] (float32 or bfloat16) as 8-bit rows."""
    if not x.is_cuda:
        raise RuntimeError("quantize_rows needs a CUDA tensor: there is no CPU path")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x has rows of at least one value")
    x = _dense(x.detach())
    q = _empty_rows(_rows_of(x), x.shape[-1], x.device)
    with torch.cuda.device(x.device):
        B.gf_fp8_quantize_rows(B.make_fp8_desc(q.rows, q.cols, dtype=x.dtype), x, q.codes, q.scales, torch.cuda.current_stream(x.device))
    return q


def quantize_weight(w: torch.Tensor) -> Fp8Matrix:
    """A weight [out, in] (float32 or bfloat16) as 8-bit blocks."""
    if not w.is_cuda:
        raise RuntimeError("quantize_weight needs a CUDA tensor: there is no CPU path")
    if w.dim() != 2 or w.numel() == 0:
        raise ValueError(f"a weight is a matrix [out, in], got {tuple(w.shape)}")
    w = _dense(w.detach())
    rows, cols = w.shape
    q = Fp8Matrix(torch.empty((rows, B.fp8_pitch(cols)), dtype=torch.uint8, device=w.device),
                  torch.empty((-(-rows // 128), -(-cols // 128)), dtype=torch.float32, device=w.device), rows, cols, True)
    with torch.cuda.device(w.device):
        B.gf_fp8_quantize_blocks(B.make_fp8_desc(rows, cols, dtype=w.dtype), w, q.codes, q.scales, torch.cuda.current_stream(w.device))
    return q


def fp8_matmul(a: Fp8Matrix, w: Fp8Matrix, bias: torch.Tensor | None = None, transposed: bool = False,
               out_dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """a W^T + bias [rows, out], or with transposed a W + bias [rows, in], of 8-bit rows and an 8-bit weight W [out, in]."""
    if a.blocks or not w.blocks:
        raise ValueError("a has scales of rows (quantize_rows), w of blocks (quantize_weight)")
    inner, outer = (w.rows, w.cols) if transposed else (w.cols, w.rows)
    if a.cols != inner:
        raise ValueError(f"a has {a.cols} columns, the weight takes {inner}")
    a.check()
    w.check()
    if not a.codes.is_cuda or any(t is not None and t.device != a.codes.device for t in (w.codes, bias)):
        raise ValueError("a, w and bias lie on one CUDA device")
    if bias is not None and bias.shape != (outer,):
        raise ValueError(f"bias has the shape ({outer},), got {tuple(bias.shape)}")
    dev = a.codes.device
    out = torch.empty((a.rows, outer), dtype=out_dtype, device=dev)
    desc = B.make_fp8_matmul_desc(a.rows, w.rows, w.cols, transposed=transposed, out_dtype=out_dtype,
                                  bias_dtype=torch.float32 if bias is None else bias.dtype)
    with torch.cuda.device(dev):
        B.gf_fp8_matmul(desc, a.codes, a.scales, w.codes, w.scales, None if bias is None else _dense(bias.detach()), out,
                        torch.cuda.current_stream(dev))
    return out


def _keep(ctx, weights, *others) -> None:
    """Saves the weights' tensors in the way that lets torch notice a change in place before the backward pass."""
    ctx.sizes = [(w.rows, w.cols) for w in weights]
    ctx.save_for_backward(*others, *(t for w in weights for t in (w.codes, w.scales)))


def _kept(ctx):
    """(others, weights) of _keep."""
    saved, n = ctx.saved_tensors, 2 * len(ctx.sizes)
    first = len(saved) - n
    return saved[:first], [Fp8Matrix(saved[first + 2 * i], saved[first + 2 * i + 1], rows, cols, True) for i, (rows, cols) in enumerate(ctx.sizes)]


class _Fp8LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, layer):
        ctx.dtype = x.dtype
        w = layer.matrix()
        _keep(ctx, [w])
        return fp8_matmul(quantize_rows(x), w, layer.bias, out_dtype=x.dtype).view(*x.shape[:-1], w.rows)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_y):
        w, = _kept(ctx)[1]
        g_x = fp8_matmul(quantize_rows(g_y), w, transposed=True, out_dtype=ctx.dtype)
        return g_x.view(*g_y.shape[:-1], w.cols), None


class Fp8Linear(torch.nn.Module):
    """A frozen linear layer (or 1 x 1 convolution, with channel_dim = 1) in 8 bits: y = x W^T + bias.

    Rows of x and, backwards, of g_y are quantised on the way in, with a scale for each 128 columns; y and the
    gradient of x have x's dtype (float32 or bfloat16).  Weight and bias get no gradients.  channel_dim 1 takes maps
    [N, C, H, W], in torch's channels_last memory format without a copy."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, channel_dim: int = -1):
        super().__init__()
        if channel_dim not in (-1, 1):
            raise ValueError("channel_dim is the last dimension, -1, or 1 for a map [N, C, H, W]")
        if weight.dim() == 4 and weight.shape[2:] == (1, 1):
            weight = weight.reshape(weight.shape[:2])
        q = quantize_weight(weight)
        if bias is not None and bias.shape != (q.rows,):
            raise ValueError(f"bias has the shape ({q.rows},), got {tuple(bias.shape)}")
        self.out_features, self.in_features, self.channel_dim = q.rows, q.cols, channel_dim
        self.register_buffer("codes", q.codes)
        self.register_buffer("scales", q.scales)
        self.register_buffer("bias", None if bias is None else bias.detach().clone())

    @classmethod
    def from_layer(cls, layer: torch.nn.Module) -> "Fp8Linear":
        """From a torch.nn.Linear, or a 1 x 1 convolution (torch.nn.Conv2d or FilteredConv2d) of stride 1 without groups.

        Other layers are refused, whatever their weight's shape: some keep it the other way round (torch.nn.ConvTranspose2d).  The gradient
        of a FilteredConv2d's input is a filtered one; that of the layer made from it is not, and is off only by the 8 bits."""
        if isinstance(layer, torch.nn.Linear):
            return cls(layer.weight, layer.bias)
        if not isinstance(layer, (torch.nn.Conv2d, FilteredConv2d)):
            raise ValueError(f"a linear layer or a 1 x 1 convolution expected, got {type(layer).__name__}")
        w, stride, padding = layer.weight, layer.stride, getattr(layer, "padding", 0)      # (a FilteredConv2d of 1 x 1 has none)
        if w.shape[2:] != (1, 1) or layer.groups != 1 or stride not in (1, (1, 1)) or padding not in (0, (0, 0), "same", "valid"):
            raise ValueError("a linear layer, or a 1 x 1 convolution of stride 1 without groups or padding, expected")
        return cls(w, layer.bias, channel_dim=1)

    def _apply(self, fn, recurse=True):
        scales = self.scales                        # stay float32 when the module is cast
        super()._apply(fn, recurse)
        if self.scales.dtype != torch.float32:
            self.scales = scales.to(self.scales.device)
        return self

    def matrix(self) -> Fp8Matrix:
        """The weight as the library's calls take it."""
        return Fp8Matrix(self.codes, self.scales, self.out_features, self.in_features, True)

    def forward(self, x):
        if self.channel_dim == 1:
            if x.dim() != 4:
                raise ValueError("channel_dim = 1 needs a map [N, C, H, W]")
            x = x.permute(0, 2, 3, 1)
        if x.shape[-1] != self.in_features:
            raise ValueError(f"x has {x.shape[-1]} channels, the layer takes {self.in_features}")
        y = _Fp8LinearFn.apply(x, self)
        return y.permute(0, 3, 1, 2) if self.channel_dim == 1 else y

    def extra_repr(self):
        return f"in_features={self.in_features}, out_features={self.out_features}, bias={self.bias is not None}"


class _RmsNormLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, seed, eps: float, p: float, layers):
        ctx.set_materialize_grads(False)
        desc = _norm_desc(x, weight, residual, eps, p)
        x = _dense(x)
        weight = None if weight is None else _dense(weight)
        residual = None if residual is None else _dense(residual)
        plain = residual is None and seed is None
        h = None if plain else torch.empty_like(x if residual is None else residual)
        rstd = torch.empty(max(desc.rows, 1), dtype=torch.float32, device=x.device)
        q = _empty_rows(desc.rows, desc.cols, x.device)
        with torch.cuda.device(x.device):
            B.gf_rms_norm_forward_fp8(desc, x, residual, seed, weight, h, q.codes, q.scales, rstd, torch.cuda.current_stream(x.device))
        weights = [layer.matrix() for layer in layers]
        outs = [fp8_matmul(q, w, layer.bias, out_dtype=x.dtype).view(*x.shape[:-1], w.rows) for w, layer in zip(weights, layers)]
        ctx.desc, ctx.x_dtype = desc, x.dtype
        _keep(ctx, weights, x if plain else h, rstd, weight, seed)
        return (h, *outs)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_h, *g_outs):
        (h, rstd, weight, seed), weights = _kept(ctx)
        need_x, need_w, need_res = ctx.needs_input_grad[:3]
        g_y = None
        for w, g in zip(weights, g_outs):
            if g is not None:            # parts are rounded to x's dtype and added in it, as torch adds the gradients of a shared input
                part = fp8_matmul(quantize_rows(g), w, transposed=True, out_dtype=ctx.x_dtype)
                g_y = part if g_y is None else g_y.add_(part)
        g_y = torch.zeros(h.shape, dtype=ctx.x_dtype, device=h.device) if g_y is None else g_y.view(h.shape)
        g_x, g_w, g_res = _norm_backward(ctx.desc, g_y, g_h, h, rstd, weight, seed, need_x, need_w, need_res, ctx.x_dtype)
        return g_x, g_w, g_res, None, None, None, None


def rms_norm_linear(x: torch.Tensor, weight: torch.Tensor | None, layers, eps: float = 1e-5, residual: torch.Tensor | None = None,
                    p: float = 0.0, training: bool = True, seed: torch.Tensor | None = None):
    """Frozen 8-bit layers (an Fp8Linear, or several that share their input) applied to rms_norm(x, weight, ..): the norm
    writes 8-bit rows, quantised from its 32-bit values, and what is kept for the backward pass is h and a number per row.

    Returns the layer's result (a tuple of them for several), and with a residual (result, h) as rms_norm does.  The
    gradient passes the rounding to 8 bits unchanged."""
    _check_args(x, weight, residual, "rms_norm_linear")
    several = not isinstance(layers, Fp8Linear)
    layers = tuple(layers) if several else (layers,)
    for layer in layers:
        if not isinstance(layer, Fp8Linear) or layer.channel_dim != -1 or layer.in_features != x.shape[-1]:
            raise ValueError(f"layers are Fp8Linear of {x.shape[-1]} features in the last dimension")
        if layer.codes.device != x.device:
            raise ValueError(f"all layers lie on the device of x, {x.device}")
    p = _check_p(p) if training else 0.0
    if residual is None and p > 0:
        raise ValueError("p > 0 drops elements of a branch that is added to a residual: there is none")
    h, *outs = _RmsNormLinearFn.apply(x, weight, residual, _seed_for(x, p, seed), float(eps), p, layers)
    out = tuple(outs) if several else outs[0]
    return out if residual is None else (out, h)
