"""The residual-block operators together, as the example uses them: frozen 8-bit blocks with a norm that adds, drops and quantises
in one pass, and a trained convolution with filtered gradients behind them.

The reference forms every step in 64 bits from elementary operations, with the library's quantisers (tested on their own) for
the roundings to 8 bits and gf.dropout's mask.  Where a value lies next to a border between two codes, the two sides may
take different ones (fp32 against 64 bits): a code is 2^-4 of its value at most, and a share of 2^-18 of the values (the
width of fp32's roundings, some 32 units, against half a code) are that near, so that sums of many values differ by about
2^-4 2^-9 = 2^-13 of their norm per rounding; twelve roundings follow one another forward and backward, with amplification by the
layers of a few times: 2^-8 of a tensor's norm is allowed.  For 16 bits 2^-8 of each value is rounded at each of some twenty
steps, and what one side rounds up the other may round down: 20^(1/2) 2^-8, under 2^-5."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("finetune_frozen", os.path.join(ROOT, "examples", "finetune_frozen.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


class _Rounded(torch.autograd.Function):
    """Rounding to 8 bits by rows, whose gradient passes unchanged."""
    @staticmethod
    def forward(ctx, x, gf):
        return gf.quantize_rows(x.float()).dequantize().double()

    @staticmethod
    def backward(ctx, g):
        return g, None


class _Product(torch.autograd.Function):
    """x W^T, with the gradient of x formed of the gradient rounded to 8 bits by rows (in the type that reaches the layer)."""
    @staticmethod
    def forward(ctx, x, W, gf, dtype):
        ctx.W, ctx.gf, ctx.dtype = W, gf, dtype
        return x @ W.t()

    @staticmethod
    def backward(ctx, g):
        return ctx.gf.quantize_rows(g.to(ctx.dtype)).dequantize().double() @ ctx.W, None, None, None


class _Kept(torch.autograd.Function):
    """A value that is kept in the run's type, as is its gradient (`both`; else the value alone)."""
    @staticmethod
    def forward(ctx, x, dtype, both=True):
        ctx.dtype, ctx.both = dtype, both
        return x.to(dtype).double()

    @staticmethod
    def backward(ctx, g):
        return g.to(ctx.dtype).double() if ctx.both else g, None, None


def _reference(gf, net, x, seeds, dtype):
    n, c, h, w = x.shape
    weights = [b.weight.detach().double().requires_grad_(True) for b in net.blocks] + [net.norm.weight.detach().double().requires_grad_(True)]
    x = x.detach().double().requires_grad_(True)
    residual = x.permute(0, 2, 3, 1).reshape(-1, c)
    branch = torch.zeros_like(residual)

    def sum_and_norm(branch, residual, weight, seed, eps, p):
        keep = gf.dropout(torch.ones(branch.shape, device="cuda", dtype=dtype), p, seed=seed) if p else torch.ones_like(branch)
        h = _Kept.apply(residual, dtype) + branch * (keep != 0).double() * (65536 / (65536 - round(p * 65536)))
        h = _Kept.apply(h, dtype, False)                # its gradient goes on in 32 bits, to be rounded on either way
        return h * (h.square().mean(1, keepdim=True) + eps).rsqrt() * weight, h

    def layer(x, frozen):
        y = _Product.apply(_Rounded.apply(x, gf), frozen.matrix().dequantize().double(), gf, dtype)
        return _Kept.apply(y if frozen.bias is None else y + frozen.bias.double(), dtype)

    for block, weight, seed in zip(net.blocks, weights, seeds):
        y, residual = sum_and_norm(branch, residual, weight, seed, block.eps, block.p if net.training else 0)
        branch = layer(_Kept.apply(torch.nn.functional.gelu(layer(y, block.up)), dtype), block.down)
    y, _ = sum_and_norm(branch, residual, weights[-1], seeds[-1], net.norm.eps, net.norm.p if net.training else 0)
    return x, weights, _Kept.apply(y, dtype).view(n, h, w, c).permute(0, 3, 1, 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("training", [True, False])
@pytest.mark.parametrize("channels,size", [(96, 12), (40, 9), (136, 14)])
def test_a_stack_of_frozen_blocks(gf, example, channels, size, training, dtype):
    torch.manual_seed(channels)
    net = example.Net(channels, blocks=2, classes=16, p=0.2, r=1, dtype=dtype).train(training)     # r = 1: exact gradients of the head
    for b in net.blocks:
        torch.nn.init.normal_(b.weight, 1.0, 0.2)
    x = torch.randn(2, channels, size, size, device="cuda").to(dtype).requires_grad_(True)
    seeds = [gf.dropout_seed("cuda") for _ in range(3)]
    out = net(x, seeds)
    g = torch.randn(out.shape, device="cuda").to(dtype)
    out.backward(g)
    rx, weights, y = _reference(gf, net, x, seeds, dtype)
    want = torch.nn.functional.conv2d(y, net.head.weight.detach().double(), None, 1, 1)
    want.backward(g.double())
    tol = 2.0 ** -8 if dtype == torch.float32 else 2.0 ** -5

    def near(got, ref):
        err = float((got.detach().double() - ref.detach()).norm() / ref.detach().norm())
        assert err <= tol, err

    near(out, want)
    near(x.grad, rx.grad)
    for p, w in zip([*(b.weight for b in net.blocks), net.norm.weight], weights):
        near(p.grad, w.grad)


def test_several_layers_share_one_norm(gf):
    """A norm into three layers gives what the layers give one by one, and the sum of their gradients; a layer whose result is not used adds none."""
    torch.manual_seed(1)
    layers = [gf.Fp8Linear(torch.randn(n, 96, device="cuda") * 0.1) for n in (64, 33, 128)]
    x, r, w = torch.randn(50, 96, device="cuda"), torch.randn(50, 96, device="cuda"), torch.randn(96, device="cuda")
    seed = gf.dropout_seed("cuda")

    def run(which):
        a, b, c = (t.clone().requires_grad_(True) for t in (x, w, r))
        outs, h = gf.rms_norm_linear(a, b, layers, residual=c, p=0.2, seed=seed)
        loss = sum((outs[k] * (k + 1)).square().sum() for k in which)
        loss.backward()
        return [o.detach() for o in outs], h.detach(), a.grad, b.grad, c.grad

    outs, h, *grads = run((0, 1, 2))
    single = []
    for k, layer in enumerate(layers):
        a, b, c = (t.clone().requires_grad_(True) for t in (x, w, r))
        o, h1 = gf.rms_norm_linear(a, b, layer, residual=c, p=0.2, seed=seed)
        (o * (k + 1)).square().sum().backward()
        assert torch.equal(o, outs[k]) and torch.equal(h1, h)
        single.append((a.grad, b.grad, c.grad))
    for got, parts in zip(grads, zip(*single)):
        want = sum(p.double() for p in parts)
        assert float((got.double() - want).norm() / want.norm()) <= 1e-5      # fp32 sums of the same parts in another order
    part = run((1,))[2:]
    for got, want in zip(part, single[1]):
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_example_runs(gf, example, dtype):
    losses = example.finetune(steps=3, batch=2, channels=32, size=16, dtype=dtype)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)


def test_a_training_step_in_a_graph(gf, example):
    """Forward and backward of the stack captured and replayed: other masks every time, gradients that match their forward pass."""
    torch.manual_seed(2)
    net = example.Net(64, blocks=1, classes=8, p=0.5, r=2)
    x = torch.randn(1, 64, 8, 8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    params = list(net.parameters())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(net(x).square().sum(), params)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = net(x)
        grads = torch.autograd.grad(y.square().sum(), params)
    seen = []
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool(torch.isfinite(g).all()) for g in grads)
        seen.append(y.clone())
    assert not torch.equal(*seen)
