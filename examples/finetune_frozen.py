"""Fine-tunes the end of a network whose earlier blocks are frozen in 8 bits, on synthetic data.

What on-device training does: most layers run forward, and backward only as far as the gradient of their input goes; a norm's
weights, and the last convolution, are trained.  The frozen blocks are residual MLPs over the channels of a map; their weights are
e4m3 codes (Fp8Linear), the norm in front of them adds the branch before it to the residual, drops elements of it and writes 8-bit
rows for the layers in one pass, and what a block keeps for the backward pass is its residual sum and one number per pixel.
The trained convolution at the end has filtered gradients (patches of 2 x 2).  Needs a B200.

    python examples/finetune_frozen.py [--steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2301_00330_b200 as gf  # noqa: E402


class FrozenBlock(torch.nn.Module):
    """h <- residual + dropout(branch); the next branch is down(gelu(up(norm(h)))): up and down frozen in 8 bits, the norm trained."""

    def __init__(self, channels: int, expansion: int, p: float, device, dtype):
        super().__init__()
        self.p, self.eps = p, 1e-6
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device, dtype=dtype))
        wide = expansion * channels
        self.up = gf.Fp8Linear(torch.randn(wide, channels, device=device) * channels ** -0.5, torch.zeros(wide, device=device))
        self.down = gf.Fp8Linear(torch.randn(channels, wide, device=device) * wide ** -0.5)

    def forward(self, branch, residual, seed=None):
        y, h = gf.rms_norm_linear(branch, self.weight, self.up, self.eps, residual, self.p, self.training, seed)
        return self.down(torch.nn.functional.gelu(y)), h


class Net(torch.nn.Module):
    """Pixels as rows through the frozen blocks, then a trained 3 x 3 convolution with filtered gradients on the map."""

    def __init__(self, channels: int = 96, expansion: int = 4, blocks: int = 3, classes: int = 21, p: float = 0.1, r: int = 2,
                 device="cuda", dtype=torch.float32):
        super().__init__()
        self.blocks = torch.nn.ModuleList(FrozenBlock(channels, expansion, p, device, dtype) for _ in range(blocks))
        self.norm = gf.RMSNorm(channels, eps=1e-6, p=p, device=device, dtype=dtype)
        self.head = gf.FilteredConv2d(channels, classes, 3, r=r, bias=False, device=device, dtype=dtype)

    def forward(self, x, seeds=None):
        """x [N, C, H, W]; seeds: one for each block and the norm after them (None: drawn)."""
        n, c, h, w = x.shape
        seeds = [None] * (len(self.blocks) + 1) if seeds is None else seeds
        residual = x.permute(0, 2, 3, 1).reshape(-1, c)
        branch = torch.zeros_like(residual)
        for block, seed in zip(self.blocks, seeds):
            branch, residual = block(branch, residual, seed)
        y, _ = gf.rms_norm(branch, self.norm.weight, self.norm.eps, residual, self.norm.p, self.training, seeds[-1])
        return self.head(y.view(n, h, w, c).permute(0, 3, 1, 2).contiguous())


def finetune(steps: int = 20, batch: int = 4, channels: int = 96, size: int = 28, dtype: torch.dtype = torch.float32, seed: int = 0) -> list[float]:
    """Losses of `steps` steps towards the classes of fixed random pixels."""
    torch.manual_seed(seed)
    net = Net(channels, dtype=dtype)
    norms = [p for n, p in net.named_parameters() if not n.startswith("head")]
    muon = gf.Muon([net.head.weight], lr=2e-2)
    sgd = torch.optim.SGD(norms, lr=1e-2, momentum=0.9)
    target = torch.randint(0, 21, (batch, size, size), device="cuda")
    x = torch.randn(batch, channels, size, size, device="cuda", dtype=dtype)
    losses = []
    for _ in range(steps):
        loss = torch.nn.functional.cross_entropy(net(x).float(), target)
        loss.backward()
        muon.step()
        sgd.step()
        for p in net.parameters():
            p.grad = None
        losses.append(loss.detach())
    return [float(v) for v in torch.stack(losses).cpu()]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    for k, v in enumerate(finetune(steps=args.steps)):
        print(f"step {k:3d}  loss {v:.6f}")


if __name__ == "__main__":
    main()
