"""Fine-tunes one inverted-residual style block on synthetic data with filtered gradients.

The block is what the package's operators are for, together: a depthwise 7x7 and two 1x1 convolutions whose
backward passes are the filtered ones (patches of 2 x 2), a layer norm over channels between them, the
kernels updated by Muon (which uses that a filtered gradient has one value for all taps) and the vectors by
SGD.  Needs a B200.

    python examples/finetune_block.py [--steps 20] [--channels-last]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2301_00330_b200 as gf  # noqa: E402


class Block(torch.nn.Module):
    """x + scale * project(gelu(expand(norm(depthwise(x)))))"""

    def __init__(self, channels: int, expansion: int, r: int, device, dtype):
        super().__init__()
        at = {"device": device, "dtype": dtype}
        self.depthwise = gf.FilteredConv2d(channels, channels, 7, r=r, groups=channels, **at)
        self.norm = gf.LayerNorm(channels, eps=1e-6, channel_dim=1, **at)
        self.expand = gf.FilteredConv2d(channels, expansion * channels, 1, r=r, **at)
        self.project = gf.FilteredConv2d(expansion * channels, channels, 1, r=r, **at)
        self.scale = torch.nn.Parameter(torch.full((channels,), 0.1, **at))

    def forward(self, x):
        y = self.project(torch.nn.functional.gelu(self.expand(self.norm(self.depthwise(x)))))
        return x + self.scale.view(1, -1, 1, 1) * y


def finetune(steps: int = 20, batch: int = 8, channels: int = 96, expansion: int = 4, size: int = 28, r: int = 2,
             dtype: torch.dtype = torch.float32, channels_last: bool = False, seed: int = 0) -> list[float]:
    """Losses of `steps` steps towards a fixed random block's outputs."""
    torch.manual_seed(seed)
    device = torch.device("cuda")
    fmt = torch.channels_last if channels_last else torch.contiguous_format
    teacher = Block(channels, expansion, r, device, dtype)
    student = Block(channels, expansion, r, device, dtype)
    # depthwise kernels are vectors per channel: they stay with the vectors
    kernels = [student.expand.weight, student.project.weight]
    vectors = [p for p in student.parameters() if all(p is not k for k in kernels)]
    muon = gf.Muon(kernels, lr=5e-3, weight_decay=1e-2)
    sgd = torch.optim.SGD(vectors, lr=5e-2, momentum=0.9)
    losses = []
    for _ in range(steps):
        x = torch.randn(batch, channels, size, size, device=device, dtype=dtype).contiguous(memory_format=fmt)
        with torch.no_grad():
            target = teacher(x)
        loss = (student(x) - target).float().square().mean()
        loss.backward()
        muon.step()
        sgd.step()
        for p in student.parameters():
            p.grad = None
        losses.append(loss.detach())
    return [float(v) for v in torch.stack(losses).cpu()]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--channels-last", action="store_true")
    args = ap.parse_args()
    losses = finetune(steps=args.steps, channels_last=args.channels_last)
    for k, v in enumerate(losses):
        print(f"step {k:3d}  loss {v:.6f}")


if __name__ == "__main__":
    main()
