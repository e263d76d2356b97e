"""The example that runs the operators together: filtered convolutions, layer norm and Muon on one block."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("finetune_block", os.path.join(ROOT, "examples", "finetune_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("channels_last", [False, True])
def test_the_block_learns(gf, example, channels_last):
    """Forty steps towards a fixed block bring the loss down, with either memory format; the loss of the last ten steps
    is below four fifths of the first ten's."""
    losses = example.finetune(steps=40, batch=4, channels=32, size=16, channels_last=channels_last)
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-10:]) < 0.8 * sum(losses[:10]), losses


def test_sixteen_bit_block_runs(gf, example):
    losses = example.finetune(steps=3, batch=2, channels=32, size=16, dtype=torch.bfloat16)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
