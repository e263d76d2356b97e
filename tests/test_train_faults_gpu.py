"""What goes wrong on the way of the fine-tuning operators, on the GPU: waits that run out end their kernels in an orderly way."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_lanes_of_a_warp_give_up_together(gf):
    """Half of the lanes are told to wait for half a millisecond, half for 32, the barrier completes after 4: the lanes that saw it must
    not go on without the others."""
    result = torch.full((32,), 7, dtype=torch.int32, device="cuda")
    gf.gf_selftest_warp_wait(result, 1_000_000)
    torch.cuda.synchronize()
    assert bool((result == 0).all()), result.tolist()
