"""Calls of the residual-block operators (include/gf_block.h) at the ends of what they take, as far as the host decides."""
import ctypes

import pytest
import torch


def test_which_product_kernel(gf):
    """Nothing is said of a descriptor that is refused, or of no rows; few rows are few at any size."""
    f, mk = gf.gf_selftest_fp8_form, gf.make_fp8_matmul_desc
    assert gf.lib().gf_selftest_fp8_form(None) == -1
    for bad in ({"M": -1}, {"M": 0}, {"N": 0}, {"K": 0}, {"transposed": 2}, {"out_dtype": 3}, {"K": (1 << 24) + 1}):
        assert f(mk(**({"M": 4, "N": 8, "K": 8} | bad))) == -1
    for t in (False, True):
        for M in (1, 16, 17, 32):
            form = f(mk(M, 4096, 4096, transposed=t))
            assert form & 255 == 0 and 1 <= form >> 8 <= 8


def test_frozen_layers_are_made_of_layers_whose_weight_is_known(gf):
    """A weight of the right shape is not enough: a transposed convolution keeps it as [in, out, 1, 1], others as [in, out]."""
    class Other(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.weight, self.bias = torch.nn.Parameter(torch.zeros(8, 8)), None

    for layer in (torch.nn.ConvTranspose2d(8, 8, 1), torch.nn.ConvTranspose2d(8, 12, 1, bias=False), Other(), torch.nn.Embedding(8, 8),
                  torch.nn.Conv1d(8, 8, 1), torch.nn.Conv2d(8, 8, 1, stride=2), torch.nn.LayerNorm(8)):
        with pytest.raises(ValueError):
            gf.Fp8Linear.from_layer(layer)
    for layer in (torch.nn.Linear(8, 12), torch.nn.Conv2d(8, 12, 1), gf.FilteredConv2d(8, 12, 1)):      # on to the quantiser
        with pytest.raises(RuntimeError, match="no CPU path"):
            gf.Fp8Linear.from_layer(layer)


def test_counts_that_no_grid_holds_are_refused(gf):
    """A block has 4096 elements and a grid 2^31 - 1 blocks; the refusal comes before anything is launched."""
    a = ctypes.c_void_p(0x1000)                          # never dereferenced
    most = ((1 << 31) - 1) * 4096
    for count in (most + 1, most + 2, 1 << 43, (1 << 43) + 1, (1 << 63) - 1):
        d = gf.make_dropout_desc(count, p=0.5)
        assert gf.lib().gf_dropout_forward(ctypes.byref(d), a, a, a, a, None) == gf.GF_ERR_UNSUPPORTED
        assert gf.lib().gf_dropout_backward(ctypes.byref(d), a, a, a, None) == gf.GF_ERR_UNSUPPORTED


def test_no_output_over_an_input_of_another_type(gf):
    """In place, an element's result would lie where another element is still to be read."""
    L, vp = gf.lib(), ctypes.c_void_p
    a, b, c, d = (vp(0x1000 * k) for k in (1, 2, 3, 4))      # never dereferenced: all calls fail on the host
    for xt, yt in ((gf.GF_F32, gf.GF_BF16), (gf.GF_BF16, gf.GF_F32)):
        desc = ctypes.byref(gf.make_dropout_desc(64, dtype=xt, out_dtype=yt, p=0.5))
        assert L.gf_dropout_forward(desc, a, b, c, a, None) == gf.GF_ERR_UNSUPPORTED
        assert L.gf_dropout_forward(desc, a, None, c, a, None) == gf.GF_ERR_UNSUPPORTED
        assert L.gf_dropout_backward(desc, a, c, a, None) == gf.GF_ERR_UNSUPPORTED
    for cols in (8, 1001, 9000):
        rms = gf.make_rms_desc(4, cols, dtype=gf.GF_BF16, residual_dtype=gf.GF_F32)
        need = gf.gf_rms_norm_backward_workspace_bytes(rms)
        desc = ctypes.byref(rms)
        assert L.gf_rms_norm_forward(desc, a, b, None, None, a, c, None, None) == gf.GF_ERR_UNSUPPORTED
        assert L.gf_rms_norm_forward_fp8(desc, a, b, None, None, a, c, d, None, None) == gf.GF_ERR_UNSUPPORTED
        assert L.gf_rms_norm_backward(desc, a, None, b, c, None, None, a, None, None, d, need, None) == gf.GF_ERR_UNSUPPORTED
