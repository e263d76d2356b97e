"""Codes of 8 bits (gf_block.h) over the whole range of scales: those of a division, also where a remainder would be subnormal."""
import numpy as np
import pytest
import torch

from block_util import e4m3_values
from test_fp8_gpu import _check_codes

pytestmark = pytest.mark.gpu

EXPONENTS = [-117, -116, -115, -113, -110, -105, -100, -95, -91, -85, -82, -81, -80, -70, 0, 60, 100, 120, 126, 127]


def _borders(exponent, cols, seed):
    """Rows with maxima of 2^exponent to 2^(exponent + 1) (the last of them the largest numbers of it), whose other values lie on a border
    between two codes, as near as fp32 comes, or a step beside it."""
    R = 2048
    g = np.random.RandomState(seed)
    top = np.ldexp((1 + g.rand(R)).astype(np.float32), exponent).astype(np.float32)
    top[-4:] = np.ldexp(np.float32(2 - 2.0 ** -23), exponent)
    table = e4m3_values(np.arange(127, dtype=np.uint8))
    borders = (table[1:] + table[:-1]) / 2
    scale = np.maximum(top * (np.float32(1) / np.float32(448)), np.float32(2.0 ** -126)).astype(np.float64)[:, None]
    v = (np.resize(borders[:125], cols - 1)[None, :] * scale).astype(np.float32)
    step = g.randint(-1, 2, v.shape)
    v = np.where(step > 0, np.nextafter(v, np.float32(np.inf)), np.where(step < 0, np.nextafter(v, np.float32(0)), v))
    v = np.minimum(v, top[:, None]) * g.choice(np.array([-1, 1], np.float32), v.shape)
    return np.concatenate([top[:, None], v], 1).astype(np.float32)


@pytest.mark.parametrize("exponent", EXPONENTS)
def test_quotients_over_the_whole_range(gf, exponent):
    for cols in (126, 128):                                                # either way of reading rows
        x = torch.from_numpy(_borders(exponent, cols, exponent + 200)).cuda()
        q = gf.quantize_rows(x)
        _check_codes(x, q.codes, q.scales, False)
        # whole blocks have one scale: a row's values in a block of its own (rows of zeros around it)
        w = torch.zeros((128 * 8, cols), device="cuda")
        w[::128] = x[-8:]
        q = gf.quantize_weight(w)
        _check_codes(w, q.codes, q.scales, True)


@pytest.mark.parametrize("exponent", [-117, -112, -106, -100, -95, -85, 126, 127])
def test_16_bit_values_of_the_smallest_and_largest_scales(gf, exponent):
    """bf16 values, of which many lie on a border exactly: all products of a value with a power of two below the largest."""
    R = 512
    g = np.random.RandomState(exponent + 300)
    v = np.ldexp((1 + g.randint(0, 128, (R, 128)) / 128.0), exponent - g.randint(0, 18, (R, 128)))
    v[:, 0] = np.ldexp(1.75, exponent)                                      # scale 2^(exponent - 8): quotients are the values themselves
    v = np.where(np.abs(v) > v[:, :1], v / 2, v) * g.choice([-1, 1], v.shape)
    v[R // 2:, 0] = np.ldexp((1 + g.randint(96, 128, R - R // 2) / 128.0), exponent)
    x = torch.from_numpy(v.astype(np.float32)).bfloat16().cuda()
    q = gf.quantize_rows(x)
    _check_codes(x, q.codes, q.scales, False)
    assert torch.equal(gf.quantize_rows(x.float()).codes, q.codes)


def test_norms_of_small_weights_in_8_bits(gf):
    """The norm's 8-bit rows are those of its fp32 result, also where that is tiny: gamma of 2^-100 to 2^-117."""
    for C in (128, 333, 9000):
        x = torch.randn(40, C, device="cuda", generator=torch.Generator("cuda").manual_seed(C))
        gamma = torch.exp2(-100.0 - torch.arange(C, device="cuda").div(128, rounding_mode="floor").remainder(18))
        y = gf.rms_norm(x, gamma)
        want = gf.quantize_rows(y)
        desc = gf.make_rms_desc(40, C)
        codes = torch.empty((40, gf.fp8_pitch(C)), dtype=torch.uint8, device="cuda")
        scales = torch.empty((-(-C // 128), 40), device="cuda")
        gf.gf_rms_norm_forward_fp8(desc, x, None, None, gamma, None, codes, scales)
        assert torch.equal(codes, want.codes) and torch.equal(scales, want.scales)
        _check_codes(y, codes, scales, False)
