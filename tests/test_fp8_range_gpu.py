"""8-bit products (gf_block.h) whose scales lie at the ends of fp32.

A row's scale times a block's may lie outside fp32's normal numbers while the scaled sum of a chunk, up to 128 448^2 = 2^24.6 of them,
does not.  Bounds: those of test_fp8_gpu.py on the terms, and where a result or a sum on the way is subnormal half a step of it for each
chunk's sum and the bias (2^-150 each), and of the result (2^-150 for fp32, 2^-134 for bf16)."""
import numpy as np
import pytest
import torch

from block_util import DTYPES, STEP, U, e4m3_values, random_codes
from test_fp8_gpu import _product

pytestmark = pytest.mark.gpu

F32, BF16 = DTYPES
SUBNORMAL = {F32: 2.0 ** -150, BF16: 2.0 ** -134}
# both kernels in both directions: few rows in one, two and four CTAs a tile, many rows with tiles of 256 and of 128 columns
SHAPES = [(9, 260, 130, False), (30, 200, 700, False), (150, 300, 520, True), (300, 130, 1100, False), (4100, 1000, 576, False), (5000, 1000, 520, True),
          (18000, 576, 96, True), (4099, 1001, 576, False)]


def _check(a, w, sa, sw, y, transposed):
    """Against 64 bits; the largest magnitude of the reference, for the caller to say what it expected of its inputs."""
    M, outer = a.shape[0], y.shape[1]
    wv = e4m3_values(w) * np.repeat(np.repeat(sw.astype(np.float64), 128, 0)[:w.shape[0]], 128, 1)[:, :w.shape[1]]
    wv = wv[:, :outer] if transposed else wv.T
    inner = wv.shape[0]
    av = e4m3_values(a[:, :inner]) * np.repeat(sa[:, :M].astype(np.float64).T, 128, 1)[:, :inner]
    if not transposed:                                                     # the codes behind the last column
        av, wv = np.nan_to_num(av, nan=0.0), np.nan_to_num(wv, nan=0.0)
    t_a, t_w = torch.from_numpy(av).cuda(), torch.from_numpy(np.ascontiguousarray(wv)).cuda()
    ref, mag = t_a @ t_w, t_a.abs() @ t_w.abs()
    chunks = -(-inner // 128)
    bound = (128 * 2 * U + (chunks + 4) * U) * mag + STEP[y.dtype] * ref.abs() + (chunks + 1) * 2.0 ** -150 + SUBNORMAL[y.dtype]
    err = (y.double() - ref).abs()
    assert bool((err <= bound).all()), float((err / bound).nan_to_num(nan=float("inf")).max())
    return ref


@pytest.mark.parametrize("out", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("M,N,K,transposed", SHAPES, ids=lambda v: str(v))
def test_scales_whose_product_is_small(gf, M, N, K, transposed, out):
    """Rows of the smallest scale and of ordinary ones by turns, blocks down to 2^-30: products to 2^-156, results from 1 to nothing."""
    inner = N if transposed else K
    g = np.random.RandomState(M)
    groups, pitch = -(-inner // 128), -(-M // 4) * 4
    sa = np.exp2(g.choice([-126, -126, -125, -120, -110, -100, -60, -5], (groups, pitch))) * (1 + g.rand(groups, pitch))
    sa = np.maximum(np.where(g.rand(groups, pitch) < 0.3, 2.0 ** -126, sa), 2.0 ** -126).astype(np.float32)
    sw = (np.exp2(-g.uniform(1, 30, (-(-N // 128), -(-K // 128))))).astype(np.float32)
    a, w, sa, sw, _, y = _product(gf, M, N, K, transposed, out, seed=M + K, sa=sa, sw=sw)
    ref = _check(a, w, sa, sw, y, transposed)
    normal = (ref.abs() >= 2.0 ** -126) & (ref.abs() < 2.0 ** -100)
    assert bool(normal.any()), "the sizes are there for normal results of the smallest scales"


def test_all_rows_of_the_smallest_scale(gf):
    """The same, with no ordinary row beside: whole tiles by the other way of scaling."""
    for M, N, K, transposed in SHAPES:
        inner = N if transposed else K
        sa = np.full((-(-inner // 128), -(-M // 4) * 4), 2.0 ** -126, np.float32)
        sw = np.full((-(-N // 128), -(-K // 128)), 3e-6, np.float32)
        a, w, sa, sw, _, y = _product(gf, M, N, K, transposed, F32, seed=M, sa=sa, sw=sw)
        _check(a, w, sa, sw, y, transposed)


def _tiny_codes(rows, cols, seed):
    """Codes of 0 and +-2^-9, what lies behind the last column NaN."""
    g = np.random.RandomState(seed)
    c = g.choice(np.array([0, 0, 1, 129], dtype=np.uint8), (rows, -(-cols // 16) * 16))
    c[rows // 2, :] = 0
    c[:, cols:] = 127
    return c


@pytest.mark.parametrize("M,N,K,transposed", SHAPES, ids=lambda v: str(v))
def test_scales_whose_product_is_large(gf, M, N, K, transposed):
    """Products of scales from 2^88 to 2^136 over sums of terms of 2^-18: results are finite (with terms of either sign some 2^4 of
    them add up, 2^122), and zero where the codes are zero (a row of A and one of W), which an infinite product turns into NaN."""
    inner, outer = (N, K) if transposed else (K, N)
    g = np.random.RandomState(M)
    groups, pitch = -(-inner // 128), -(-M // 4) * 4
    sa = np.exp2(g.choice([30, 62, 70, 76], (groups, pitch)) - g.rand(groups, pitch)).astype(np.float32)
    sw = np.exp2(g.uniform(59, 59.9, (-(-N // 128), -(-K // 128)))).astype(np.float32)
    a, w = _tiny_codes(M, inner, M), _tiny_codes(N, K, K)
    a, w, sa, sw, _, y = _product(gf, M, N, K, transposed, F32, sa=sa, sw=sw, a=a, w=w)
    ref = _check(a, w, sa, sw, y, transposed)
    assert bool((y[M // 2] == 0).all()) and float(ref.abs().max()) < 2.0 ** 128
    assert bool((sa[:, :M].max() * sw.max().astype(np.float64)) > 2.0 ** 128)


@pytest.mark.parametrize("M,N,K,transposed", SHAPES, ids=lambda v: str(v))
def test_small_ordinary_and_large_scales_by_turns(gf, M, N, K, transposed):
    """Every chunk of a row has a scale of its own size, from the smallest to 2^80: sums stay below 2^80 2^25 16."""
    inner = N if transposed else K
    g = np.random.RandomState(M + 1)
    groups, pitch = -(-inner // 128), -(-M // 4) * 4
    sa = np.exp2(g.choice([-126, -126, -124, -60, -3, 20, 80], (groups, pitch)) + g.rand(groups, pitch) * (g.rand(groups, pitch) < 0.7)).astype(np.float32)
    sw = np.exp2(-g.uniform(0, 20, (-(-N // 128), -(-K // 128)))).astype(np.float32)
    a, w = random_codes(M, inner, M), random_codes(N, K, K)
    a[::5, :inner] = 0
    a, w, sa, sw, _, y = _product(gf, M, N, K, transposed, F32, sa=sa, sw=sw, a=a, w=w)
    _check(a, w, sa, sw, y, transposed)
    assert bool((y[::5] == 0).all())


def test_a_row_does_not_depend_on_its_neighbours_scales(gf):
    """An ordinary row gives the same bits beside rows of the smallest scale as beside ordinary ones."""
    for M, N, K, transposed in SHAPES:
        inner = N if transposed else K
        groups, pitch = -(-inner // 128), -(-M // 4) * 4
        g = np.random.RandomState(3)
        sa = np.exp2(g.uniform(-9, 0, (groups, pitch))).astype(np.float32)
        sw = np.exp2(g.uniform(-12, -6, (-(-N // 128), -(-K // 128)))).astype(np.float32)
        a, w = random_codes(M, inner, 4), random_codes(N, K, 5)
        alone = _product(gf, M, N, K, transposed, F32, sa=sa.copy(), sw=sw, a=a, w=w)[-1]
        mixed = sa.copy()
        mixed[:, ::3] = 2.0 ** -126
        got = _product(gf, M, N, K, transposed, F32, sa=mixed, sw=sw, a=a, w=w)[-1]
        keep = torch.arange(M, device="cuda") % 3 != 0
        assert torch.equal(got[keep], alone[keep])


def test_layers_of_small_values_against_large_ones(gf):
    """Rows of magnitude 1e-34 to 1e-36 through a layer with weights of 0.05, and the same values times 2^100: a power of two changes no
    code, and of the results what is subnormal on the way (2^-150 for each of five chunks and the result) and the roundings that
    follow, one step, 2^-23 of the row's largest result, for each of the six sums at most."""
    for M in (20, 9000):
        x = torch.randn(M, 576, device="cuda", generator=torch.Generator("cuda").manual_seed(M))
        x *= torch.exp2(-torch.arange(M, device="cuda").remainder(6).float() - 112)[:, None]
        small, large = gf.quantize_rows(x), gf.quantize_rows(x * 2.0 ** 100)
        assert torch.equal(small.codes, large.codes)
        layer = gf.Fp8Linear(torch.randn(640, 576, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 0.05)
        y, want = layer(x).double(), layer(x * 2.0 ** 100).double() * 2.0 ** -100
        assert bool(((y - want).abs() <= 6 * 2 * U * want.abs().amax(1, keepdim=True) + 6 * 2.0 ** -150).all())
