"""8-bit matrices and their products (gf_block.h) against the formulas in 64 bits.

Quantisers: scales are the largest magnitude times 1 / 448, both in fp32; codes are compared for equality with the value divided by the
stored scale in fp32 and rounded to the nearest e4m3 value, ties to even (a table search on the host).

Products: codes and scales are given, so that products of codes are exact.  A chunk's 128 additions on the tensor cores are
off by at most one step of fp32 each, 2^-23 of the chunk's sum of magnitudes; scaling, adding chunks and the bias
add half a step for each chunk and four more: (128 * 2^-23 + (chunks + 4) 2^-24) sum |terms|, and half a step of the result's type."""
import numpy as np
import pytest
import torch

from block_util import DTYPES, STEP, U, draw, e4m3_codes, e4m3_values, random_codes
from parity_util import Guarded, f64

pytestmark = pytest.mark.gpu


def _amax(a, R, C, blocks):
    G, B = -(-C // 128), -(-R // 128) if blocks else R
    p = np.zeros((B * (128 if blocks else 1), G * 128), dtype=np.float32)
    p[:R, :C] = np.abs(a)
    p = p.reshape(B, -1, G, 128)
    return p.max((1, 3))                                                    # NaN where a group holds one


def _check_codes(x, codes, scales, blocks):
    """codes [R, pitch] and scales as the library wrote them, against x [R, C] in fp32 on the host."""
    a = x.float().cpu().numpy()
    R, C = a.shape
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    assert (c[:, C:] == 0).all()
    top = _amax(a, R, C, blocks)
    s = s if blocks else s[:, :R].T
    with np.errstate(invalid="ignore"):
        want = np.maximum(top * (np.float32(1) / np.float32(448)), np.float32(2.0 ** -126))
        want = np.where(np.isfinite(top), want, top)
    assert np.array_equal(s, want, equal_nan=True)
    wide = np.repeat(np.repeat(s, 128, 0)[:R] if blocks else s, 128, 1)[:, :C]
    with np.errstate(invalid="ignore", over="ignore"):
        q = (a / wide).astype(np.float32)
    q = np.where(np.isfinite(wide), np.clip(q, -448, 448), np.nan)
    assert np.array_equal(c[:, :C] & (127 if not np.isfinite(top).all() else 255),
                          e4m3_codes(q) & (127 if not np.isfinite(top).all() else 255))


def _values(R, C, seed, dtype):
    """Rows that span many binary orders, with zeros, ties (powers of two) and a row of zeros among them."""
    x = draw((R, C), seed) * torch.exp2(draw((R, 1), seed + 1, scale=8.0).round())
    x = torch.where(draw((R, C), seed + 2) > 1.5, torch.exp2(draw((R, C), seed + 3, scale=3.0).round()) * 448, x)
    x = torch.where(draw((R, C), seed + 4) > 1.8, torch.zeros(()), x)
    x[R // 2] = 0
    if R > 3:
        x[R - 1] *= 2.0 ** -120                                             # scales at their smallest
    return x.to(dtype)


SHAPES = [(1, 1), (2, 7), (3, 8), (17, 127), (16, 128), (15, 129), (33, 500), (7, 512), (40, 513), (130, 257), (300, 1001), (64, 4096), (5, 4100), (20001, 24), (3, 20000)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("R,C", SHAPES, ids=lambda v: str(v))
def test_quantisers(gf, R, C, dtype):
    x = _values(R, C, 1, dtype).cuda()
    desc = gf.make_fp8_desc(R, C, dtype=dtype)
    codes = Guarded((R, gf.fp8_pitch(C)), torch.uint8)
    scales = Guarded((-(-C // 128), gf.fp8_scale_pitch(R)), torch.float32)
    gf.gf_fp8_quantize_rows(desc, x, codes.t, scales.t)
    _check_codes(x, codes.t, scales.t, False)
    assert bool((scales.t[:, R:] == 12345.0).all()), "places behind the last row"
    codes.check()
    scales.check()
    codes, scales = Guarded((R, gf.fp8_pitch(C)), torch.uint8), Guarded((-(-R // 128), -(-C // 128)), torch.float32)
    gf.gf_fp8_quantize_blocks(desc, x, codes.t, scales.t)
    _check_codes(x, codes.t, scales.t, True)
    codes.check()
    scales.check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("C", [100, 256, 333])
def test_a_non_finite_value_spoils_its_group_alone(gf, C, bad):
    x = draw((9, C), 3).cuda()
    good = gf.quantize_rows(x).dequantize()
    x[4, 70] = bad
    got = gf.quantize_rows(x)
    assert bool((got.codes[:, C:] == 0).all())
    v = got.dequantize()
    assert not bool(torch.isfinite(v[4, :128]).any())
    v[4, :128] = good[4, :128]
    assert torch.equal(v, good)
    w = gf.quantize_weight(x).dequantize()
    assert not bool(torch.isfinite(w[:, :128]).any()) and bool(torch.isfinite(w[:, 128:]).all())


def test_quotients_are_those_of_a_division(gf):
    """Values whose quotient by the scale lies on or beside a border between two codes, for many scales."""
    R = 4096
    g = np.random.RandomState(5)
    top = (1 + g.rand(R)).astype(np.float32) * np.exp2(g.randint(-60, 60, R)).astype(np.float32)
    table = e4m3_values(np.arange(127, dtype=np.uint8))
    borders = ((table[1:] + table[:-1]) / 2).astype(np.float32)
    scale = (top * (np.float32(1) / np.float32(448)))[:, None]
    v = (borders[None, :125] * scale).astype(np.float32)                   # as near as fp32 comes to a border
    step = g.randint(-1, 2, v.shape)
    v = np.where(step > 0, np.nextafter(v, np.float32(np.inf)), np.where(step < 0, np.nextafter(v, np.float32(0)), v))
    x = torch.from_numpy(np.concatenate([top[:, None], v], 1)).cuda()
    q = gf.quantize_rows(x)
    _check_codes(x, q.codes, q.scales, False)


def _product(gf, M, N, K, transposed, out, bias=None, seed=1, sa=None, sw=None, a=None, w=None):
    inner, outer = (N, K) if transposed else (K, N)
    a = random_codes(M, inner, seed) if a is None else a
    w = random_codes(N, K, seed + 1) if w is None else w
    g = np.random.RandomState(seed + 2)
    sp = -(-M // 4) * 4
    sa = np.exp2(g.randint(-8, 3, (-(-inner // 128), sp)) + g.rand(-(-inner // 128), sp)).astype(np.float32) if sa is None else sa
    sw = np.exp2(g.randint(-12, -6, (-(-N // 128), -(-K // 128))) + g.rand(-(-N // 128), -(-K // 128))).astype(np.float32) if sw is None else sw
    sa[:, M:] = np.nan                                                     # not to be used
    at = Guarded(a.shape, torch.uint8)
    at.t.copy_(torch.from_numpy(a))
    y = Guarded((M, outer), out)
    b = None if bias is None else draw((outer,), seed + 3, bias, 2.0).cuda()
    desc = gf.make_fp8_matmul_desc(M, N, K, transposed=transposed, out_dtype=out, bias_dtype=torch.float32 if bias is None else bias)
    wd, sad, swd = (torch.from_numpy(t).cuda() for t in (w, sa, sw))
    gf.gf_fp8_matmul(desc, at.t, sad, wd, swd, b, y.t)
    assert gf.gf_last_async_status(torch.zeros(256, dtype=torch.uint8, device="cuda")) == gf.GF_OK
    y.check()
    return a, w, sa, sw, b, y.t


def _check_product(a, w, sa, sw, b, y, transposed):
    M, outer = a.shape[0], y.shape[1]
    wv = e4m3_values(w) * np.repeat(np.repeat(sw, 128, 0)[:w.shape[0]], 128, 1)[:, :w.shape[1]]
    wv = wv[:, :outer] if transposed else wv.T
    inner = wv.shape[0]
    av = e4m3_values(a[:, :inner]) * np.repeat(sa[:, :M].T, 128, 1)[:, :inner]
    if not transposed:                                                     # the codes behind the last column
        av, wv = np.nan_to_num(av, nan=0.0), np.nan_to_num(wv, nan=0.0)
    t_a, t_w = torch.from_numpy(av).cuda(), torch.from_numpy(np.ascontiguousarray(wv)).cuda()
    ref, mag = t_a @ t_w, t_a.abs() @ t_w.abs()
    if b is not None:
        ref, mag = ref + b.double(), mag + b.double().abs()
    chunks = -(-inner // 128)
    got = y.double()
    bound = (128 * 2 * U + (chunks + 4) * U) * mag + STEP[y.dtype] * ref.abs()
    assert bool(((got - ref).abs() <= bound).all()), float(((got - ref).abs() / bound.clamp_min(1e-300)).max())


# few and many rows around the tiles' sizes, odd sizes in every place, one chunk and many, cut in parts or not
PRODUCTS = [(1, 1, 1), (1, 128, 128), (2, 5, 3), (7, 130, 129), (8, 768, 2304), (15, 300, 77), (16, 128, 1000), (17, 200, 512), (32, 1001, 576), (33, 96, 96),
            (64, 640, 384), (65, 257, 1300), (100, 4096, 4096), (127, 129, 127), (128, 128, 128), (129, 1001, 300), (255, 513, 257), (256, 256, 256),
            (257, 300, 4100), (300, 64, 8192), (300, 8192, 64), (777, 999, 555), (1024, 1024, 1024), (2000, 96, 576), (4099, 1001, 576), (5000, 16, 40)]


@pytest.mark.parametrize("transposed", [False, True], ids=["layer", "input_gradient"])
@pytest.mark.parametrize("M,N,K", PRODUCTS, ids=lambda v: str(v))
def test_products(gf, M, N, K, transposed):
    k = M + N + K
    out, bias = DTYPES[k % 2], (None, *DTYPES)[k % 3]
    _check_product(*_product(gf, M, N, K, transposed, out, bias, seed=k), transposed)


@pytest.mark.parametrize("transposed", [False, True], ids=["layer", "input_gradient"])
def test_integers_are_exact(gf, transposed):
    """Codes of whole numbers up to 8 and scales of one: sums below 2^24 come out exactly, at every place."""
    for M, N, K in ((33, 260, 300), (700, 520, 390)):
        g = np.random.RandomState(1)
        whole = np.array([0, 0x38, 0x40, 0x44, 0x48, 0x4A, 0x4C, 0x4E, 0x50], dtype=np.uint8)       # 0, 1, 2, 3, 4, 5, 6, 7, 8
        assert np.array_equal(e4m3_values(whole), np.arange(9))
        inner, outer = (N, K) if transposed else (K, N)
        a = np.zeros((M, -(-inner // 16) * 16), dtype=np.uint8)
        w = np.zeros((N, -(-K // 16) * 16), dtype=np.uint8)
        a[:, :inner], w[:, :K] = whole[g.randint(0, 9, (M, inner))], whole[g.randint(0, 9, (N, K))]
        sa, sw = np.ones((-(-inner // 128), -(-M // 4) * 4), np.float32), np.ones((-(-N // 128), -(-K // 128)), np.float32)
        y = _product(gf, M, N, K, transposed, torch.float32, sa=sa, sw=sw, a=a, w=w)[-1]
        av, wv = e4m3_values(a)[:, :inner], e4m3_values(w)[:, :K]
        assert np.array_equal(f64(y), av @ (wv if transposed else wv.T))


def test_a_nan_stays_in_its_row_and_column(gf):
    for M, N, K in ((40, 300, 256), (600, 300, 256)):
        a, w = random_codes(M, K, 1), random_codes(N, K, 2)
        good = _product(gf, M, N, K, False, torch.float32, a=a, w=w)[-1]
        a[5, 100], w[7, 3] = 127, 255
        got = _product(gf, M, N, K, False, torch.float32, a=a, w=w)[-1]
        bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
        bad[5], bad[:, 7] = True, True
        assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], good[~bad])


def test_no_rows(gf):
    gf.gf_fp8_quantize_rows(gf.make_fp8_desc(0, 64), None, None, None)
    gf.gf_fp8_matmul(gf.make_fp8_matmul_desc(0, 64, 64), None, None, None, None, None, None)
    layer = gf.Fp8Linear(draw((48, 64), 1).cuda())
    x = torch.empty((0, 64), device="cuda", requires_grad=True)
    y = layer(x)
    y.sum().backward()
    assert y.shape == (0, 48) and x.grad.shape == (0, 64)


def test_offsets_past_32_bits(gf):
    """A of 2.2e9 codes and a result of 2.3e9 values: the last rows and a few in between."""
    M, N, K = 4_300_003, 528, 520
    q = torch.randint(0, 120, (M, 528), dtype=torch.uint8, device="cuda")
    sa = torch.rand((5, M + 1), device="cuda") + 0.5
    w = random_codes(N, K, 3)
    sw = np.random.RandomState(4).rand(5, 5).astype(np.float32)
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    gf.gf_fp8_matmul(gf.make_fp8_matmul_desc(M, N, K), q, sa, torch.from_numpy(w).cuda(), torch.from_numpy(sw).cuda(), None, out)
    for first in (0, (1 << 31) // 528 - 3, M - 7):
        a, s = q[first:first + 7].cpu().numpy(), sa[:, first:first + 7].cpu().numpy()
        _check_product(a, w, s, sw, None, out[first:first + 7], False)
    x = torch.randn((M, K), device="cuda").bfloat16()
    codes, scales = q, sa
    gf.gf_fp8_quantize_rows(gf.make_fp8_desc(M, K, dtype=torch.bfloat16), x, codes, scales)
    _check_codes(x[-5:], codes[-5:], scales[:, M - 5:M], False)
    del q, x, out, codes
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M", [9, 700])
def test_results_repeat_bit_for_bit_and_in_a_graph(gf, M):
    x, layer = draw((M, 520), 1).cuda(), gf.Fp8Linear(draw((264, 520), 2).cuda(), draw((264,), 3).cuda())
    first = layer(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, first) and torch.equal(layer(x), first)


def test_two_streams_at_once(gf):
    """Products of different kinds side by side on streams of their own give what they give alone."""
    shapes = [(4, 512, 1024), (100, 640, 2048), (700, 512, 512), (1500, 768, 384)]
    work = [(draw((m, k), i).cuda(), gf.Fp8Linear(draw((n, k), i + 9).cuda())) for i, (m, n, k) in enumerate(shapes)]
    alone = [layer(x) for x, layer in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(20):
        got = []
        for s, (x, layer) in zip(streams, work):
            with torch.cuda.stream(s):
                got.append(layer(x))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("form", ["rows", "bf16", "3d", "strided", "unaligned", "map", "channels_last", "cast", "copied"])
def test_frozen_layer_through_autograd(gf, form):
    """y and the gradient of x against products of the dequantised operands."""
    K, N = 200, 136
    w, b = draw((N, K), 1, scale=K ** -0.5).cuda(), draw((N,), 2).cuda()
    if form in ("map", "channels_last"):
        conv = gf.FilteredConv2d(K, N, 1, device="cuda")
        with torch.no_grad():
            conv.weight.copy_(w.view(N, K, 1, 1))
            conv.bias.copy_(b)
        layer = gf.Fp8Linear.from_layer(conv)
        x = draw((3, K, 5, 7), 3).cuda()
        if form == "channels_last":
            x = x.contiguous(memory_format=torch.channels_last)
    else:
        lin = torch.nn.Linear(K, N, device="cuda")
        with torch.no_grad():
            lin.weight.copy_(w)
            lin.bias.copy_(b)
        layer = gf.Fp8Linear.from_layer(lin)
        x = {"3d": lambda: draw((4, 9, K), 3), "strided": lambda: draw((K, 30), 3).t(), "unaligned": lambda: draw((30 * K + 1,), 3)[1:].view(30, K)}.get(
            form, lambda: draw((30, K), 3))().cuda()
    if form == "bf16":
        x = x.bfloat16()
    elif form == "cast":
        layer = layer.to(torch.bfloat16).cuda()
        assert layer.scales.dtype == torch.float32 and layer.codes.dtype == torch.uint8 and layer.bias.dtype == torch.bfloat16
    elif form == "copied":
        import copy
        other = gf.Fp8Linear(torch.zeros((N, K), device="cuda"), torch.zeros(N, device="cuda"))
        other.load_state_dict(copy.deepcopy(layer).state_dict())
        layer = other
    assert not list(layer.parameters())
    x = x.detach().requires_grad_(True)
    y = layer(x)
    gy = torch.randn_like(y)
    y.backward(gy)
    rows = (lambda t: t.permute(0, 2, 3, 1).reshape(-1, t.shape[1])) if x.dim() == 4 else (lambda t: t.reshape(-1, t.shape[-1]))
    W = layer.matrix().dequantize().double()
    ref = gf.quantize_rows(rows(x)).dequantize().double() @ W.t() + layer.bias.double()
    gref = gf.quantize_rows(rows(gy)).dequantize().double() @ W
    assert y.dtype == x.dtype and x.grad.shape == x.shape
    if form == "channels_last":
        assert y.is_contiguous(memory_format=torch.channels_last)
    for got, want in ((y, ref), (x.grad, gref)):
        # the bound of the products, with at most 200 terms of at most 4 deviations each under the sum of magnitudes
        assert float((rows(got.detach()).double() - want).abs().max()) <= (STEP[x.dtype] + 150 * U * 20) * float(want.abs().max())
    # and the layer is what it stands for: each operand is off by at most 2^-4 of its values, about 2.6 % of its norm
    exact = rows(x.detach()).double() @ w.double().t() + layer.bias.double()
    assert float((rows(y.detach()).double() - exact).norm() / exact.norm()) < 2.0 ** -4 * 2


@pytest.mark.parametrize("out", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1300, 328, 200), (40000, 160, 136), (9000, 488, 264), (20001, 72, 300), (2500, 2120, 96)], ids=lambda v: str(v))
def test_products_of_many_tiles(gf, M, N, K, out):
    """More tiles than the SMs take at once, with last tiles that lack rows and columns: a column part that is missing in
    some tiles only, results that leave by the copy engine and by hand."""
    for transposed in (False, True):
        _check_product(*_product(gf, M, N, K, transposed, out, torch.float32, seed=M + N), transposed)


@pytest.mark.gpu
@pytest.mark.parametrize("normed", [False, True], ids=["layer", "norm_and_layer"])
def test_a_weight_changed_before_the_backward_pass_is_refused(gf, normed):
    """The gradient is that of the weight that ran forward, or an error as for torch's layers: never another weight's."""
    gen = torch.Generator().manual_seed(21)
    w, other = (torch.randn(96, 160, generator=gen).cuda() for _ in range(2))

    def forward(layer):
        x = torch.randn(40, 160, generator=torch.Generator().manual_seed(22)).cuda().requires_grad_()
        return x, gf.rms_norm_linear(x, None, layer) if normed else layer(x)

    x, y = forward(gf.Fp8Linear(w))
    y.sum().backward()
    layer = gf.Fp8Linear(w)
    x2, y2 = forward(layer)
    layer.load_state_dict(gf.Fp8Linear(other).state_dict())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y2.sum().backward()
    layer = gf.Fp8Linear(w)
    x3, y3 = forward(layer)
    layer.codes, layer.scales = gf.Fp8Linear(other).codes, gf.Fp8Linear(other).scales      # put in their place, the old ones live on
    y3.sum().backward()
    assert torch.equal(x3.grad, x.grad)
