"""GPU parity of layer normalisation (gf_train.h) with a plain implementation in 64 bits.

Bounds, u = 2^-24 the unit roundoff of fp32:
  y, g_x   error relative to the tensor's largest magnitude: fp32 2e-5 (sums of C terms on paths of at
           most 50 additions, 3e-6, times the spread max|x| / sigma of a row, at most 6 here); bf16
           adds one rounding of the result, 2^-9 of an element: 2^-8.  g_x = rstd (h - mean h - xh mean(h xh))
           may cancel (for C = 2 it is zero but for eps), so its 2e-5 is of the largest sum of the three
           magnitudes.
  sums     |error| <= 128 u sum |terms| per channel: at most 100 additions lie between a term and the
           sum, and a term itself carries a few roundings.
"""
import numpy as np
import pytest
import torch

from parity_util import Guarded, f64, relerr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TOL = {torch.float32: 2e-5, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float32, torch.bfloat16]


def _draw(shape, seed, dtype=torch.float32, scale=1.0, shift=0.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype)


def _plain(x, gamma, beta, eps, gy=None, given=None):
    """Rows [R, C] in fp64: y, mean, rstd and, for gy, g_x, g_gamma, g_beta and the sums of magnitudes.
    given: the (mean, rstd) that the backward call is handed, instead of the exact ones."""
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    xh = (x - mean) * rstd
    out = {"y": xh * gamma + beta, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if gy is not None:
        if given is not None:
            mean, rstd = (v[:, None] for v in given)
            xh = (x - mean) * rstd
        h = gy * gamma
        out["gx"] = rstd * (h - h.mean(1, keepdims=True) - xh * (h * xh).mean(1, keepdims=True))
        out["gx_terms"] = (rstd * (np.abs(h) + np.abs(h.mean(1, keepdims=True))
                                   + np.abs(xh * (h * xh).mean(1, keepdims=True)))).max()
        out["ggamma"], out["gbeta"] = (gy * xh).sum(0), gy.sum(0)
        out["ggamma_abs"], out["gbeta_abs"] = np.abs(gy * xh).sum(0), np.abs(gy).sum(0)
    return out


def _rows(t, nchw):
    """The tensor [N, C, H, W] / [N, H, W, C] as fp64 rows [R, C]."""
    a = f64(t)
    return (a.transpose(0, 2, 3, 1) if nchw else a).reshape(-1, a.shape[1] if nchw else a.shape[-1])


def _run(gf, x, gy, gamma, beta, nchw, eps=1e-5, inplace=False):
    if nchw:
        N, C, H, W = x.shape
    else:
        N, H, W, C = x.shape
    desc = gf.make_norm_desc(N, C, H, W, dtype=x.dtype, param_dtype=gamma.dtype if gamma is not None else torch.float32,
                             layout=gf.GF_NCHW if nchw else gf.GF_NHWC, eps=eps)
    R = N * H * W
    y, gx = Guarded(x.shape, x.dtype), Guarded(x.shape, x.dtype)
    mean, rstd = Guarded((R,), torch.float32), Guarded((R,), torch.float32)
    gw, gb = Guarded((C,), torch.float32), Guarded((C,), torch.float32)
    ws = Guarded((gf.gf_layer_norm_backward_workspace_bytes(desc),), torch.uint8)
    before = gf.gf_kernel_launch_count()
    src = x
    if inplace:
        y.t.copy_(x)
        gx.t.copy_(gy)
        src, gy_src = y.t, gx.t
    else:
        gy_src = gy
    gf.gf_layer_norm_forward(desc, src, gamma, beta, y.t, mean.t, rstd.t)
    gf.gf_layer_norm_backward(desc, gy_src, x, gamma, mean.t, rstd.t, gx.t, gw.t, gb.t, ws.t)
    assert gf.gf_last_async_status(ws.t) == gf.GF_OK
    assert gf.gf_kernel_launch_count() >= before + 3
    for g in (y, gx, mean, rstd, gw, gb, ws):
        g.check()
    return y.t, mean.t, rstd.t, gx.t, gw.t, gb.t


def _check(got, x, gy, gamma, beta, nchw, eps=1e-5):
    y, mean, rstd, gx, gw, gb = got
    C = x.shape[1] if nchw else x.shape[-1]
    ref = _plain(_rows(x, nchw), f64(gamma) if gamma is not None else np.ones(C), f64(beta) if beta is not None else np.zeros(C),
                 eps, _rows(gy, nchw), (f64(mean), f64(rstd)))
    tol = TOL[x.dtype]
    assert relerr(_rows(y, nchw), ref["y"]) <= tol
    assert relerr(f64(mean), ref["mean"]) <= TOL[torch.float32]
    assert relerr(f64(rstd), ref["rstd"]) <= TOL[torch.float32]
    bound = TOL[torch.float32] * ref["gx_terms"] + (tol * np.abs(ref["gx"]).max() if x.dtype == torch.bfloat16 else 0)
    assert np.abs(_rows(gx, nchw) - ref["gx"]).max() <= bound
    for g, name in ((gw, "ggamma"), (gb, "gbeta")):
        assert (np.abs(f64(g) - ref[name]) <= 128 * U * ref[name + "_abs"] + 1e-30).all(), name


# widths that meet each way a row is shared out, and their neighbours: odd widths, one element, a
# vector more or less than a warp or a block holds, rows that do not fit the registers
ROWS = [(1, 2), (3, 3), (7, 8), (33, 31), (300, 64), (257, 100), (5, 255), (130, 257), (64, 768), (301, 1001), (40, 1024),
        (17, 1025), (9, 2056), (700, 2048), (3, 4096), (5, 8190), (6, 8192), (3, 8200), (2, 16384), (3, 20001), (2, 33000), (1, 40000)]


# many rows: batches of rows in flight per team of threads, rows that start anywhere in a 16-byte piece, a
# tensor whose size is no multiple of 16 bytes, one team per block
ROWS += [(20001, 19), (30000, 1), (9001, 96), (6001, 257), (5003, 1001), (2500, 4096), (1500, 8192), (1201, 7001), (700, 16384), (40000, 8)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("R,C", ROWS, ids=lambda v: str(v))
def test_rows(gf, R, C, dtype):
    pdt = DTYPES[C % 2]
    x, gy = _draw((R, 1, 1, C), 1, dtype, 1.5, 0.7).cuda(), _draw((R, 1, 1, C), 2, dtype, 0.1).cuda()
    gamma, beta = _draw((C,), 3, pdt, 0.3, 1.0).cuda(), _draw((C,), 4, pdt, 0.3).cuda()
    _check(_run(gf, x, gy, gamma, beta, False), x, gy, gamma, beta, False)


PLANES = [(1, 1, 1, 1), (2, 3, 1, 1), (2, 5, 1, 2), (3, 8, 7, 7), (2, 33, 5, 5), (1, 96, 9, 11), (4, 64, 14, 14), (2, 100, 16, 16),
          (3, 130, 6, 6), (2, 256, 7, 7), (1, 257, 4, 4), (2, 511, 3, 5), (2, 512, 8, 8), (1, 513, 6, 6), (1, 1024, 3, 3),
          (2, 1500, 4, 4), (1, 2100, 5, 5), (1, 2048, 4, 8), (3, 700, 13, 13), (40, 130, 31, 33), (300, 64, 16, 16), (1, 12, 56, 57), (64, 96, 28, 28), (5, 16, 33, 31)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", PLANES, ids=lambda s: "x".join(map(str, s)))
def test_planes(gf, shape, dtype):
    C = shape[1]
    pdt = DTYPES[(C + 1) % 2]
    x, gy = _draw(shape, 5, dtype, 1.5, 0.7).cuda(), _draw(shape, 6, dtype, 0.1).cuda()
    gamma, beta = _draw((C,), 7, pdt, 0.3, 1.0).cuda(), _draw((C,), 8, pdt, 0.3).cuda()
    _check(_run(gf, x, gy, gamma, beta, True), x, gy, gamma, beta, True)


@pytest.mark.parametrize("nchw,shape", [(False, (37, 1, 1, 200)), (True, (3, 40, 5, 7)), (False, (4, 6, 6, 24))])
def test_in_place_and_without_parameters(gf, nchw, shape):
    x, gy = _draw(shape, 9, shift=0.3).cuda(), _draw(shape, 10).cuda()
    _check(_run(gf, x, gy, None, None, nchw, inplace=True), x, gy, None, None, nchw)


@pytest.mark.parametrize("nchw", [False, True])
def test_one_channel_and_constant_rows(gf, nchw):
    """C = 1: xh = 0, so y = beta, g_x = 0, g_gamma = 0.  Constant rows: the same with eps > 0."""
    for C in (1, 48):
        shape = (5, C, 3, 3) if nchw else (5, 3, 3, C)
        x = torch.full(shape, 3.25, device="cuda")
        gy = _draw(shape, 11).cuda()
        gamma, beta = _draw((C,), 12).cuda(), _draw((C,), 13).cuda()
        y, mean, rstd, gx, gw, gb = _run(gf, x, gy, gamma, beta, nchw)
        assert bool((mean == 3.25).all())
        assert torch.equal(_t_rows(y, nchw), beta.expand(45, C))
        assert bool((gw == 0).all())
        if C == 1:
            assert bool((gx.abs() <= 1e-4 * gy.abs().max() * 316.3).all())


def _t_rows(t, nchw):
    return (t.permute(0, 2, 3, 1) if nchw else t).reshape(-1, t.shape[1] if nchw else t.shape[-1])


@pytest.mark.parametrize("nchw", [False, True])
def test_a_large_offset_does_not_cancel(gf, nchw):
    """Rows of mean 1000 and deviation 1: a difference of mean squares would lose 20 of 24 bits.
    The mean carries at most 50 u * 1000 = 3e-3 worst, typically 1e-4; bound 1e-3 on y of size 4."""
    shape = (6, 96, 5, 5) if nchw else (6, 5, 5, 96)
    x, gy = _draw(shape, 14, shift=1000.0).cuda(), _draw(shape, 15).cuda()
    y = _run(gf, x, gy, None, None, nchw)[0]
    ref = _plain(_rows(x, nchw), np.ones(96), np.zeros(96), 1e-5)
    assert np.abs(_rows(y, nchw) - ref["y"]).max() <= 1e-3


@pytest.mark.parametrize("nchw", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_non_finite_value_stays_in_its_row(gf, nchw, bad):
    shape = (4, 40, 3, 5) if nchw else (4, 3, 5, 40)
    x, gy = _draw(shape, 16).cuda(), _draw(shape, 17).cuda()
    good = [t.clone() for t in _run(gf, x, gy, None, None, nchw)]
    x.view(-1)[0] = bad
    got = _run(gf, x, gy, None, None, nchw)
    for k in (0, 3):
        a, b = _t_rows(got[k], nchw), _t_rows(good[k], nchw)
        assert not bool(torch.isfinite(a[0]).any()) and torch.equal(a[1:], b[1:])
    assert torch.equal(got[5], good[5]) and not bool(torch.isfinite(got[4]).any())


def test_zero_rows(gf):
    desc = gf.make_norm_desc(0, 24)
    gw, gb = torch.full((24,), 7.0, device="cuda"), torch.full((24,), 7.0, device="cuda")
    gf.gf_layer_norm_forward(desc, None, None, None, None)
    gf.gf_layer_norm_backward(desc, None, None, None, None, None, None, gw, gb, None)
    torch.cuda.synchronize()
    assert bool((gw == 0).all()) and bool((gb == 0).all())


@pytest.mark.parametrize("nchw,shape", [(False, (2000, 1, 1, 768)), (True, (8, 96, 28, 28))])
def test_results_repeat_bit_for_bit_and_outputs_may_be_left_out(gf, nchw, shape):
    x, gy = _draw(shape, 18).cuda(), _draw(shape, 19).cuda()
    C = shape[1] if nchw else shape[-1]
    gamma = _draw((C,), 20).cuda()
    first = _run(gf, x, gy, gamma, None, nchw)
    again = _run(gf, x, gy, gamma, None, nchw)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    N, H, W = (shape[0], shape[2], shape[3]) if nchw else shape[:3]
    desc = gf.make_norm_desc(N, C, H, W, layout=gf.GF_NCHW if nchw else gf.GF_NHWC)
    ws = torch.empty(gf.gf_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    y, gx, gw, gb = torch.empty_like(x), torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    gf.gf_layer_norm_forward(desc, x, gamma, None, y)
    gf.gf_layer_norm_backward(desc, gy, x, gamma, first[1], first[2], gx, None, None, None)
    gf.gf_layer_norm_backward(desc, gy, x, gamma, first[1], first[2], None, gw, None, ws)
    gf.gf_layer_norm_backward(desc, gy, x, gamma, first[1], first[2], None, None, gb, ws)
    assert torch.equal(y, first[0]) and torch.equal(gx, first[3]) and torch.equal(gw, first[4]) and torch.equal(gb, first[5])


@pytest.mark.parametrize("channel_dim,shape", [(-1, (6, 10, 48)), (1, (3, 24, 5, 6))])
def test_gradients_against_differences(gf, channel_dim, shape):
    """Central differences of L = sum(y v) along a random direction, steps of 1e-2: truncation h^2 / 6
    times a third derivative of order 10, and rounding u sqrt(n) / h: below 1e-3 of the slope's scale."""
    C = shape[channel_dim]
    x, v = _draw(shape, 21).cuda(), _draw(shape, 22).cuda()
    w, b = _draw((C,), 23, scale=0.3, shift=1.0).cuda(), _draw((C,), 24).cuda()
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    (gf.layer_norm(*leaves, channel_dim=channel_dim) * v).sum().backward()
    for k in range(3):
        d = _draw(leaves[k].shape, 25 + k).cuda()

        def loss(sign):
            moved = [t.detach() for t in leaves]
            moved[k] = moved[k] + sign * 1e-2 * d
            return float((gf.layer_norm(*moved, channel_dim=channel_dim).double() * v.double()).sum())

        slope = (loss(1) - loss(-1)) / 2e-2
        want = float((leaves[k].grad.double() * d.double()).sum())
        scale = float(leaves[k].grad.double().norm() * d.double().norm())
        assert abs(slope - want) <= 2e-3 * scale, (k, slope, want)


@pytest.mark.parametrize("form", ["rows", "strided", "unaligned", "nchw", "channels_last", "empty", "other_stream"])
def test_module_through_autograd(gf, form):
    C = 24
    cd = 1 if form in ("nchw", "channels_last") else -1
    if cd == 1:
        x = _draw((3, C, 6, 5), 30).cuda()
        if form == "channels_last":
            x = x.contiguous(memory_format=torch.channels_last)
    elif form == "strided":
        x = _draw((C, 35), 31).cuda().t()
    elif form == "unaligned":
        x = _draw((35 * C + 1,), 32).cuda()[1:].view(35, C)
    elif form == "empty":
        x = torch.empty((0, C), device="cuda")
    else:
        x = _draw((5, 7, C), 33).cuda()
    m = gf.LayerNorm(C, channel_dim=cd, device="cuda")
    with torch.no_grad():
        m.weight.copy_(_draw((C,), 34, shift=1.0))
        m.bias.copy_(_draw((C,), 35))
    xa = x.clone(memory_format=torch.preserve_format).requires_grad_(True) if form != "unaligned" else x.requires_grad_(True)
    gy = torch.randn_like(x.detach())
    side = torch.cuda.Stream() if form == "other_stream" else torch.cuda.current_stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = m(xa)
        y.backward(gy)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert y.shape == x.shape and y.dtype == x.dtype
    if form == "empty":
        assert bool((m.weight.grad == 0).all()) and xa.grad.shape == x.shape
        return
    to_rows = (lambda t: f64(t.permute(0, 2, 3, 1)).reshape(-1, C)) if cd == 1 else (lambda t: f64(t).reshape(-1, C))
    ref = _plain(to_rows(x), f64(m.weight), f64(m.bias), m.eps, to_rows(gy))
    assert relerr(to_rows(y), ref["y"]) <= 2e-5 and relerr(to_rows(xa.grad), ref["gx"]) <= 2e-5
    assert relerr(f64(m.weight.grad), ref["ggamma"]) <= 2e-5 and relerr(f64(m.bias.grad), ref["gbeta"]) <= 2e-5
    if form == "channels_last":
        assert y.is_contiguous(memory_format=torch.channels_last) and xa.grad.is_contiguous(memory_format=torch.channels_last)


def test_more_elements_than_32_bits_count(gf):
    """270001 rows of 8192 (2.2e9 elements): the last rows against a plain form on the device, the rest by their statistics."""
    R, C = 270001, 8192
    g = torch.Generator(device="cuda")
    g.manual_seed(40)
    x = torch.empty((R, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    desc = gf.make_norm_desc(R, C, dtype=torch.bfloat16)
    y, mean, rstd = torch.empty_like(x), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    gf.gf_layer_norm_forward(desc, x, None, None, y, mean, rstd)
    ws = torch.empty(gf.gf_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    gw, gb, gx = torch.empty(C, device="cuda"), torch.empty(C, device="cuda"), torch.empty_like(x)
    gf.gf_layer_norm_backward(desc, y, x, None, mean, rstd, gx, gw, gb, ws)          # g_y = y
    torch.cuda.synchronize()
    tail = x[-3:].double()
    xh = (tail - tail.mean(1, keepdim=True)) / (tail.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    assert float((y[-3:].double() - xh).abs().max()) <= 2.0 ** -8 * float(xh.abs().max())
    assert float((mean.double().mean())) == pytest.approx(0.0, abs=1e-4) and float(rstd.double().mean()) == pytest.approx(1.0, abs=1e-3)
    # g_y = y = xh (rounded): g_x is what is left of it, rounding; g_gamma sums xh^2
    assert float(gx[-3:].float().abs().max()) <= 2.0 ** -8 * float(xh.abs().max()) * 3
    assert float((gw.double() / R - 1).abs().max()) <= 0.02
    del x, y, gx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("nchw,shape", [(False, (3000, 1, 1, 768)), (True, (8, 96, 28, 28))])
def test_calls_can_be_captured_in_a_graph(gf, nchw, shape):
    x, gy = _draw(shape, 41).cuda(), _draw(shape, 42).cuda()
    want = _run(gf, x, gy, None, None, nchw)                     # first calls set function attributes
    N, H, W = (shape[0], shape[2], shape[3]) if nchw else shape[:3]
    C = shape[1] if nchw else shape[-1]
    desc = gf.make_norm_desc(N, C, H, W, layout=gf.GF_NCHW if nchw else gf.GF_NHWC)
    ws = torch.empty(gf.gf_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(t) for t in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gf.gf_layer_norm_forward(desc, x, None, None, out[0], out[1], out[2])
        gf.gf_layer_norm_backward(desc, gy, x, None, out[1], out[2], out[3], out[4], out[5], ws)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, want):
        assert torch.equal(a, b)
