"""Root-mean-square norm of a residual sum (gf_block.h) against the formulas in 64 bits.

Bounds, u = 2^-24:
  h        as dropout's: 3 u (|residual| + |x scale|) and half a step of h's type.  Everything after it is held against
           the h that the kernel kept, as that is what the norm is defined on.
  rstd, y  the squares are summed on paths of at most 64 additions of positive terms (24 per thread, 5 to 10 across
           threads, up to 33 of 1024 threads in long rows): 64 u of the sum, half of that after the root, with the
           roundings of the products 64 u in all; y adds half a step of its type.
  scales   64 u of y's largest magnitude and two roundings (of 1 / 448 and of the product); codes are off by half a step of e4m3, 2^-4 of the value or 2^-10
           of the scale, and 64 u of the value.
  g        128 u of rstd (|q| + |xh| mean |q xh|) + |g_h|, and half a step of the type.
  g_gamma  256 u of the sum of magnitudes: at most 200 additions lie between a term and the sum at these sizes."""
import numpy as np
import pytest
import torch

from block_util import DTYPES, STEP, U, draw, dropped, e4m3_values, seed_words
from parity_util import Guarded, f64

pytestmark = pytest.mark.gpu

PAIRS = [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)]
IDS = ["f32", "bf16_f32", "bf16"]
# each way a row is dealt out, and neighbours: one element, part of a warp, one to three octets per lane, blocks, rows that start
# anywhere in an octet, rows longer than a block's registers; few and many rows
ROWS = [(1, 1), (3, 2), (5, 7), (7, 8), (9, 9), (33, 31), (300, 64), (257, 100), (5, 127), (5, 128), (5, 129), (130, 257), (64, 512), (31, 520),
        (64, 768), (17, 769), (12, 775), (301, 1001), (40, 1024), (17, 1025), (9, 2056), (30, 2048), (5, 4090), (3, 4096), (5, 4097), (5, 8185), (6, 8192),
        (3, 8193), (4, 9000), (2, 16384), (11, 20001), (20001, 19), (9001, 96), (6001, 257), (2503, 1001), (1500, 4096), (700, 8192)]


def _gamma(C):
    return draw((C,), 3, DTYPES[C % 2], 0.3, 1.0).cuda()


def _forward(gf, R, C, xt, rt, p, residual=True, out8=False, x=None, res=None, gamma=None, eps=1e-5):
    x = draw((R, C), 1, xt).cuda() if x is None else x
    if residual and res is None:
        res = draw((R, C), 2, rt, 1.5, 0.3).cuda()
    seed, words = seed_words(R * 1000003 + C, C)
    desc = gf.make_rms_desc(R, C, dtype=xt, residual_dtype=rt if residual else xt, eps=eps, p=p,
                            param_dtype=torch.float32 if gamma is None else gamma.dtype)
    plain = not residual and p == 0
    h = None if plain else Guarded((R, C), rt if residual else xt)
    rstd = Guarded((R,), torch.float32)
    seed = seed if p > 0 else None
    if out8:
        codes = Guarded((R, gf.fp8_pitch(C)), torch.uint8)
        scales = Guarded((-(-C // 128), gf.fp8_scale_pitch(R)), torch.float32)
        gf.gf_rms_norm_forward_fp8(desc, x, res, seed, gamma, None if plain else h.t, codes.t, scales.t, rstd.t)
        out = (codes, scales)
    else:
        y = Guarded((R, C), xt)
        gf.gf_rms_norm_forward(desc, x, res, seed, gamma, None if plain else h.t, y.t, rstd.t)
        out = (y,)
    torch.cuda.synchronize()
    for g in (rstd, *out, *(() if plain else (h,))):
        g.check()
    # h against its definition, the rest against h
    want = dropped(f64(x), p, words)
    kept = x if plain else h.t
    if not plain:
        r = f64(res) if residual else 0.0
        assert (np.abs(f64(kept) - (want + r)) <= 3 * U * (np.abs(want) + np.abs(r)) + STEP[kept.dtype] * np.abs(want + r)).all()
    hk = f64(kept)
    ref_rstd = 1 / np.sqrt((hk ** 2).mean(1) + eps)
    assert (np.abs(f64(rstd.t) - ref_rstd) <= 64 * U * ref_rstd).all()
    ref = hk * ref_rstd[:, None] * (1.0 if gamma is None else f64(gamma))
    if not out8:
        assert (np.abs(f64(y.t) - ref) <= (64 * U + STEP[xt]) * np.abs(ref)).all()
        return x, kept, rstd.t, y.t, desc, seed, words
    G = -(-C // 128)
    top = np.stack([np.abs(ref[:, 128 * g:128 * g + 128]).max(1) for g in range(G)])
    s = f64(scales.t)
    assert (np.abs(s[:, :R] - np.maximum(top / 448, 2.0 ** -126)) <= 66 * U * np.maximum(top / 448, 2.0 ** -126)).all()
    assert (s[:, R:] == 12345.0).all(), "places behind the last row"
    c = codes.t.cpu().numpy()
    assert (c[:, C:] == 0).all()
    wide = np.repeat(s[:, :R].T, 128, 1)[:, :C]
    got = e4m3_values(c[:, :C]) * wide
    assert (np.abs(got - ref) <= 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * wide + 64 * U * np.abs(ref)).all()
    return x, kept, rstd.t, (codes.t, scales.t), desc, seed, words


@pytest.mark.parametrize("xt,rt", PAIRS, ids=IDS)
@pytest.mark.parametrize("R,C", ROWS, ids=lambda v: str(v))
def test_forward_with_residual_and_dropout(gf, R, C, xt, rt):
    _forward(gf, R, C, xt, rt, 0.1 * (C % 3), gamma=_gamma(C))


@pytest.mark.parametrize("xt,rt", PAIRS, ids=IDS)
@pytest.mark.parametrize("R,C", ROWS, ids=lambda v: str(v))
def test_forward_in_8_bits(gf, R, C, xt, rt):
    _forward(gf, R, C, xt, rt, 0.1 * ((C + 1) % 3), out8=True, gamma=_gamma(C))


@pytest.mark.parametrize("out8", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("R,C", [(4, 8), (70, 100), (33, 768), (9, 2001), (3, 9001), (2, 8200)])
def test_without_residual_and_without_gamma(gf, R, C, p, out8):
    for t in DTYPES:
        _forward(gf, R, C, t, t, p, residual=False, out8=out8)


def _check_backward(gf, R, C, xt, rt, p, want=("gres", "gx", "ggamma"), with_gh=True, gamma=None, alias=None):
    h, gy = draw((R, C), 5, rt, 1.5, 0.2).cuda(), draw((R, C), 6, xt, 0.1).cuda()
    gh = draw((R, C), 7, rt, 0.1).cuda() if with_gh else None
    rstd = torch.from_numpy(1 / np.sqrt((f64(h) ** 2).mean(1) + 1e-5)).float().cuda()
    seed, words = seed_words(-R, C)
    desc = gf.make_rms_desc(R, C, dtype=xt, residual_dtype=rt, p=p, param_dtype=torch.float32 if gamma is None else gamma.dtype)
    out = {"gres": Guarded((R, C), rt), "gx": Guarded((R, C), xt), "ggamma": Guarded((C,), torch.float32)}
    ws = Guarded((gf.gf_rms_norm_backward_workspace_bytes(desc),), torch.uint8)
    q_in, gh_in = gy, gh
    if alias == "gx":                                    # g_x over g_y, g_residual over g_h
        out["gx"].t.copy_(gy)
        q_in = out["gx"].t
        out["gres"].t.copy_(gh)
        gh_in = out["gres"].t
    gf.gf_rms_norm_backward(desc, q_in, gh_in, h, rstd, gamma, seed if p > 0 else None, *(out[k].t if k in want else None for k in out), ws.t)
    torch.cuda.synchronize()
    for g in (*out.values(), ws):
        g.check()
    g64 = 1.0 if gamma is None else f64(gamma)
    xh = f64(h) * f64(rstd)[:, None]
    q = f64(gy) * g64
    add = f64(gh) if with_gh else 0.0
    r = f64(rstd)[:, None]
    dot = (q * xh).mean(1, keepdims=True)
    ref = r * (q - xh * dot) + add
    terms = r * (np.abs(q) + np.abs(xh) * np.abs(q * xh).mean(1, keepdims=True)) + np.abs(add)
    if "gres" in want:
        assert (np.abs(f64(out["gres"].t) - ref) <= 128 * U * terms + STEP[rt] * np.abs(ref)).all()
    if "gx" in want:
        d, dt = dropped(ref, p, words), dropped(terms, p, words)
        assert (np.abs(f64(out["gx"].t) - d) <= 130 * U * dt + STEP[xt] * np.abs(d)).all()
    if "ggamma" in want:
        t = f64(gy) * xh
        assert (np.abs(f64(out["ggamma"].t) - t.sum(0)) <= 256 * U * np.abs(t).sum(0) + 1e-30).all()
    for k in out:
        if k not in want:
            assert bool((out[k].t == out[k].sentinel).all())
    return {k: v.t for k, v in out.items()}


@pytest.mark.parametrize("xt,rt", PAIRS, ids=IDS)
@pytest.mark.parametrize("R,C", ROWS, ids=lambda v: str(v))
def test_backward(gf, R, C, xt, rt):
    _check_backward(gf, R, C, xt, rt, 0.15 * (C % 3), with_gh=C % 5 != 0, gamma=_gamma(C))


@pytest.mark.parametrize("R,C", [(40, 96), (33, 1001), (9, 4096), (5, 9001)])
def test_outputs_may_be_left_out_and_lie_over_inputs(gf, R, C):
    full = _check_backward(gf, R, C, torch.float32, torch.float32, 0.0)
    assert torch.equal(full["gx"], full["gres"])                   # nothing dropped, one type
    again = _check_backward(gf, R, C, torch.float32, torch.float32, 0.0, alias="gx")
    for k in full:
        assert torch.equal(full[k], again[k])                      # bit for bit, in place or not
    for want in (("gres",), ("gx",), ("ggamma",), ("gx", "ggamma")):
        some = _check_backward(gf, R, C, torch.float32, torch.float32, 0.0, want=want)
        for k in want:
            assert torch.equal(some[k], full[k]), (want, k)


@pytest.mark.parametrize("C", [96, 1001, 9001])
def test_in_place_forward(gf, C):
    R, p = 37, 0.2
    x, res = draw((R, C), 1).cuda(), draw((R, C), 2, torch.float32, 1.5, 0.3).cuda()
    _, h, rstd, y, desc, seed, _ = _forward(gf, R, C, torch.float32, torch.float32, p, x=x.clone(), res=res.clone())
    gf.gf_rms_norm_forward(desc, x, res, seed, None, res, x, None)            # h over residual, y over x
    assert torch.equal(res, h) and torch.equal(x, y)


@pytest.mark.parametrize("out8", [False, True])
@pytest.mark.parametrize("C", [40, 1001, 4096, 9001])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_non_finite_value_stays_in_its_row(gf, C, bad, out8):
    R = 20
    x, res = draw((R, C), 8).cuda(), draw((R, C), 9).cuda()
    desc = gf.make_rms_desc(R, C)

    def run():
        h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(R, device="cuda")
        if not out8:
            gf.gf_rms_norm_forward(desc, x, res, None, None, h, y, rstd)
            return y
        codes = torch.empty((R, gf.fp8_pitch(C)), dtype=torch.uint8, device="cuda")
        scales = torch.zeros((-(-C // 128), gf.fp8_scale_pitch(R)), device="cuda")
        gf.gf_rms_norm_forward_fp8(desc, x, res, None, None, h, codes, scales, rstd)
        return gf.Fp8Matrix(codes, scales, R, C, False).dequantize()

    good = run()
    x[3, C // 2] = bad
    got = run()
    assert torch.equal(got[:3], good[:3]) and torch.equal(got[4:], good[4:])
    # an infinite sum of squares: rstd 0, and 0 times infinity where the value was
    assert not bool(torch.isfinite(got[3, C // 2])) and (bad == float("inf") or not bool(torch.isfinite(got[3]).any()))


def test_zero_rows_and_rows_of_zeros(gf):
    d = gf.make_rms_desc(0, 24)
    gw = torch.full((24,), 7.0, device="cuda")
    gf.gf_rms_norm_forward(d, None, None, None, None, None, None, None)
    gf.gf_rms_norm_backward(d, None, None, None, None, None, None, None, None, gw, None)
    torch.cuda.synchronize()
    assert bool((gw == 0).all())
    x, y = torch.zeros((5, 300), device="cuda"), torch.full((5, 300), 3.0, device="cuda")
    gf.gf_rms_norm_forward(gf.make_rms_desc(5, 300), x, None, None, None, None, y, None)
    assert bool((y == 0).all())
    codes, scales = torch.full((5, 304), 9, dtype=torch.uint8, device="cuda"), torch.zeros((3, 8), device="cuda")
    gf.gf_rms_norm_forward_fp8(gf.make_rms_desc(5, 300, eps=0.0), x + 1e-30, None, None, None, None, codes, scales, None)
    assert bool((codes[:, 300:] == 0).all())


def test_more_elements_than_32_bits_count(gf):
    """270001 rows of 8192 and as many of 8191 (2.2e9 elements): the last rows against the formula, with their own mask."""
    for C in (8192, 8191):
        R, p = 270001, 0.25
        x = torch.ones((R, C), dtype=torch.bfloat16, device="cuda")
        x[-3:] = draw((3, C), 1, torch.bfloat16).cuda()
        seed, words = seed_words(77, 3)
        desc = gf.make_rms_desc(R, C, dtype=torch.bfloat16, p=p)
        h, rstd = torch.empty_like(x), torch.empty(R, device="cuda")
        gf.gf_rms_norm_forward(desc, x, None, seed, None, h, x, rstd)                 # y over x
        first = (R - 3) * C // 8 * 8
        want = dropped(np.concatenate([np.ones((R - 3) * C - first), f64(draw((3, C), 1, torch.bfloat16)).reshape(-1)]), p, words, first)
        want = want[(R - 3) * C - first:].reshape(3, C)
        assert (np.abs(f64(h[-3:]) - want) <= 1.01 * 2.0 ** -8 * np.abs(want)).all()
        hk = f64(h[-3:])
        ref = hk / np.sqrt((hk ** 2).mean(1, keepdims=True) + 1e-5)
        assert (np.abs(f64(x[-3:]) - ref) <= 1.01 * 2.0 ** -8 * np.abs(ref)).all()
        gw = torch.empty(C, device="cuda")
        ws = torch.empty(gf.gf_rms_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        gf.gf_rms_norm_backward(desc, x, None, h, rstd, None, seed, None, x, gw, ws)      # g_y = y, g_x over it
        q = f64(torch.from_numpy(ref).to(torch.bfloat16))
        xh = hk * f64(rstd[-3:])[:, None]
        g = f64(rstd[-3:])[:, None] * (q - xh * (q * xh).mean(1, keepdims=True))
        mask = want != 0
        # (y's rounding in the kernel and here may differ by a step: 2^-7 of q)
        assert (np.abs(f64(x[-3:]) - np.where(mask, g / 0.75, 0)) <= 2.0 ** -6 * np.abs(q) * f64(rstd[-3:])[:, None] + 1e-6).all()
        del x, h
        torch.cuda.empty_cache()


@pytest.mark.parametrize("out8", [False, True])
def test_results_repeat_bit_for_bit_and_in_a_graph(gf, out8):
    R, C, p = 1200, 520, 0.1
    x, res, gamma = draw((R, C), 1, torch.bfloat16).cuda(), draw((R, C), 2).cuda(), draw((C,), 3, shift=1.0).cuda()
    gy = draw((R, C), 4, torch.bfloat16).cuda()
    desc = gf.make_rms_desc(R, C, dtype=torch.bfloat16, residual_dtype=torch.float32, p=p)
    seed, _ = seed_words(1, 2)

    def outputs():
        o = {"h": torch.empty_like(res), "rstd": torch.empty(R, device="cuda"), "gx": torch.empty_like(x), "gres": torch.empty_like(res),
             "gw": torch.empty(C, device="cuda"), "ws": torch.empty(gf.gf_rms_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")}
        return o | ({"codes": torch.zeros((R, 528), dtype=torch.uint8, device="cuda"), "scales": torch.zeros((5, R), device="cuda")} if out8
                    else {"y": torch.empty_like(x)})

    def run(o):
        if out8:
            gf.gf_rms_norm_forward_fp8(desc, x, res, seed, gamma, o["h"], o["codes"], o["scales"], o["rstd"])
        else:
            gf.gf_rms_norm_forward(desc, x, res, seed, gamma, o["h"], o["y"], o["rstd"])
        gf.gf_rms_norm_backward(desc, gy, res, o["h"], o["rstd"], gamma, seed, o["gres"], o["gx"], o["gw"], o["ws"])

    a, b = outputs(), outputs()
    run(a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(b)
    graph.replay()
    torch.cuda.synchronize()
    for k in a:
        if k != "ws":
            assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_gradients_against_differences(gf, p):
    """Central differences of L = sum(y v) + sum(h w) along a random direction, steps of 1e-2: truncation h^2 / 6 times a
    third derivative of order 10 and rounding u sqrt(n) / h, below 2e-3 of the slope's scale."""
    shape, C = (6, 10, 47), 47
    seed = seed_words(17)[0]
    x, res, w = draw(shape, 1).cuda(), draw(shape, 2).cuda(), draw((C,), 3, scale=0.3, shift=1.0).cuda()
    v, u = draw(shape, 4).cuda(), draw(shape, 5).cuda()
    leaves = [t.clone().requires_grad_(True) for t in (x, w, res)]

    def loss(a, b, c):
        y, h = gf.rms_norm(a, b, residual=c, p=p, seed=seed)
        return (y.double() * v.double()).sum() + (h.double() * u.double()).sum()

    loss(*leaves).backward()
    for k in range(3):
        d = draw(leaves[k].shape, 6 + k).cuda()
        ends = []
        for sign in (1, -1):
            moved = [t.detach() for t in leaves]
            moved[k] = moved[k] + sign * 1e-2 * d
            ends.append(float(loss(*moved)))
        slope = (ends[0] - ends[1]) / 2e-2
        want = float((leaves[k].grad.double() * d.double()).sum())
        assert abs(slope - want) <= 2e-3 * float(leaves[k].grad.double().norm() * d.double().norm()), (k, slope, want)


@pytest.mark.parametrize("form", ["rows", "strided", "unaligned", "empty", "other_stream", "mixed", "only_h", "only_y", "frozen", "no_residual"])
def test_module_through_autograd(gf, form):
    C = 24
    shape = (0, C) if form == "empty" else (35, C)
    x, res = draw(shape, 30).cuda(), draw(shape, 31).cuda()
    if form == "strided":
        x = draw((C, 35), 30).cuda().t()
    elif form == "unaligned":
        x = draw((35 * C + 1,), 30).cuda()[1:].view(35, C)
    elif form == "mixed":
        x = x.bfloat16()
    m = gf.RMSNorm(C, device="cuda")
    with torch.no_grad():
        m.weight.copy_(draw((C,), 34, shift=1.0))
    a, r = x.detach().requires_grad_(True), res.clone().requires_grad_(form != "frozen")
    gy, gh = torch.randn(shape, device="cuda", dtype=x.dtype), torch.randn(shape, device="cuda")
    side = torch.cuda.Stream() if form == "other_stream" else torch.cuda.current_stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        if form == "no_residual":
            y, h = m(a), None
            y.backward(gy)
        else:
            y, h = m(a, r)
            if form == "only_h":
                h.backward(gh)
            elif form == "only_y":
                y.backward(gy)
            else:
                torch.autograd.backward([y, h], [gy, gh])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    b, s, w = x.double().requires_grad_(True), res.double().requires_grad_(True), m.weight.detach().double().requires_grad_(True)
    hr = b if form == "no_residual" else b + s
    yr = hr * (hr.square().mean(-1, keepdim=True) + m.eps).rsqrt() * w
    total = (0 if form == "only_h" else (yr * gy.double()).sum()) + (0 if form in ("only_y", "no_residual") else (hr * gh.double()).sum())
    total.backward()
    tol = dict(rtol=0, atol=2.0 ** -7 * 8 if form == "mixed" else 2e-5)          # 16 bits: half a step of values up to 8
    assert y.dtype == x.dtype and torch.allclose(y.detach().double(), yr.detach(), **tol)
    assert torch.allclose(a.grad.double(), b.grad, **tol)
    if form not in ("frozen", "no_residual"):
        assert torch.allclose(r.grad.double(), s.grad, **tol)
    if form != "only_h":
        assert torch.allclose(m.weight.grad.double(), w.grad, rtol=0, atol=0.1 if form == "mixed" else 1e-4)


def test_rms_norm_adds_what_dropout_adds(gf):
    """The same seed: the sum that the norm forms is gf.dropout's, bit for bit."""
    for C in (64, 77):
        x, res, seed = draw((50, C), 1).cuda(), draw((50, C), 2).cuda(), seed_words(3, 4)[0]
        y, h = gf.rms_norm(x, None, residual=res, p=0.3, seed=seed)
        assert torch.equal(h, gf.dropout(x, 0.3, residual=res, seed=seed))
        assert torch.equal(y, gf.rms_norm(h, None))
