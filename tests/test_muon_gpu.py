"""GPU parity of the Newton-Schulz iterates and the Muon step (gf_train.h) with plain 64-bit numpy.

Bounds.  A step rounds its operands a handful of times (X, A, b A + c A A, the sums): c = 8
roundings of relative size u, u = 2^-11 for fp16 operands (GF_NS_F16) and 2^-21 for pairs with fp32
sums (GF_NS_F32).  A perturbation E of X_k changes the later iterates by at most a factor a (3.4445, the
slope at 0) per step, so
    ||error||_F <= c u sum_k a^(K - k) ||X_k||_F                        (any input: `worst`)
Where all singular values are within a factor kappa of one another, perturbations and signal grow
alike: relative error <= kappa sqrt(K c) u / sqrt(3) for independent roundings, with kappa <= 4 for
the wide Gaussian matrices here: 4 sqrt(40) u / sqrt(3) = 7e-3 (F16) and 7e-6 (F32)  (`even`).
A bf16 result adds 2^-9 relative per element.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from parity_util import Guarded, f64

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
UNIT = {"f16": 2.0 ** -11, "f32": 2.0 ** -21}


def _plain(G, steps=5, eps=1e-7, coeffs=None):
    """Iterates of one matrix in fp64, and the bound on the error of unit roundings, relative to the result."""
    X = G if G.shape[0] <= G.shape[1] else G.T
    X = X / (np.linalg.norm(X) + eps)
    worst = 0.0
    for k in range(steps):
        a, b, c = coeffs[k] if coeffs else (A, B, C)
        slope = abs(a)
        worst = slope * (worst + np.linalg.norm(X))
        S = X @ X.T
        X = a * X + (b * S + c * (S @ S)) @ X
    worst = 8 * (worst + np.linalg.norm(X)) / max(np.linalg.norm(X), 1e-300)
    return (X if G.shape[0] <= G.shape[1] else X.T), worst


def _err(got, ref):
    return float(np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300))


def _draw(shape, seed, scale=1.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g) * scale


def _run(gf, G, precision="f32", out=torch.float32, steps=5, eps=1e-7, coeffs=None):
    b, m, n = G.shape
    desc = gf.make_ns_desc(b, m, n, in_dtype=G.dtype, out_dtype=out, precision=gf.GF_NS_F16 if precision == "f16" else gf.GF_NS_F32,
                           steps=steps, eps=eps)
    O, ws = Guarded(G.shape, out), Guarded((gf.gf_newton_schulz_workspace_bytes(desc),), torch.uint8)
    before = gf.gf_kernel_launch_count()
    gf.gf_newton_schulz(desc, G, O.t, ws.t, None, coeffs)
    assert gf.gf_last_async_status(ws.t) == gf.GF_OK
    torch.cuda.synchronize()
    assert gf.gf_kernel_launch_count() > before
    O.check()
    ws.check()
    return O.t


SHAPES = [(1, 1, 1), (2, 1, 7), (1, 9, 1), (3, 5, 3), (1, 16, 16), (2, 31, 33), (5, 64, 64), (1, 64, 200), (2, 127, 129), (1, 128, 128),
          (3, 129, 100), (1, 96, 576), (2, 576, 96), (1, 200, 1000), (1, 255, 257), (1, 256, 256), (4, 257, 255), (1, 300, 301),
          (1, 385, 640), (2, 1001, 130), (1, 512, 2048), (1, 700, 513), (3, 100, 1025), (1, 2048, 128), (2, 17, 2047), (1, 128, 2049),
          (1, 3, 5000), (30, 33, 40), (1, 300, 3000), (2, 129, 2500), (1, 700, 1500)]


@pytest.mark.parametrize("precision", ["f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_newton_schulz(gf, shape, precision):
    G = _draw(shape, 100 + shape[1], 1e-3).cuda()
    got = f64(_run(gf, G, precision))
    for b in range(shape[0]):
        ref, worst = _plain(f64(G[b]))
        bound = worst * UNIT[precision]
        if max(shape[1:]) >= 4 * min(shape[1:]):
            bound = min(bound, 7e-3 if precision == "f16" else 7e-6)
        assert _err(got[b], ref) <= bound, (b, _err(got[b], ref), bound)


@pytest.mark.parametrize("shape", [(2, 96, 512), (1, 512, 100), (3, 33, 200)])
def test_sixteen_bit_input_and_output(gf, shape):
    G = _draw(shape, 7, 3.0).cuda().bfloat16()
    for precision in ("f16", "f32"):
        got = _run(gf, G, precision, torch.bfloat16)
        for b in range(shape[0]):
            ref, _ = _plain(f64(G[b]))
            assert _err(f64(got[b]), ref) <= 2.0 ** -9 + (7e-3 if precision == "f16" else 7e-6)


def test_large_matrix_against_torch(gf):
    """Many tiles per multiprocessor, all tile widths of the symmetric products, 64-bit torch on the GPU as reference."""
    for shape, precision in (((1, 1500, 2100), "f16"), ((1, 2100, 1500), "f32"), ((3, 800, 900), "f16")):
        G = _draw(shape, 8).cuda()
        got = _run(gf, G, precision).double()
        for b in range(shape[0]):
            X = G[b].double()
            tall = X.shape[0] > X.shape[1]
            X = X.T if tall else X
            X = X / X.norm()
            worst = 0.0
            for _ in range(5):
                worst = A * (worst + float(X.norm()))
                S = X @ X.T
                X = A * X + (B * S + C * S @ S) @ X
            bound = 8 * UNIT[precision] * (worst + float(X.norm())) / float(X.norm())
            X = X.T if tall else X
            assert float((got[b] - X).norm() / X.norm()) <= bound


def test_rank_one_and_zero_and_scale(gf):
    """A rank-one matrix has one singular value, 1: O = p(1) u v^T with p the five-fold quintic.  Zeros
    stay zeros, also with eps = 0.  The scale of G only enters through eps."""
    s = 1.0
    for _ in range(5):
        s = A * s + B * s ** 3 + C * s ** 5
    u, v = _draw((70, 1), 1), _draw((1, 90), 2)
    G = (u / u.norm()) @ (v / v.norm())
    got = f64(_run(gf, G[None].cuda(), eps=0.0))[0]
    assert _err(got, s * f64(G)) <= _plain(f64(G), eps=0.0)[1] * UNIT["f32"]
    for eps in (0.0, 1e-7):
        assert bool((_run(gf, torch.zeros((2, 40, 50), device="cuda"), eps=eps) == 0).all())
    H = _draw((1, 60, 80), 3).cuda()
    a = _run(gf, H, eps=0.0)
    for scale in (2.0 ** -40, 2.0 ** 40):
        assert torch.equal(a, _run(gf, H * scale, eps=0.0))          # powers of two change no rounding


def test_one_bad_matrix_leaves_the_others_alone(gf):
    G = _draw((3, 50, 70), 4).cuda()
    good = _run(gf, G)
    for bad in (float("nan"), float("inf")):
        H = G.clone()
        H[1, 3, 5] = bad
        got = _run(gf, H)
        assert torch.equal(got[0], good[0]) and torch.equal(got[2], good[2])
        assert not bool(torch.isfinite(got[1]).all())


def test_coefficients_and_steps(gf):
    cubic = (1.5, -0.5, 0.0)
    for coeffs in ([cubic] * 8, [(A, B, C)], [(A, B, C)] * 3 + [cubic] * 3, [(8.0, -22.0, 16.0), (3.9, -2.8, 0.5)]):
        G = _draw((1, 40, 160), 5).cuda()
        got = f64(_run(gf, G, steps=len(coeffs), coeffs=coeffs))[0]
        ref, worst = _plain(f64(G[0]), len(coeffs), coeffs=coeffs)
        assert _err(got, ref) <= worst * UNIT["f32"]


def test_wrapper(gf):
    G = _draw((2, 3, 40, 24), 6).cuda()
    O = gf.newton_schulz(G)
    assert O.shape == G.shape and O.dtype == torch.float32
    assert torch.equal(O.reshape(6, 40, 24), _run(gf, G.reshape(6, 40, 24)))
    assert gf.newton_schulz(G.bfloat16()).dtype == torch.bfloat16
    assert torch.equal(gf.newton_schulz(G.mT), gf.newton_schulz(G.mT.contiguous()))
    assert gf.newton_schulz(G[:0]).shape == (0, 3, 40, 24)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P = gf.newton_schulz(G)
    side.synchronize()
    assert torch.equal(P, O)


@pytest.mark.parametrize("shape", [(2, 96, 600), (1, 300, 3000), (2, 700, 500)])
def test_results_repeat_and_calls_can_be_captured(gf, shape):
    """Bit for bit the same from call to call (split tiles are added in a fixed order), and from a captured graph."""
    G = _draw(shape, 9).cuda()
    want = _run(gf, G).clone()
    for _ in range(5):
        assert torch.equal(_run(gf, G), want)
    desc = gf.make_ns_desc(*shape)
    O, ws = torch.zeros_like(G), torch.empty(gf.gf_newton_schulz_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gf.gf_newton_schulz(desc, G, O, ws)
    for _ in range(2):
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)


# ---- the Muon step ---------------------------------------------------------------------------------------

def _plain_muon(g, mom, w, taps, lr, wd, scale, mu, nesterov):
    """One layer from its whole flattened gradient, fp64: (W', M', worst-case factor)."""
    rows, cols = g.shape[:2]
    new = mu * mom + (1 - mu) * g[..., 0]
    full = np.repeat(new[..., None], taps, -1)
    u = (1 - mu) * g + mu * full if nesterov else full
    O, worst = _plain(u.reshape(rows, cols * taps))
    return (1 - lr * wd) * w - lr * scale * O.reshape(w.shape), new, worst, lr * scale * np.linalg.norm(O)


@pytest.mark.parametrize("count,rows,cols,taps,wdt,gdt,nesterov,inplace", [
    (1, 16, 24, 1, torch.float32, torch.float32, True, False),
    (6, 64, 48, 9, torch.float32, torch.float32, True, True),
    (2, 33, 35, 25, torch.bfloat16, torch.float32, False, False),
    (3, 100, 40, 1, torch.bfloat16, torch.bfloat16, True, True),
    (50, 9, 7, 9, torch.float32, torch.float32, True, False),      # more layers than one launch's arguments hold
    (1, 200, 1, 9, torch.float32, torch.float32, True, False),     # a depthwise kernel: one column
    (1, 1, 1, 1, torch.float32, torch.float32, True, False),
])
def test_muon_step(gf, count, rows, cols, taps, wdt, gdt, nesterov, inplace):
    lr, wd, scale, mu = 0.02, 0.1, 0.2 * math.sqrt(max(rows, cols * taps)), 0.9
    g = [_draw((rows, cols, 1), 10 + k, 1e-2).expand(rows, cols, taps).contiguous().to(gdt).cuda() for k in range(count)]
    mom = [_draw((rows, cols), 200 + k, 1e-2).cuda() for k in range(count)]
    w = [_draw((rows, cols, taps), 400 + k, 0.1).to(wdt).cuda() for k in range(count)]
    desc = gf.make_muon_desc(count, rows, cols, taps, grad_dtype=gdt, weight_dtype=wdt, precision=gf.GF_NS_F32, nesterov=nesterov,
                             momentum=mu, lr=lr, weight_decay=wd, scale=scale)
    ws = Guarded((gf.gf_muon_workspace_bytes(desc),), torch.uint8)
    m_out, w_out = [Guarded(t.shape, t.dtype) for t in mom], [Guarded(t.shape, t.dtype) for t in w]
    m_in, w_in = mom, w
    if inplace:
        for o, t in zip(m_out + w_out, mom + w):
            o.t.copy_(t)
        m_in, w_in = [o.t for o in m_out], [o.t for o in w_out]
    gf.gf_muon_step(desc, g, m_in, w_in, [o.t for o in m_out], [o.t for o in w_out], ws.t)
    assert gf.gf_last_async_status(ws.t) == gf.GF_OK
    torch.cuda.synchronize()
    for o in m_out + w_out + [ws]:
        o.check()
    for k in range(count):
        W, M, worst, step = _plain_muon(f64(g[k]), f64(mom[k]), f64(w[k]), taps, desc.lr, desc.weight_decay, desc.scale, desc.momentum,
                                        nesterov)
        assert np.abs(f64(m_out[k].t) - M).max() <= 4 * 2.0 ** -24 * max(np.abs(M).max(), np.abs(f64(mom[k])).max())
        off = np.linalg.norm(f64(w_out[k].t) - W)
        rounding = (2.0 ** -8 if wdt == torch.bfloat16 else 4 * 2.0 ** -24) * np.linalg.norm(W)
        assert off <= worst * UNIT["f32"] * step + rounding, (k, off)


def test_optimizer_trains_filtered_layers(gf):
    """Two steps of Muon on a block of filtered convolutions and a layer norm; equal taps give the update of
    the flattened kernel, and layers of one shape share a call."""
    torch.manual_seed(0)
    block = torch.nn.Sequential(gf.FilteredConv2d(16, 32, 3, r=2, device="cuda"), gf.LayerNorm(32, channel_dim=1, device="cuda"),
                                gf.FilteredConv2d(32, 32, 3, r=2, device="cuda"), gf.FilteredConv2d(32, 16, 1, r=2, device="cuda"))
    x = torch.randn(2, 16, 16, 16, device="cuda")
    kernels = [m.weight for m in block if isinstance(m, gf.FilteredConv2d)]
    assert all(k.filtered_taps for k in kernels)
    opt = gf.Muon(kernels, lr=1e-2, weight_decay=0.1)
    twins = [k.detach().clone().requires_grad_(True) for k in kernels]       # the same without the knowledge of equal taps
    other = gf.Muon(twins, lr=1e-2, weight_decay=0.1)
    losses = []
    for _ in range(2):
        loss = (block(x) - x).square().mean()
        loss.backward()
        losses.append(float(loss.detach()))
        for t, k in zip(twins, kernels):
            t.grad = k.grad.clone()
        opt.step()
        other.step()
        for p in block.parameters():
            p.grad = None
    assert losses[1] < losses[0]
    for t, k in zip(twins, kernels):
        assert _err(f64(t.detach()), f64(k.detach())) <= 1e-5
    assert opt.state[kernels[0]]["momentum"].shape == (32, 16) and other.state[twins[0]]["momentum"].shape == (32, 144)


def test_optimizer_state_survives_saving(gf):
    """A state that was saved and loaded (torch casts it to the parameters' dtype) goes on as fp32; one kept with taps is
    refused where taps are used, and the other way round."""
    conv = gf.FilteredConv2d(8, 16, 3, r=2, bias=False, device="cuda", dtype=torch.bfloat16)
    grad = _draw((16, 8, 1, 1), 70).expand(16, 8, 3, 3).contiguous().to("cuda", torch.bfloat16)
    opt = gf.Muon([conv.weight], lr=0.1)
    conv.weight.grad = grad
    opt.step()
    again = gf.Muon([conv.weight], lr=0.1)
    again.load_state_dict(opt.state_dict())
    again.step()
    m = again.state[conv.weight]["momentum"]
    assert m.dtype == torch.float32 and m.shape == (16, 8) and bool(torch.isfinite(conv.weight).all())
    flat = gf.Muon([conv.weight], lr=0.1, filtered_taps=False)
    flat.step()
    assert flat.state[conv.weight]["momentum"].shape == (16, 72)
    flat.load_state_dict(opt.state_dict())           # brings filtered_taps = True along with the state
    flat.param_groups[0]["filtered_taps"] = False
    with pytest.raises(ValueError, match="filtered_taps"):
        flat.step()


def test_muon_takes_slices_of_a_flat_buffer(gf):
    """Parameters, momenta and gradients that lie one behind the other, off 16-byte boundaries."""
    rows, cols = 13, 9
    flat = [_draw((3 * rows * cols + 1,), 60 + k, 1e-2).cuda() for k in range(3)]
    cut = [[f[1 + k * rows * cols:1 + (k + 1) * rows * cols].view(rows, cols) for k in range(3)] for f in flat]
    want = [[t.clone() for t in ts] for ts in cut]
    desc = gf.make_muon_desc(3, rows, cols, lr=0.1, scale=1.0)
    ws = torch.empty(gf.gf_muon_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    for g, m, w in (want, cut):
        gf.gf_muon_step(desc, g, m, w, m, w, ws)
    torch.cuda.synchronize()
    for a, b in zip(want, cut):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_step_refusals_reach_the_caller(gf):
    t = torch.zeros(4, 4, device="cuda")
    d = gf.make_muon_desc(2, 4, 4)
    with pytest.raises(ValueError):
        gf.gf_muon_step(d, [t], [t, t], [t, t], [t, t], [t, t], None)
    with pytest.raises(gf.GfError) as e:
        gf.gf_muon_step(d, [t, t], [t, t], [t, t], [t, t], [t, t], torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == gf.GF_ERR_WORKSPACE
    p = torch.nn.Parameter(torch.zeros(6, 4, device="cuda").t())
    opt = gf.Muon([p])
    p.grad = torch.zeros_like(p)
    with pytest.raises(ValueError, match="contiguous"):
        opt.step()
