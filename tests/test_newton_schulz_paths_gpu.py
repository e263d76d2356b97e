"""Newton-Schulz and Muon on every way through the library, with bounds that bind for matrices of any shape.

The matrices here have singular values within a factor kappa = 4 of one another, about random singular vectors.  Rounding
errors and signal then grow alike through the steps: with c = 8 roundings of relative size u per step (X, A, b A + c A A, the
sums), K = 5 steps and independent roundings the result is off by at most kappa sqrt(K c) u / sqrt(3) of its norm,
    GF_NS_F16  (u = 2^-11, fp16 operands)                7.2e-3
    GF_NS_F32  (u = 2^-21, pairs of fp16, fp32 sums)      7.0e-6
whatever the shape.  (Without the low parts of the pairs the second would be at the first's size; zeros are off by 1.)  A bf16
result adds its own rounding: at most 2^-8 of an element, 1.7e-3 root mean square, so below 2^-9 of the norm of the hundreds of
elements and more that bf16 results have here; an fp32 one 2^-24 per operation.
"""
import math

import pytest
import torch

from parity_util import Guarded

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
BOUND = {"f16": 4 * math.sqrt(40 / 3) * 2.0 ** -11, "f32": 4 * math.sqrt(40 / 3) * 2.0 ** -21}


def _vectors(batch, rows, cols, seed):
    """Orthonormal U [batch, rows, k] and V [batch, cols, k], fp64 on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k = min(rows, cols)
    return tuple(torch.linalg.qr(torch.randn((batch, n, k), generator=g, device="cuda", dtype=torch.float64))[0] for n in (rows, cols))


def _with_values(U, V, seed, lo=1.0, hi=4.0, scale=1e-3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = lo + (hi - lo) * torch.rand((U.shape[0], 1, U.shape[2]), generator=g, device="cuda", dtype=torch.float64)
    s[..., 0], s[..., -1] = lo, hi
    return scale * (U * s) @ V.mT


def _plain(G, eps=1e-7):
    """Iterates of a batch of matrices in 64 bits, elementary operations only."""
    X = G if G.shape[-2] <= G.shape[-1] else G.mT
    X = X / ((X * X).sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(5):
        S = X @ X.mT
        X = A * X + (B * S + C * (S @ S)) @ X
    return X if G.shape[-2] <= G.shape[-1] else X.mT


def _check_newton_schulz(gf, shape, precision, out=torch.float32, seed=0):
    U, V = _vectors(*shape, seed)
    G = _with_values(U, V, seed + 1).to(torch.float32)
    desc = gf.make_ns_desc(*shape, out_dtype=out, precision=gf.GF_NS_F16 if precision == "f16" else gf.GF_NS_F32)
    O, ws = Guarded(shape, out), Guarded((gf.gf_newton_schulz_workspace_bytes(desc),), torch.uint8)
    gf.gf_newton_schulz(desc, G, O.t, ws.t)
    assert gf.gf_last_async_status(ws.t) == gf.GF_OK
    O.check()
    ws.check()
    ref = _plain(G.double())
    rounding = 2.0 ** -9 if out == torch.bfloat16 else 2.0 ** -24
    for b in range(shape[0]):
        err = float((O.t[b].double() - ref[b]).norm() / ref[b].norm())
        assert err <= BOUND[precision] + rounding, (b, err)


# on one CTA and on clusters; just past what these hold; general, with tall, square and odd shapes, and split tiles
SHAPES = [(1, 16, 16), (3, 17, 13), (1, 64, 64), (2, 127, 128), (1, 128, 2048), (1, 600, 128), (1, 129, 129), (2, 130, 2049), (1, 200, 136),
          (1, 256, 256), (1, 301, 131), (1, 385, 640), (1, 500, 500), (1, 700, 513), (3, 257, 400), (1, 1001, 1030)]


@pytest.mark.parametrize("precision", ["f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_shapes_of_any_proportion(gf, shape, precision):
    _check_newton_schulz(gf, shape, precision, seed=shape[1])


# sizes at which fp16 operands run on pairs of CTAs (tiles of 256 x 128 and 256 x 256, ragged in both directions), and pairs of
# fp16 with many tiles per multiprocessor
@pytest.mark.parametrize("shape", [(1, 1792, 1792), (1, 1500, 2100), (1, 2049, 1793), (2, 1537, 1800), (1, 2300, 2563), (1, 2049, 4100)],
                         ids=lambda s: "x".join(map(str, s)))
def test_large_matrices(gf, shape):
    _check_newton_schulz(gf, shape, "f16", seed=shape[2])
    _check_newton_schulz(gf, shape, "f16", torch.bfloat16, seed=shape[2] + 7)


@pytest.mark.parametrize("shape", [(1, 1793, 2049), (2, 1300, 1300)], ids=lambda s: "x".join(map(str, s)))
def test_large_matrices_in_pairs_of_fp16(gf, shape):
    _check_newton_schulz(gf, shape, "f32", seed=shape[2])


def _muon_inputs(count, rows, cols, taps, gdt, wdt, seed):
    """Gradient and momentum about the same singular vectors, values of both within [1, 3], so that those of their combination
    stay within a factor of 4 (also where the gradient is rounded to bf16: 2^-9 of its norm, spread over all directions)."""
    U, V = _vectors(count, rows, cols, seed)
    grad = _with_values(U, V, seed + 1, 1.0, 3.0)[..., None].expand(count, rows, cols, taps).contiguous().to(gdt)
    mom = _with_values(U, V, seed + 2, 1.0, 3.0).to(torch.float32)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 3)
    weight = (torch.randn((count, rows, cols, taps), generator=g, device="cuda") * 2e-3).to(wdt)      # about the size of the step
    return grad, mom, weight


def _check_muon(gf, desc, grad, mom, weight, mom_out, weight_out, precision):
    """mom_out and weight_out against the step on the whole flattened gradient, in 64 bits."""
    taps, mu = grad.shape[-1], desc.momentum
    g = grad.double()
    M = mu * mom.double() + (1 - mu) * g[..., 0]
    full = M[..., None].expand(g.shape)
    u = (1 - mu) * g + mu * full if desc.nesterov else full
    for b in range(g.shape[0]):
        O = _plain(u[b].reshape(1, desc.rows, desc.cols * taps), desc.eps)[0].reshape(g.shape[1:])
        W = (1 - desc.lr * desc.weight_decay) * weight[b].double() - desc.lr * desc.scale * O
        step = desc.lr * desc.scale * float(O.norm())
        rounding = 2.0 ** -9 * float(W.norm()) if weight.dtype == torch.bfloat16 else 4 * 2.0 ** -24 * float(weight[b].double().norm() + step)
        assert float((mom_out[b].double() - M[b]).abs().max()) <= 4 * 2.0 ** -24 * max(float(M[b].abs().max()), float(mom[b].abs().max())), b
        off = float((weight_out[b].double() - W).norm())
        assert off <= BOUND[precision] * step + rounding, (b, off, step)


MUON = [
    # count, rows, cols, taps, weights, gradients, precision, nesterov, in place
    (2, 200, 136, 9, torch.float32, torch.float32, "f32", True, True),
    (2, 200, 136, 9, torch.bfloat16, torch.float32, "f16", True, True),
    (1, 301, 131, 1, torch.float32, torch.float32, "f32", False, False),
    (1, 131, 301, 25, torch.bfloat16, torch.bfloat16, "f16", False, False),
    (3, 160, 256, 1, torch.float32, torch.bfloat16, "f32", True, False),
    (3, 160, 256, 1, torch.bfloat16, torch.bfloat16, "f16", True, True),
    (50, 130, 140, 1, torch.float32, torch.float32, "f32", True, True),      # more layers than one launch's arguments hold
    (49, 140, 130, 4, torch.bfloat16, torch.float32, "f16", True, False),
    (6, 256, 256, 9, torch.float32, torch.float32, "f32", True, True),
    (1, 1800, 1900, 1, torch.bfloat16, torch.bfloat16, "f16", True, True),    # on pairs of CTAs
    # matrices that a cluster holds, in the precision of 16-bit weights
    (4, 96, 40, 1, torch.bfloat16, torch.bfloat16, "f16", True, True),
    (2, 64, 64, 9, torch.bfloat16, torch.float32, "f16", False, False),
    (12, 576, 96, 1, torch.bfloat16, torch.float32, "f16", True, True),
    (2, 100, 1500, 1, torch.float32, torch.float32, "f16", True, False),
]


@pytest.mark.parametrize("count,rows,cols,taps,wdt,gdt,precision,nesterov,inplace", MUON,
                         ids=lambda v: {torch.float32: "f32", torch.bfloat16: "bf16"}.get(v, str(v)))
def test_muon_step(gf, count, rows, cols, taps, wdt, gdt, precision, nesterov, inplace):
    grad, mom, weight = _muon_inputs(count, rows, cols, taps, gdt, wdt, rows + taps)
    desc = gf.make_muon_desc(count, rows, cols, taps, grad_dtype=gdt, weight_dtype=wdt, nesterov=nesterov, momentum=0.9, lr=0.02,
                             precision=gf.GF_NS_F16 if precision == "f16" else gf.GF_NS_F32, weight_decay=0.1,
                             scale=0.2 * math.sqrt(max(rows, cols * taps)))
    ws = Guarded((gf.gf_muon_workspace_bytes(desc),), torch.uint8)
    m_out, w_out = [Guarded(t.shape, t.dtype) for t in mom], [Guarded(t.shape, t.dtype) for t in weight]
    if inplace:
        for o, t in zip(m_out + w_out, list(mom) + list(weight)):
            o.t.copy_(t)
    m_in, w_in = ([o.t for o in m_out], [o.t for o in w_out]) if inplace else ([t.clone() for t in mom], [t.clone() for t in weight])
    gf.gf_muon_step(desc, [t.clone() for t in grad], m_in, w_in, [o.t for o in m_out], [o.t for o in w_out], ws.t)
    assert gf.gf_last_async_status(ws.t) == gf.GF_OK
    for o in m_out + w_out + [ws]:
        o.check()
    _check_muon(gf, desc, grad, mom, weight, torch.stack([o.t for o in m_out]), torch.stack([o.t for o in w_out]), precision)


@pytest.mark.parametrize("taps", [1, 3])
def test_general_muon_takes_slices_of_a_flat_buffer(gf, taps):
    """Matrices that a cluster does not hold, in buffers off 16-byte boundaries: as from aligned ones, bit for bit."""
    rows, cols, count = 161, 136, 3
    grad, mom, weight = _muon_inputs(count, rows, cols, taps, torch.float32, torch.float32, 5)
    desc = gf.make_muon_desc(count, rows, cols, taps, lr=0.02, weight_decay=0.1, momentum=0.9, scale=0.2 * math.sqrt(rows))
    ws = torch.empty(gf.gf_muon_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    results = []
    for shift in (0, 1):
        def cut(t):
            flat = torch.cat([torch.zeros(shift, device="cuda"), t.reshape(-1)])
            return list(flat[shift:].view(t.shape))
        g, m, w = cut(grad), cut(mom), cut(weight)
        assert (g[0].data_ptr() % 16 == 0) == (shift == 0)
        gf.gf_muon_step(desc, g, m, w, m, w, ws)
        results.append((torch.stack(m), torch.stack(w)))
    assert torch.equal(results[0][0], results[1][0])
    _check_muon(gf, desc, grad, mom, weight, *results[0], "f32")
    _check_muon(gf, desc, grad, mom, weight, *results[1], "f32")
