"""Tensors of more elements than 32 bits count, on the ways that index them differently: the first and the last of them against
a plain form in 64 bits on the GPU.  Bounds as in the tests of the small sizes: a bf16 result is off by its rounding, 2^-8 of the
largest magnitude covers it; Newton-Schulz with fp16 operands and values within a factor of 4 by 7.2e-3 and that rounding."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("side", [56, 55], ids=["whole_pieces", "odd_planes"])
def test_layer_norm_of_maps(gf, side):
    C = 256
    N = 2 ** 31 // (C * side * side) + 3
    g = torch.Generator(device="cuda")
    g.manual_seed(side)
    x = torch.empty((N, C, side, side), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    assert x.numel() > 2 ** 31
    desc = gf.make_norm_desc(N, C, side, side, dtype=torch.bfloat16, layout=gf.GF_NCHW)
    R = N * side * side
    y, mean, rstd = torch.empty_like(x), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    gf.gf_layer_norm_forward(desc, x, None, None, y, mean, rstd)
    ws = torch.empty(gf.gf_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    gw, gb, gx = torch.empty(C, device="cuda"), torch.empty(C, device="cuda"), torch.empty_like(x)
    gf.gf_layer_norm_backward(desc, x, x, None, mean, rstd, gx, gw, gb, ws)          # g_y = x
    assert gf.gf_last_async_status(ws) == gf.GF_OK
    for part in (slice(0, 2), slice(N - 2, N)):
        t = x[part].double()
        m = t.mean(1, keepdim=True)
        r = ((t - m).square().mean(1, keepdim=True) + 1e-5).rsqrt()
        xh = (t - m) * r
        want = r * (t - m - xh * (t * xh).mean(1, keepdim=True))      # all but cancels: bound by its terms
        assert float((y[part].double() - xh).abs().max()) <= 2.0 ** -8 * float(xh.abs().max())
        assert float((gx[part].double() - want).abs().max()) <= 2e-5 * float((r * t).abs().max()) * 3 + 2.0 ** -8 * float(want.abs().max())
    # sums over the pixels: of xh x = xh^2 / r, with mean 1 to a few parts in sqrt(R); and of x
    assert float((gw.double() / R - 1).abs().max()) <= 0.01 and float((gb.double() / R).abs().max()) <= 0.01


def test_newton_schulz_of_a_batch(gf):
    batch, m, n = 2 ** 31 // (16 * 16384) + 9, 16, 16384
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    G = torch.empty((batch, m, n), dtype=torch.bfloat16, device="cuda").normal_(generator=g)      # wide and Gaussian: values alike
    assert G.numel() > 2 ** 31
    desc = gf.make_ns_desc(batch, m, n, in_dtype=torch.bfloat16, out_dtype=torch.bfloat16, precision=gf.GF_NS_F16)
    O, ws = torch.empty_like(G), torch.empty(gf.gf_newton_schulz_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    gf.gf_newton_schulz(desc, G, O, ws)
    assert gf.gf_last_async_status(ws) == gf.GF_OK
    for b in (0, 1, batch // 2, batch - 2, batch - 1):
        X = G[b].double()
        X = X / (X.norm() + 1e-7)
        for _ in range(5):
            S = X @ X.mT
            X = 3.4445 * X + (-4.7750 * S + 2.0315 * S @ S) @ X
        assert float((O[b].double() - X).norm() / X.norm()) <= 7.2e-3 + 2.0 ** -9, b
