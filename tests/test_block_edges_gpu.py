"""In-place forms of the residual-block operators (gf_block.h) that lie over another input than those of the operators' own tests: the same
bits as side by side."""
import pytest
import torch

from block_util import DTYPES, draw, seed_words

pytestmark = pytest.mark.gpu

F32, BF16 = DTYPES
SIZES = [(40, 64), (37, 97), (33, 768), (21, 1001), (9, 4096), (5, 9001)]      # each way a row is dealt out


@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("t", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("R,C", SIZES, ids=lambda v: str(v))
def test_norm_forward_with_the_sum_over_its_branch(gf, R, C, t, p):
    x, res, gamma = draw((R, C), 1, t).cuda(), draw((R, C), 2, t).cuda(), draw((C,), 3, shift=1.0).cuda()
    seed = seed_words(7)[0] if p else None
    desc = gf.make_rms_desc(R, C, dtype=t, p=p)

    def run(over, out8):
        a = x.clone()
        h, y, rstd = a if over else torch.empty_like(a), torch.empty_like(a), torch.empty(R, device="cuda")
        if not out8:
            gf.gf_rms_norm_forward(desc, a, res, seed, gamma, h, y, rstd)
            return h, y, rstd
        codes = torch.empty((R, gf.fp8_pitch(C)), dtype=torch.uint8, device="cuda")
        scales = torch.zeros((-(-C // 128), gf.fp8_scale_pitch(R)), device="cuda")
        gf.gf_rms_norm_forward_fp8(desc, a, res, seed, gamma, h, codes, scales, rstd)
        return h, codes, scales, rstd

    for out8 in (False, True):
        for got, want in zip(run(True, out8), run(False, out8)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("t", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("R,C", SIZES, ids=lambda v: str(v))
def test_norm_backward_with_the_residuals_gradient_over_that_of_y(gf, R, C, t, p):
    h, gy, gh, gamma = draw((R, C), 1, t).cuda(), draw((R, C), 2, t).cuda(), draw((R, C), 3, t).cuda(), draw((C,), 4, shift=1.0).cuda()
    rstd = (h.double().square().mean(1) + 1e-5).rsqrt().float()
    seed = seed_words(7)[0] if p else None
    desc = gf.make_rms_desc(R, C, dtype=t, p=p)
    ws = torch.empty(gf.gf_rms_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def run(over):
        a = gy.clone()
        gres, gx, gw = a if over else torch.empty_like(a), torch.empty_like(a), torch.empty(C, device="cuda")
        gf.gf_rms_norm_backward(desc, a, gh, h, rstd, gamma, seed, gres, gx, gw, ws)
        return gres, gx, gw

    for got, want in zip(run(True), run(False)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("xt,rt", [(F32, BF16), (BF16, F32), (BF16, BF16)], ids=["f32_bf16", "bf16_f32", "bf16"])
def test_dropout_over_a_residual_of_another_type(gf, xt, rt):
    n = 100003
    x, res, seed = draw((n,), 1, xt).cuda(), draw((n,), 2, rt).cuda(), seed_words(3)[0]
    desc = gf.make_dropout_desc(n, dtype=xt, out_dtype=rt, p=0.3)
    want, got = torch.empty_like(res), res.clone()
    gf.gf_dropout_forward(desc, x, res, seed, want)
    gf.gf_dropout_forward(desc, x, got, seed, got)
    assert torch.equal(got, want)
