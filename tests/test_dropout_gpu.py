"""Dropout from a counter (gf_block.h) against the definition on the host.

Bounds: a kept value is x times a scale that is rounded to fp32, and the sum is rounded: three half steps of fp32 on
|x scale| + |residual|, and half a step of the result's type.  A mask that differs anywhere is off by whole values."""
import numpy as np
import pytest
import torch

from block_util import DTYPES, STEP, U, draw, dropped, philox_bits, seed_words
from parity_util import Guarded, f64

pytestmark = pytest.mark.gpu


def test_the_generator_gives_the_published_vectors():
    """Known answers of Philox4x32 with ten rounds: zero counter and key; all ones; digits of pi."""
    ones = 0xFFFFFFFFFFFFFFFF
    for low, high, key, want in ((0, 0, 0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                                 (ones, ones, ones, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                                 (0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822,
                                  (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        got = philox_bits(8, key, high, low * 8).view("<u4")
        assert tuple(int(v) for v in got) == want


@pytest.mark.parametrize("xt", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rt", [None, *DTYPES], ids=["alone", "f32res", "bf16res"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1000, 4097, 6144, 1 << 20, 3000001])
def test_forward_and_backward(gf, xt, rt, n):
    p = 0.1 + 0.3 * (n % 3)
    x, res = draw(n, 1, xt).cuda(), None if rt is None else draw(n, 2, rt, 2.0).cuda()
    yt = xt if rt is None else rt
    seed, words = seed_words(-123456789 * n, n)
    desc = gf.make_dropout_desc(n, dtype=xt, out_dtype=yt, p=p)
    y, gx = Guarded((n,), yt), Guarded((n,), xt)
    gf.gf_dropout_forward(desc, x, res, seed, y.t)
    want = dropped(f64(x), p, words)
    r = 0.0 if res is None else f64(res)
    assert (np.abs(f64(y.t) - (want + r)) <= 3 * U * (np.abs(want) + np.abs(r)) + STEP[yt] * np.abs(want + r)).all()
    gy = draw(n, 3, yt, 1e-2).cuda()
    gf.gf_dropout_backward(desc, gy, seed, gx.t)
    want = dropped(f64(gy), p, words)
    assert (np.abs(f64(gx.t) - want) <= (3 * U + STEP[xt]) * np.abs(want)).all()
    y.check()
    gx.check()


@pytest.mark.parametrize("p,share", [(0.0, 0.0), (1e-6, 0.0), (2.0 ** -16, 2.0 ** -16), (0.25, 0.25), (1.0 - 2.0 ** -16, 1 - 2.0 ** -16), (1.0, 1.0)])
def test_share_and_scale_at_the_ends(gf, p, share):
    """The share that is dropped is p, rounded to a multiple of 2^-16 (five deviations of 4e6 draws), and what is kept is
    scaled by the rounded p's 1 / (1 - p); none at all and all are exact."""
    n = 4_000_000
    x = torch.ones(n, device="cuda")
    seed, _ = seed_words(99)
    y = torch.empty_like(x)
    gf.gf_dropout_forward(gf.make_dropout_desc(n, p=p), x, None, seed if share > 0 else None, y)
    zero = float((y == 0).double().mean())
    assert abs(zero - share) <= 5 * (share * (1 - share) / n) ** 0.5
    if share < 1:
        kept = y[y != 0]
        assert float((kept.double() - 1 / (1 - share)).abs().max()) <= 2 * U / (1 - share)


def test_masked_values_do_not_pass_and_in_place(gf):
    """A dropped NaN or infinity counts as zero; y may be x or residual."""
    n, p = 5003, 0.5
    seed, words = seed_words(5, -1)
    x, res = draw(n, 4), draw(n, 5)
    gone = dropped(np.ones(n), p, words) == 0
    x[torch.from_numpy(gone)] = float("nan")
    x[torch.from_numpy(np.flatnonzero(gone)[::2].copy())] = float("inf")
    desc = gf.make_dropout_desc(n, p=p)
    want = np.where(gone, 0, np.nan_to_num(f64(x), nan=0, posinf=0) * 2) + f64(res)
    for into in ("new", "x", "res"):
        a, b = x.cuda(), res.cuda()
        y = {"new": torch.empty_like(a), "x": a, "res": b}[into]
        gf.gf_dropout_forward(desc, a, b, seed, y)
        assert (np.abs(f64(y) - want) <= 4 * U * (2 * np.abs(want) + 4 * np.abs(f64(res)))).all()


def test_another_seed_or_offset_is_another_mask_and_elements_are_independent(gf):
    n = 1 << 20
    x = torch.ones(n, device="cuda")
    masks = []
    for a, b in ((1, 0), (2, 0), (1, 1), (1 + (1 << 32), 0), (1, 1 << 40)):
        y = torch.empty_like(x)
        gf.gf_dropout_forward(gf.make_dropout_desc(n, p=0.5), x, None, seed_words(a, b)[0], y)
        masks.append((y > 0).double() * 2 - 1)
    for i, a in enumerate(masks):
        for b in masks[i + 1:]:
            assert abs(float((a * b).mean())) <= 5 * n ** -0.5
        for lag in (1, 2, 3, 4, 8, 31, 1024):
            assert abs(float((a[lag:] * a[:-lag]).mean())) <= 5.1 * n ** -0.5


def test_more_elements_than_32_bits_count(gf):
    """2^32 + 24 elements of bf16: the last ones have the mask of their own index."""
    n, p = (1 << 32) + 21, 0.5
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    seed, words = seed_words(11, 12)
    gf.gf_dropout_forward(gf.make_dropout_desc(n, dtype=torch.bfloat16, p=p), x, None, seed, x)
    first = (1 << 32) - 4096
    assert np.array_equal(f64(x[first:]), dropped(np.ones(n - first), p, words, first))
    assert np.array_equal(f64(x[:4096]), dropped(np.ones(4096), p, words))
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("form", ["rows", "strided", "unaligned", "channels_last", "empty", "other_stream", "mixed", "eval", "p1"])
def test_module_through_autograd(gf, form):
    shape = {"channels_last": (3, 24, 5, 7), "empty": (0, 24)}.get(form, (35, 24))
    x, res = draw(shape, 6).cuda(), draw(shape, 7).cuda()
    if form == "strided":
        x = draw(shape[::-1], 6).cuda().t()
    elif form == "unaligned":
        x = draw((35 * 24 + 1,), 6).cuda()[1:].view(shape)
    elif form == "channels_last":
        x, res = (t.contiguous(memory_format=torch.channels_last) for t in (x, res))
    elif form == "mixed":
        x = x.bfloat16()
    a, r = x.detach().requires_grad_(True), res.clone(memory_format=torch.preserve_format).requires_grad_(True)
    p = 1.0 if form == "p1" else 0.3
    m = gf.Dropout(p)
    if form == "eval":
        m.eval()
    torch.manual_seed(3)
    side = torch.cuda.Stream() if form == "other_stream" else torch.cuda.current_stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = m(a, r)
        gy = torch.randn_like(y)
        y.backward(gy)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert y.shape == x.shape and y.dtype == res.dtype and a.grad.dtype == x.dtype and torch.equal(r.grad, gy)
    if form == "channels_last":
        assert y.is_contiguous(memory_format=torch.channels_last)
    scale = 1.0 if form == "eval" else 0.0 if form == "p1" else 65536 / (65536 - round(0.3 * 65536))
    kept = (a.grad != 0) if form != "eval" else torch.ones_like(a.grad, dtype=torch.bool)
    tol = dict(rtol=2.0 ** -7 if form == "mixed" else 1e-5, atol=1e-6)
    assert torch.allclose(y.detach(), torch.where(kept, x.float() * scale, 0.0) + res, **tol)
    assert torch.allclose(a.grad.float(), torch.where(kept, gy * scale, 0.0), **tol)
    if x.numel() and form not in ("eval", "p1"):
        assert 0.5 < float(kept.float().mean()) < 0.9


def test_seeds_follow_torchs_generator_and_a_graph_draws_anew(gf):
    x = torch.ones(4096, device="cuda")
    torch.manual_seed(7)
    a = gf.dropout(x, 0.5)
    b = gf.dropout(x, 0.5)
    torch.manual_seed(7)
    assert torch.equal(gf.dropout(x, 0.5), a) and not torch.equal(a, b)
    s = gf.dropout_seed("cuda")
    assert torch.equal(gf.dropout(x, 0.5, seed=s), gf.dropout(x, 0.5, seed=s))
    leaf = torch.ones(4096, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t = leaf.detach().requires_grad_(True)
        y = gf.dropout(t, 0.5)
        g, = torch.autograd.grad(y.sum(), t)
    seen = []
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, g)                          # the same mask both ways
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


@pytest.mark.parametrize("normed", [False, True], ids=["dropout", "norm"])
@pytest.mark.parametrize("n", [4096, 4099])
def test_ties_of_the_sum_are_those_of_the_exact_sum(gf, n, normed):
    """p = 1/4 scales by 4/3, which fp32 holds only nearly.  For x = 3 k the scaled value is the integer 4 k, as the product rounded to
    fp32 is too (4/3 is off by a third of a step, 2^-25 of it: less than half a step of any product), and its sum with an integer residual below 2^12 is exact in fp32: rounded to
    bf16 (to even in ties, which fall on many of these sums) the result is that of 64 bits, to the bit."""
    gen = torch.Generator().manual_seed(5)
    x = 3.0 * torch.randint(-85, 86, (8, n), generator=gen)
    residual = torch.randint(-256, 257, (8, n), generator=gen).double()      # (both exact in bf16: 8 bits)
    seed = torch.tensor([11, 12], device="cuda")
    xb, rb = x.cuda().bfloat16(), residual.cuda().bfloat16()
    assert torch.equal(xb.double().cpu(), x.double()) and torch.equal(rb.double().cpu(), residual)
    kept = gf.dropout(torch.ones(8, n, device="cuda"), 0.25, seed=seed) != 0
    want = (residual + torch.where(kept.cpu(), x.double() / 3.0 * 4.0, 0.0)).cuda()
    got = gf.rms_norm(xb, None, residual=rb, p=0.25, seed=seed)[1] if normed else gf.dropout(xb, 0.25, residual=rb, seed=seed)
    assert torch.equal(got, want.bfloat16())
