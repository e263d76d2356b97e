"""What goes wrong on the way of the fine-tuning operators, on the GPU: waits that run out end their kernels in an orderly way."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_lanes_of_a_warp_give_up_together(gf):
    """Half of the lanes are told to wait for half a millisecond, half for 32, the barrier completes after 4: the lanes that saw it must
    not go on without the others."""
    result = torch.full((32,), 7, dtype=torch.int32, device="cuda")
    gf.gf_selftest_warp_wait(result, 1_000_000)
    torch.cuda.synchronize()
    assert bool((result == 0).all()), result.tolist()


def test_a_resumed_optimizer_goes_on_as_the_uninterrupted_one(gf):
    """16-bit weights, 32-bit momentum: saving and loading between two steps changes no bit of the weights."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    start = torch.randn(40, 24, generator=g, device="cuda").bfloat16()
    grads = [torch.randn(40, 24, generator=g, device="cuda").bfloat16() for _ in range(3)]
    p = torch.nn.Parameter(start.clone())
    opt = gf.Muon([p], lr=0.1)
    for k, grad in enumerate(grads):
        if k == 2:      # a second optimiser takes over here
            q = torch.nn.Parameter(p.detach().clone())
            other = gf.Muon([q], lr=0.1)
            other.load_state_dict(opt.state_dict())
            q.grad = grad.clone()
            other.step()
        p.grad = grad.clone()
        opt.step()
    assert torch.equal(p, q) and torch.equal(opt.state[p]["momentum"], other.state[q]["momentum"])
    assert not torch.equal(p, start)


def test_switching_a_layer_to_exact_gradients_reaches_its_update(gf):
    """Two steps with filtered gradients, two with exact ones after conv.r = 1, one with filtered ones again: the updates are those
    of an optimiser that never counted on equal taps.  Bound as where equal taps are compared with flattened kernels; with
    one tap read for all the weights would be off by the size of a step, about 1e-2 of them."""
    torch.manual_seed(5)
    conv = gf.FilteredConv2d(12, 20, 3, r=2, bias=False, device="cuda")
    twin = torch.nn.Parameter(conv.weight.detach().clone())
    opt, other = gf.Muon([conv.weight], lr=1e-2, weight_decay=0.1), gf.Muon([twin], lr=1e-2, weight_decay=0.1, filtered_taps=False)
    for r in (2, 2, 1, 1, 2):
        conv.r = r
        x = torch.randn(2, 12, 16, 16, device="cuda")
        conv.weight.grad = None
        conv(x).square().mean().backward()
        taps = conv.weight.grad.flatten(2)
        assert bool((taps == taps[..., :1]).all()) == (r == 2)
        twin.grad = conv.weight.grad.clone()
        opt.step()
        other.step()
        assert float((conv.weight - twin).detach().norm() / twin.detach().norm()) <= 1e-5, r
    assert opt.state[conv.weight]["momentum"].shape == (20, 108)


@pytest.mark.parametrize("bad", ["transposed", "too wide", "16-bit float", "sparse", "momentum", "on the CPU"])
def test_a_step_that_is_refused_changes_nothing(gf, bad):
    """A parameter that Muon cannot take, behind others that it can: their weights and their state stay as they were."""
    good = torch.nn.Parameter(torch.ones(8, 6, device="cuda"))
    other = torch.nn.Parameter({"transposed": lambda: torch.ones(6, 4, device="cuda").t(),
                                "too wide": lambda: torch.ones(2, 16385, device="cuda"),
                                "16-bit float": lambda: torch.ones(4, 6, device="cuda", dtype=torch.float16),
                                "on the CPU": lambda: torch.ones(4, 6)}.get(bad, lambda: torch.ones(4, 6, device="cuda"))())
    opt = gf.Muon([{"params": [good]}, {"params": [other]}])
    good.grad = torch.ones_like(good)
    other.grad = torch.ones_like(other).to_sparse() if bad == "sparse" else torch.ones_like(other)
    if bad == "momentum":
        opt.state[other]["momentum"] = torch.zeros(3, 3, device="cuda")
    before = gf.gf_kernel_launch_count()
    with pytest.raises((ValueError, TypeError, RuntimeError)):      # GfError is a RuntimeError
        opt.step()
    torch.cuda.synchronize()
    assert bool((good == 1).all()) and "momentum" not in opt.state.get(good, {}) and gf.gf_kernel_launch_count() == before


def test_autograd_sees_that_a_step_has_changed_the_weights(gf):
    """backward() through a graph that saved a weight before the step is refused, as with torch's optimisers, instead of
    giving gradients of a mixture of old activations and new weights."""
    p = torch.nn.Parameter(torch.randn(6, 5, device="cuda"))
    x = torch.randn(3, 5, device="cuda", requires_grad=True)
    opt = gf.Muon([p])
    y = x @ p.t()
    p.grad = torch.ones_like(p)
    version = p._version
    opt.step()
    assert p._version > version
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()


def test_the_timing_of_a_step_covers_all_its_kernels(gf):
    """Sums of squares, products and the kernel that writes the results: each launch lies between events of its own kind."""
    rows, cols = 200, 160
    G = torch.randn(1, rows, cols, device="cuda")
    O, desc = torch.empty_like(G), gf.make_ns_desc(1, rows, cols)
    muon = gf.make_muon_desc(1, rows, cols)
    ws = torch.empty(max(gf.gf_newton_schulz_workspace_bytes(desc), gf.gf_muon_workspace_bytes(muon)), dtype=torch.uint8, device="cuda")
    m, w = torch.zeros(rows, cols, device="cuda"), torch.zeros(rows, cols, device="cuda")
    gf.gf_profile_read()
    gf.gf_profile_configure(2)
    try:
        gf.gf_newton_schulz(desc, G, O, ws)
        gf.gf_muon_step(muon, [G], [m], [w], [m], [w], ws)
        got = gf.gf_profile_read()
    finally:
        gf.gf_profile_configure(0)
    assert {name: n for name, (n, _) in got.items()} == {"ns_prepare": 2, "ns_product": 2, "ns_finish": 2}
    assert all(ms > 0 for _, ms in got.values())
