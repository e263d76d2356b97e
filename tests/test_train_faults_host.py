"""What goes wrong on the way of the fine-tuning operators has to be seen: waits that run out, copies of an optimiser or a
layer, settings that change between steps.  No GPU needed."""
import copy
import pickle

import pytest
import torch


@pytest.mark.parametrize("turns", [1, 3, 15])
def test_a_wait_that_runs_out_in_any_turn_is_reported(gf, turns):
    """Also in the last one, after which the blocks do not meet."""
    for turn in range(turns):
        assert not gf.gf_selftest_end_of_turn(turn, turns, ok=False, met=True), turn
        assert gf.gf_selftest_end_of_turn(turn, turns, ok=True, met=True), turn
    for turn in range(turns - 1):
        assert not gf.gf_selftest_end_of_turn(turn, turns, ok=True, met=False), turn


def test_the_warp_wait_checks_its_arguments(gf):
    for bad in (0, -1, 10 ** 8 + 1):
        with pytest.raises(gf.GfError) as e:
            gf.gf_selftest_warp_wait(0x1000, bad, 0)
        assert e.value.status == gf.GF_ERR_BAD_DESC
    with pytest.raises(gf.GfError) as e:
        gf.gf_selftest_warp_wait(None, 1000, 0)
    assert e.value.status == gf.GF_ERR_NULL


@pytest.mark.parametrize("how", ["deepcopy", "pickle"])
def test_a_copied_optimizer_has_its_workspaces(gf, how):
    """torch's base class copies settings, state and groups only; step() needs the rest too."""
    opt = gf.Muon([torch.nn.Parameter(torch.zeros(4, 6))], lr=0.5)
    again = copy.deepcopy(opt) if how == "deepcopy" else pickle.loads(pickle.dumps(opt))
    assert again._workspaces == {} and again._workspaces is not opt._workspaces
    assert again.param_groups[0]["lr"] == 0.5
    p = again.param_groups[0]["params"][0]
    p.grad = torch.zeros_like(p)
    with pytest.raises(RuntimeError, match="no CPU path"):      # as far as a step gets here
        again.step()


def test_a_loaded_momentum_keeps_its_32_bits(gf):
    """Also with 16-bit parameters, to whose dtype torch casts a state; the saved tensors stay the saver's own, and a hook that
    changes the state on its way in is heard."""
    params = [torch.nn.Parameter(torch.zeros(4, 6, dtype=dt)) for dt in (torch.bfloat16, torch.float32, torch.bfloat16)]
    opt = gf.Muon([{"params": params[:2]}, {"params": params[2:], "lr": 0.25}])
    g = torch.Generator()
    g.manual_seed(1)
    for p in params[:2]:      # the third has not been updated yet
        opt.state[p]["momentum"] = torch.randn(4, 6, generator=g)
    saved = opt.state_dict()
    fresh = [torch.nn.Parameter(p.detach().clone()) for p in params]
    again = gf.Muon([{"params": fresh[:2]}, {"params": fresh[2:]}])
    again.load_state_dict(saved)
    for p, q in zip(params[:2], fresh):
        m = again.state[q]["momentum"]
        assert m.dtype == torch.float32 and torch.equal(m, opt.state[p]["momentum"])
        m.zero_()
        assert bool(opt.state[p]["momentum"].any())
    assert "momentum" not in again.state.get(fresh[2], {}) and again.param_groups[1]["lr"] == 0.25

    def doubled(_, d):
        return {**d, "state": {k: {"momentum": 2 * v["momentum"]} for k, v in d["state"].items()}}

    again.register_load_state_dict_pre_hook(doubled)
    again.load_state_dict(saved)
    assert torch.equal(again.state[fresh[0]]["momentum"], 2 * opt.state[params[0]]["momentum"])


@pytest.mark.parametrize("how", ["deepcopy", "copy", "pickle", "inside"])
def test_a_copied_layer_keeps_what_its_weight_says_of_the_gradient(gf, how):
    for r in (1, 2):
        conv = gf.FilteredConv2d(4, 6, 3, r=r)
        if how == "pickle":
            again = pickle.loads(pickle.dumps(conv))
        elif how == "inside":      # a layer of a model, copied with its optimiser
            model, opt = copy.deepcopy((torch.nn.Sequential(conv), gf.Muon([conv.weight])))
            again = model[0]
            assert opt.param_groups[0]["params"][0] is again.weight
        else:
            again = getattr(copy, how)(conv)
        assert again.weight.filtered_taps is (r == 2)
        assert torch.equal(again.weight, conv.weight) and again.r == r and "_weight_filtered_taps" not in again.__dict__


def test_exact_gradients_take_the_mark_of_equal_taps_off(gf, monkeypatch):
    """r is read at every call: once a call with r = 1 can put exact gradients into a weight, Muon must not read one tap for
    all of them any more, whatever r is set to later."""
    from paper_2301_00330_b200 import autograd
    monkeypatch.setattr(autograd._FilteredConv2dFn, "apply", lambda x, *_: x)
    x = torch.zeros(1, 4, 6, 6)
    conv = gf.FilteredConv2d(4, 6, 3, r=2, bias=False)
    conv(x)
    assert conv.weight.filtered_taps
    conv.r = 1
    with torch.no_grad():
        conv(x)
    assert conv.weight.filtered_taps            # nothing was tracked
    conv(x)
    assert not conv.weight.filtered_taps
    conv.r = 2
    conv(x)
    assert not conv.weight.filtered_taps        # the momentum holds exact gradients
    conv = gf.FilteredConv2d(4, 6, 3, r=2, bias=False)
    gf.filtered_conv2d(x, conv.weight, r=1)
    assert not conv.weight.filtered_taps


def test_every_parameter_group_is_checked(gf):
    """Groups that are added later, and settings of a group of its own."""
    matrix = lambda: torch.nn.Parameter(torch.zeros(8, 4))  # noqa: E731
    opt = gf.Muon([matrix()])
    with pytest.raises(ValueError, match="matrices"):
        opt.add_param_group({"params": [torch.nn.Parameter(torch.zeros(8))]})
    for bad in ({"lr": -1.0}, {"momentum": 1.0}, {"weight_decay": -0.1}, {"precision": "tf32"}):
        with pytest.raises(ValueError):
            opt.add_param_group({"params": [matrix()], **bad})
        with pytest.raises(ValueError):
            gf.Muon([{"params": [matrix()], **bad}])
    assert len(opt.param_groups) == 1
    opt.add_param_group({"params": (matrix() for _ in range(2)), "lr": 0.5})
    opt.add_param_group({"params": matrix()})
    assert [len(g["params"]) for g in opt.param_groups] == [1, 2, 1] and opt.param_groups[1]["lr"] == 0.5
    named = gf.Muon(torch.nn.Linear(4, 8, bias=False).named_parameters())
    assert len(named.param_groups[0]["params"]) == 1


@pytest.mark.parametrize("shape", [(0, 4), (4, 0), (6, 0, 3, 3)])
def test_a_parameter_without_elements_is_left_alone(gf, shape):
    p = torch.nn.Parameter(torch.zeros(shape))
    opt = gf.Muon([p])
    p.grad = torch.zeros(shape)
    opt.step()
    assert not opt.state


def test_layer_norm_refuses_parameters_of_another_device(gf):
    """A weight of another GPU would reach the kernel as an address.  (Tensors without memory stand in for those of two GPUs.)"""
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        x, near, far = (torch.empty(n, device=f"cuda:{d}") for n, d in (((4, 8), 0), ((8,), 0), ((8,), 1)))
        assert x.is_cuda and far.device.index == 1
        for weight, bias in ((far, None), (None, far), (near, far), (far, near)):
            with pytest.raises(ValueError, match="device"):
                gf.layer_norm(x, weight, bias)


def test_newton_schulz_refuses_an_unknown_precision(gf):
    """As Muon does, and not as a missing key.  (Tensors without memory stand in for those of a GPU.)"""
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        G = torch.empty((4, 8), device="cuda:0")
        with pytest.raises(ValueError, match="precision"):
            gf.newton_schulz(G, precision="tf32")
