"""Argument checks of the fine-tuning operators (include/gf_train.h): everything that the host can
detect is refused with its status before anything touches the device."""
import ctypes

import pytest
import torch


def _status(gf, fn, *args, **kw):
    try:
        fn(*args, **kw)
    except gf.GfError as e:
        return e.status
    return gf.GF_OK


def test_norm_descriptor(gf):
    def st(**kw):
        a = {"N": 2, "C": 8, "H": 4, "W": 4} | kw
        return _status(gf, gf.gf_layer_norm_backward_workspace_bytes, gf.make_norm_desc(**a))

    assert st() == gf.GF_OK and st(N=0) == gf.GF_OK and st(layout=gf.GF_NCHW) == gf.GF_OK
    for bad in ({"N": -1}, {"C": 0}, {"H": 0}, {"W": -2}, {"dtype": 3}, {"param_dtype": -1}, {"layout": 2}, {"eps": -1.0},
                {"eps": float("nan")}):
        assert st(**bad) == gf.GF_ERR_BAD_DESC, bad
    assert st(N=1 << 20, H=1 << 10, W=1 << 10) == gf.GF_ERR_UNSUPPORTED       # pixels are counted in 32 bits
    assert st(C=(1 << 24) + 1) == gf.GF_ERR_UNSUPPORTED
    with pytest.raises(TypeError):
        gf.make_norm_desc(1, 8, dtype=torch.float16)


def test_norm_pointers(gf):
    L, vp = gf.lib(), ctypes.c_void_p
    d = gf.make_norm_desc(4, 8)
    r, a, odd = ctypes.byref(d), vp(0x1000), vp(0x1004)      # never dereferenced: all calls fail on the host
    assert L.gf_layer_norm_forward(None, a, a, a, a, a, a, None) == gf.GF_ERR_NULL
    assert L.gf_layer_norm_forward(r, None, a, a, a, a, a, None) == gf.GF_ERR_NULL
    assert L.gf_layer_norm_forward(r, a, a, a, None, a, a, None) == gf.GF_ERR_NULL
    assert L.gf_layer_norm_forward(r, a, a, a, a, a, None, None) == gf.GF_ERR_NULL      # mean without rstd
    assert L.gf_layer_norm_forward(r, a, odd, a, a, a, a, None) == gf.GF_ERR_ALIGN
    big = 1 << 30
    assert L.gf_layer_norm_backward(r, None, a, a, a, a, a, a, a, a, big, None) == gf.GF_ERR_NULL
    assert L.gf_layer_norm_backward(r, a, a, a, a, a, a, a, a, None, big, None) == gf.GF_ERR_NULL
    assert L.gf_layer_norm_backward(r, a, a, a, odd, a, a, a, a, a, big, None) == gf.GF_ERR_ALIGN
    need = gf.gf_layer_norm_backward_workspace_bytes(d)
    assert L.gf_layer_norm_backward(r, a, a, a, a, a, a, a, a, a, need - 1, None) == gf.GF_ERR_WORKSPACE
    assert L.gf_layer_norm_backward(r, a, a, a, a, a, None, None, None, None, 0, None) == gf.GF_OK    # nothing wanted


def test_layer_norm_refuses_what_it_cannot_take(gf):
    with pytest.raises(RuntimeError, match="no CPU path"):
        gf.layer_norm(torch.zeros(2, 8))
    with pytest.raises(ValueError):
        gf.layer_norm(torch.zeros(2, 8, 4), channel_dim=1)
    with pytest.raises(ValueError):
        gf.layer_norm(torch.zeros(2, 8, 4, 4), channel_dim=2)


def test_newton_schulz_and_muon_descriptors(gf):
    def ns(**kw):
        a = {"batch": 1, "rows": 8, "cols": 8} | kw
        return _status(gf, gf.gf_newton_schulz_workspace_bytes, gf.make_ns_desc(**a))

    def muon(**kw):
        a = {"count": 1, "rows": 8, "cols": 8} | kw
        return _status(gf, gf.gf_muon_workspace_bytes, gf.make_muon_desc(**a))

    assert ns() == gf.GF_OK and ns(batch=0) == gf.GF_OK and muon() == gf.GF_OK and muon(taps=49) == gf.GF_OK
    common = ({"rows": 0}, {"cols": -1}, {"precision": 2}, {"steps": 0}, {"steps": gf.GF_NS_MAX_STEPS + 1}, {"eps": -1e-7})
    for bad in common + ({"batch": -1}, {"in_dtype": 2}, {"out_dtype": -1}):
        assert ns(**bad) == gf.GF_ERR_BAD_DESC, bad
    for bad in common + ({"count": -1}, {"grad_dtype": 2}, {"weight_dtype": 5}, {"taps": 0}, {"nesterov": 2}):
        assert muon(**bad) == gf.GF_ERR_BAD_DESC, bad
    assert ns(rows=16385) == gf.GF_ERR_UNSUPPORTED and muon(cols=16385) == gf.GF_ERR_UNSUPPORTED
    assert muon(taps=5000) == gf.GF_ERR_UNSUPPORTED


def test_newton_schulz_and_muon_pointers(gf):
    L, vp = gf.lib(), ctypes.c_void_p
    a, odd, big = vp(0x1000), vp(0x1008), 1 << 30
    d = gf.make_ns_desc(1, 8, 8)
    r, need = ctypes.byref(d), gf.gf_newton_schulz_workspace_bytes(d)
    assert L.gf_newton_schulz(r, None, a, a, big, None, None) == gf.GF_ERR_NULL
    assert L.gf_newton_schulz(r, a, None, a, big, None, None) == gf.GF_ERR_NULL
    assert L.gf_newton_schulz(r, a, a, None, big, None, None) == gf.GF_ERR_NULL
    assert L.gf_newton_schulz(r, a, odd, a, big, None, None) == gf.GF_ERR_ALIGN
    assert L.gf_newton_schulz(r, a, a, a, need - 1, None, None) == gf.GF_ERR_WORKSPACE
    m = gf.make_muon_desc(2, 8, 8)
    r, need = ctypes.byref(m), gf.gf_muon_workspace_bytes(m)
    two, hole, off = (vp * 2)(0x1000, 0x2000), (vp * 2)(0x1000, 0), (vp * 2)(0x1000, 0x2002)
    assert L.gf_muon_step(r, None, two, two, two, two, a, big, None, None) == gf.GF_ERR_NULL
    assert L.gf_muon_step(r, two, two, hole, two, two, a, big, None, None) == gf.GF_ERR_NULL
    assert L.gf_muon_step(r, two, two, two, two, off, a, big, None, None) == gf.GF_ERR_ALIGN
    assert L.gf_muon_step(r, two, two, two, two, two, a, need - 1, None, None) == gf.GF_ERR_WORKSPACE
    empty = gf.make_muon_desc(0, 8, 8)
    assert L.gf_muon_step(ctypes.byref(empty), None, None, None, None, None, None, 0, None, None) == gf.GF_OK


def test_muon_and_newton_schulz_refuse_what_they_cannot_take(gf):
    with pytest.raises(RuntimeError, match="no CPU path"):
        gf.newton_schulz(torch.zeros(4, 4))
    with pytest.raises(ValueError):
        gf.Muon([torch.nn.Parameter(torch.zeros(8))])
    with pytest.raises(ValueError):
        gf.Muon([torch.nn.Parameter(torch.zeros(8, 8))], precision="tf32")
    with pytest.raises(ValueError):
        gf.gf_newton_schulz(gf.make_ns_desc(1, 8, 8), None, None, None, 0, [(1.0, 2.0, 3.0)], 0)      # one triple for five steps
    p = torch.nn.Parameter(torch.zeros(8, 8))
    p.grad = torch.zeros(8, 8)
    with pytest.raises(RuntimeError, match="no CPU path"):
        gf.Muon([p]).step()
