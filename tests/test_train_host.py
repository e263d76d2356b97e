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
