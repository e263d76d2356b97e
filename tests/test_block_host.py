"""Argument checks of the residual-block operators (include/gf_block.h): everything that the host can detect is refused with its
status before anything touches the device."""
import ctypes

import pytest
import torch


def _status(gf, fn, *args, **kw):
    try:
        fn(*args, **kw)
    except gf.GfError as e:
        return e.status
    return gf.GF_OK


def test_dropout_refusals(gf):
    L, vp = gf.lib(), ctypes.c_void_p
    a, odd = vp(0x1000), vp(0x1008)                      # never dereferenced: all calls fail on the host

    def fwd(desc, x=a, res=a, seed=odd, y=a):
        return L.gf_dropout_forward(ctypes.byref(desc), x, res, seed, y, None)

    def mk(count=8, p=0.5, **kw):
        return gf.make_dropout_desc(count, p=p, **kw)

    assert L.gf_dropout_forward(None, a, a, a, a, None) == gf.GF_ERR_NULL
    assert fwd(mk(0), None, None, None, None) == gf.GF_OK
    for bad in (mk(-1), mk(p=-0.1), mk(p=1.5), mk(p=float("nan")), mk(dtype=2), mk(out_dtype=-1)):
        assert fwd(bad) == gf.GF_ERR_BAD_DESC
    assert fwd(mk((1 << 43) + 1)) == gf.GF_ERR_UNSUPPORTED
    assert fwd(mk(), None) == gf.GF_ERR_NULL and fwd(mk(), y=None) == gf.GF_ERR_NULL and fwd(mk(), seed=None) == gf.GF_ERR_NULL
    assert fwd(mk(), odd) == gf.GF_ERR_ALIGN and fwd(mk(), res=odd) == gf.GF_ERR_ALIGN and fwd(mk(), y=odd) == gf.GF_ERR_ALIGN
    assert fwd(mk(), seed=vp(0x1004)) == gf.GF_ERR_ALIGN
    d = ctypes.byref(mk())
    assert L.gf_dropout_backward(d, None, a, a, None) == gf.GF_ERR_NULL and L.gf_dropout_backward(d, a, None, a, None) == gf.GF_ERR_NULL
    assert L.gf_dropout_backward(d, a, a, odd, None) == gf.GF_ERR_ALIGN
    with pytest.raises(TypeError):
        gf.make_dropout_desc(8, dtype=torch.float16, p=0.1)
    x = torch.zeros(4, 8)
    with pytest.raises(RuntimeError, match="no CPU path"):
        gf.dropout(x, 0.1)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError):
            gf.dropout(x, p)
        with pytest.raises(ValueError):
            gf.Dropout(p)


def test_rms_descriptor(gf):
    def st(**kw):
        a = {"rows": 4, "cols": 8} | kw
        return _status(gf, gf.gf_rms_norm_backward_workspace_bytes, gf.make_rms_desc(**a))

    assert st() == gf.GF_OK and st(rows=0) == gf.GF_OK and st(p=1.0) == gf.GF_OK
    for bad in ({"rows": -1}, {"cols": 0}, {"dtype": 3}, {"residual_dtype": 2}, {"param_dtype": -1}, {"eps": -1.0}, {"eps": float("nan")},
                {"p": -0.5}, {"p": 1.01}, {"p": float("nan")}):
        assert st(**bad) == gf.GF_ERR_BAD_DESC, bad
    for far in ({"cols": (1 << 24) + 1}, {"rows": 1 << 59}, {"dtype": gf.GF_F32, "residual_dtype": gf.GF_BF16}):
        assert st(**far) == gf.GF_ERR_UNSUPPORTED, far


def test_rms_pointers(gf):
    L, vp = gf.lib(), ctypes.c_void_p
    a, odd = vp(0x1000), vp(0x1008)
    plain, drop = gf.make_rms_desc(4, 8), gf.make_rms_desc(4, 8, p=0.5)

    def fwd(d=plain, x=a, res=a, seed=None, gamma=a, h=a, y=a, rstd=a):
        return L.gf_rms_norm_forward(ctypes.byref(d), x, res, seed, gamma, h, y, rstd, None)

    def fwd8(d=plain, x=a, res=a, seed=None, gamma=a, h=a, codes=a, scales=a, rstd=a):
        return L.gf_rms_norm_forward_fp8(ctypes.byref(d), x, res, seed, gamma, h, codes, scales, rstd, None)

    assert L.gf_rms_norm_forward(None, a, a, a, a, a, a, a, None) == gf.GF_ERR_NULL
    assert L.gf_rms_norm_forward_fp8(None, a, a, a, a, a, a, a, a, None) == gf.GF_ERR_NULL
    for f in (fwd, fwd8):
        assert f(x=None) == gf.GF_ERR_NULL and f(h=None) == gf.GF_ERR_NULL and f(d=drop) == gf.GF_ERR_NULL
        assert f(d=drop, res=None, seed=a, h=None) == gf.GF_ERR_NULL
        assert f(res=None) == gf.GF_ERR_BAD_DESC                     # h is x: it is not written
        assert f(d=gf.make_rms_desc(4, 8, dtype=gf.GF_BF16, residual_dtype=gf.GF_F32), res=None, h=None) == gf.GF_ERR_BAD_DESC
        for k in ("x", "res", "gamma", "h", "rstd"):
            assert f(**{k: odd}) == gf.GF_ERR_ALIGN, k
        assert f(d=drop, seed=vp(0x1004)) == gf.GF_ERR_ALIGN
    assert fwd(y=None) == gf.GF_ERR_NULL and fwd(y=odd) == gf.GF_ERR_ALIGN
    assert fwd8(codes=None) == gf.GF_ERR_NULL and fwd8(scales=None) == gf.GF_ERR_NULL and fwd8(codes=odd) == gf.GF_ERR_ALIGN
    assert fwd8(d=gf.make_rms_desc(1 << 31, 8)) == gf.GF_ERR_UNSUPPORTED

    for cols in (8, 1001, 20000):
        d = gf.make_rms_desc(4, cols)
        need = gf.gf_rms_norm_backward_workspace_bytes(d)

        def bwd(d=d, gy=a, gh=a, h=a, rstd=a, gamma=a, seed=None, gres=a, gx=a, gw=a, ws=a, n=need):
            return L.gf_rms_norm_backward(ctypes.byref(d), gy, gh, h, rstd, gamma, seed, gres, gx, gw, ws, n, None)

        for k in ("gy", "h", "rstd", "ws"):
            assert bwd(**{k: None}) == gf.GF_ERR_NULL, k
        for k in ("gy", "gh", "h", "rstd", "gamma", "gres", "gx", "gw", "ws"):
            assert bwd(**{k: odd}) == gf.GF_ERR_ALIGN, k
        assert bwd(n=need - 1) == gf.GF_ERR_WORKSPACE
        assert bwd(d=gf.make_rms_desc(4, cols, p=0.5)) == gf.GF_ERR_NULL
        assert bwd(gres=None, gx=None, gw=None, ws=None, n=0, gy=None) == gf.GF_OK          # nothing wanted


def test_rms_norm_refuses_what_it_cannot_take(gf):
    x = torch.zeros(4, 8)
    for fn in (gf.rms_norm, lambda t, *a, **k: gf.rms_norm_linear(t, None, [], *a, **k)):
        with pytest.raises(RuntimeError, match="no CPU path"):
            fn(x)
    with pytest.raises(ValueError):
        gf.RMSNorm(8, p=2.0)


def test_fp8_refusals(gf):
    L, vp = gf.lib(), ctypes.c_void_p
    a, odd = vp(0x1000), vp(0x1008)
    for fn in (L.gf_fp8_quantize_rows, L.gf_fp8_quantize_blocks):
        def st(x=a, codes=a, scales=a, **kw):
            return fn(ctypes.byref(gf.make_fp8_desc(**({"rows": 4, "cols": 8} | kw))), x, codes, scales, None)

        assert fn(None, a, a, a, None) == gf.GF_ERR_NULL
        assert st(rows=0, x=None, codes=None, scales=None) == gf.GF_OK
        for bad in ({"rows": -1}, {"cols": 0}, {"dtype": 2}):
            assert st(**bad) == gf.GF_ERR_BAD_DESC
        assert st(cols=(1 << 24) + 1) == gf.GF_ERR_UNSUPPORTED
        for k in ("x", "codes", "scales"):
            assert st(**{k: None}) == gf.GF_ERR_NULL and st(**{k: odd}) == gf.GF_ERR_ALIGN

    def mm(a_=a, sa=a, w=a, sw=a, bias=a, out=a, **kw):
        d = gf.make_fp8_matmul_desc(**({"M": 4, "N": 8, "K": 8} | kw))
        return L.gf_fp8_matmul(ctypes.byref(d), a_, sa, w, sw, bias, out, None)

    assert L.gf_fp8_matmul(None, a, a, a, a, a, a, None) == gf.GF_ERR_NULL
    assert mm(M=0, a_=None, sa=None, w=None, sw=None, bias=None, out=None) == gf.GF_OK
    for bad in ({"M": -1}, {"N": 0}, {"K": 0}, {"transposed": 2}, {"out_dtype": 3}, {"bias_dtype": 2}):
        assert mm(**bad) == gf.GF_ERR_BAD_DESC, bad
    assert mm(N=(1 << 24) + 1) == gf.GF_ERR_UNSUPPORTED and mm(K=(1 << 24) + 1) == gf.GF_ERR_UNSUPPORTED
    for k in ("a_", "sa", "w", "sw", "out"):
        assert mm(**{k: None}) == gf.GF_ERR_NULL and mm(**{k: odd}) == gf.GF_ERR_ALIGN, k
    assert mm(bias=odd) == gf.GF_ERR_ALIGN


def test_fp8_wrappers_refuse_what_they_cannot_take(gf):
    for fn in (gf.quantize_rows, gf.quantize_weight, gf.Fp8Linear):
        with pytest.raises(RuntimeError, match="no CPU path"):
            fn(torch.zeros(4, 8))
    with pytest.raises(ValueError):
        gf.Fp8Linear(torch.zeros(4, 8), channel_dim=2)
    for bad in (torch.nn.Conv2d(8, 8, 3), torch.nn.Conv2d(8, 8, 1, stride=2), torch.nn.Conv2d(8, 8, 1, groups=2), torch.nn.Conv2d(8, 8, 1, padding=1),
                gf.FilteredConv2d(8, 8, 3), gf.FilteredConv2d(8, 8, 1, stride=2)):
        with pytest.raises(ValueError):
            gf.Fp8Linear.from_layer(bad)
    rows = gf.Fp8Matrix(torch.zeros((4, 16), dtype=torch.uint8), torch.zeros(1, 4), 4, 8, False)
    blocks = gf.Fp8Matrix(torch.zeros((4, 16), dtype=torch.uint8), torch.zeros(1, 1), 4, 8, True)
    for args in ((rows, rows), (blocks, blocks)):
        with pytest.raises(ValueError, match="scales"):
            gf.fp8_matmul(*args)
    with pytest.raises(ValueError, match="columns"):
        gf.fp8_matmul(rows, blocks, transposed=True)
    with pytest.raises(ValueError, match="CUDA"):
        gf.fp8_matmul(rows, blocks)
    for bad in (gf.Fp8Matrix(torch.zeros((4, 8), dtype=torch.uint8), rows.scales, 4, 8, False), gf.Fp8Matrix(rows.codes, torch.zeros(1, 3), 4, 8, False),
                gf.Fp8Matrix(rows.codes.short(), rows.scales, 4, 8, False), gf.Fp8Matrix(rows.codes, rows.scales.double(), 4, 8, False)):
        with pytest.raises(ValueError, match="expected"):
            gf.fp8_matmul(bad, blocks)
        with pytest.raises(ValueError, match="expected"):
            bad.dequantize()


def test_the_format_of_8_bit_values(gf):
    """The tests' own table of e4m3 against torch's type."""
    from block_util import e4m3_codes, e4m3_values
    import numpy as np

    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(e4m3_values(codes), want, equal_nan=True)
    v = np.concatenate([np.linspace(-448, 448, 100001), 2.0 ** -np.arange(0, 14.0), want[np.isfinite(want)]]).astype(np.float32)
    assert np.array_equal(e4m3_codes(v), torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert gf.fp8_pitch(17) == 32 and gf.fp8_pitch(16) == 16 and gf.fp8_scale_pitch(5) == 8
