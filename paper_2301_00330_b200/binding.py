"""ctypes binding over the C ABI declared in include/gf.h, include/gf_train.h and include/gf_block.h.

Argument marshalling only: every step of the method runs in the CUDA kernels
of libgf_b200.so.  torch is used for device memory and streams.  There is no
CPU fallback: if the library is missing or cannot be loaded, every entry point
raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

from . import build as _build

GF_OK, GF_ERR_NULL, GF_ERR_BAD_DESC, GF_ERR_UNSUPPORTED = 0, 1, 2, 3
GF_ERR_WORKSPACE, GF_ERR_ALIGN, GF_ERR_CUDA, GF_ERR_TIMEOUT = 4, 5, 6, 7
GF_F32, GF_BF16 = 0, 1
GF_NCHW, GF_NHWC = 0, 1
GF_PATH_AUTO, GF_PATH_FUSED, GF_PATH_SPLIT = 0, 1, 2
GF_ACT_NONE, GF_ACT_RELU, GF_ACT_RELU6 = 0, 1, 2
GF_NS_F16, GF_NS_F32 = 0, 1
GF_NS_MAX_STEPS = 16

EXPORTS = (
    "gf_stash_dims", "gf_stash_bytes", "gf_backward_workspace_bytes", "gf_stash_forward",
    "gf_backward", "gf_last_async_status", "gf_host_step_arena_bytes", "gf_layer_step_host",
    "gf_kernel_launch_count", "gf_status_string", "gf_profile_configure", "gf_profile_read",
    "gf_kernel_name", "gf_kernel_id_count", "gf_backward_static_scratch", "gf_set_dense_path",
    "gf_snr_terms", "gf_filter_snr_terms", "gf_dcac_ratio", "gf_act_stash_forward",
    "gf_backward_int8", "gf_backward_int8_workspace_bytes", "gf_selftest_bounded_wait",
    "gf_layer_norm_forward", "gf_layer_norm_backward_workspace_bytes", "gf_layer_norm_backward",
    "gf_newton_schulz_workspace_bytes", "gf_newton_schulz", "gf_muon_workspace_bytes", "gf_muon_step",
    "gf_selftest_end_of_turn", "gf_selftest_warp_wait",
    "gf_dropout_forward", "gf_dropout_backward", "gf_rms_norm_forward", "gf_rms_norm_forward_fp8",
    "gf_rms_norm_backward_workspace_bytes", "gf_rms_norm_backward", "gf_fp8_quantize_rows", "gf_fp8_quantize_blocks",
    "gf_fp8_matmul", "gf_selftest_fp8_form",
)


class gf_conv_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("N", "C_in", "C_out", "H", "W", "KH", "KW", "stride", "pad_h", "pad_w",
                 "groups", "r", "dtype", "layout")]


class gf_norm_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "C", "H", "W", "dtype", "param_dtype", "layout")] + [("eps", ctypes.c_float)]


class gf_ns_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "rows", "cols", "in_dtype", "out_dtype", "precision", "steps")] + [("eps", ctypes.c_float)]


class gf_muon_desc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("count", "rows", "cols", "taps", "grad_dtype", "weight_dtype", "precision",
                                               "steps", "nesterov")]
                + [(n, ctypes.c_float) for n in ("eps", "momentum", "lr", "weight_decay", "scale")])


class gf_dropout_desc(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int64), ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("p", ctypes.c_float)]


class gf_rms_desc(ctypes.Structure):
    _fields_ = ([("rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("cols", "dtype", "residual_dtype", "param_dtype")]
                + [("eps", ctypes.c_float), ("p", ctypes.c_float)])


class gf_fp8_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "cols", "dtype")]


class gf_fp8_matmul_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("M", "N", "K", "transposed", "out_dtype", "bias_dtype")]


class gf_kernel_time(ctypes.Structure):
    _fields_ = [("kernel_id", ctypes.c_int32), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_double)]


class GfError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


_lib = None


def library_path() -> str:
    return _build.LIB


def build_library(force: bool = False) -> str:
    """Compile libgf_b200.so for sm_100a if it is missing or stale."""
    return _build.build(force=force)


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with `python -m paper_2301_00330_b200.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(path)
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        dp = ctypes.POINTER(gf_conv_desc)
        L.gf_stash_dims.argtypes = [dp, ctypes.POINTER(ctypes.c_int64 * 4)]
        L.gf_stash_bytes.argtypes = [dp, ctypes.POINTER(sz)]
        L.gf_backward_workspace_bytes.argtypes = [dp, ctypes.POINTER(sz)]
        L.gf_stash_forward.argtypes = [dp, vp, vp, vp]
        L.gf_act_stash_forward.argtypes = [dp, ctypes.c_int32, vp, vp, vp, vp]
        L.gf_act_stash_forward.restype = ctypes.c_int
        L.gf_backward.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gf_backward_int8.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gf_backward_int8.restype = ctypes.c_int
        L.gf_backward_int8_workspace_bytes.argtypes = [dp, ctypes.POINTER(sz)]
        L.gf_backward_int8_workspace_bytes.restype = ctypes.c_int
        L.gf_backward_static_scratch.argtypes = [dp, vp, vp, vp, vp, vp, vp]
        L.gf_backward_static_scratch.restype = ctypes.c_int
        L.gf_last_async_status.argtypes = [vp, vp]
        L.gf_host_step_arena_bytes.argtypes = [dp, ctypes.POINTER(sz)]
        L.gf_layer_step_host.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gf_kernel_launch_count.argtypes = []
        L.gf_kernel_launch_count.restype = ctypes.c_uint64
        L.gf_profile_configure.argtypes = [ctypes.c_int32, ctypes.c_int32]
        L.gf_profile_configure.restype = ctypes.c_int
        L.gf_profile_read.argtypes = [ctypes.POINTER(gf_kernel_time), ctypes.c_int32]
        L.gf_profile_read.restype = ctypes.c_int32
        L.gf_kernel_name.argtypes = [ctypes.c_int32]
        L.gf_kernel_name.restype = ctypes.c_char_p
        L.gf_kernel_id_count.argtypes = []
        L.gf_kernel_id_count.restype = ctypes.c_int32
        L.gf_set_dense_path.argtypes = [ctypes.c_int32]
        L.gf_set_dense_path.restype = ctypes.c_int
        i32, i64 = ctypes.c_int32, ctypes.c_int64
        L.gf_snr_terms.argtypes = [vp, vp, i64, i32, vp, vp]
        L.gf_filter_snr_terms.argtypes = [vp, i64, i32, i32, i32, i32, vp, vp]
        L.gf_dcac_ratio.argtypes = [vp, i32, i32, i32, i32, i32, i32, i32, vp, vp]
        for name in ("gf_snr_terms", "gf_filter_snr_terms", "gf_dcac_ratio"):
            getattr(L, name).restype = ctypes.c_int
        nd, sd, md = ctypes.POINTER(gf_norm_desc), ctypes.POINTER(gf_ns_desc), ctypes.POINTER(gf_muon_desc)
        L.gf_layer_norm_forward.argtypes = [nd, vp, vp, vp, vp, vp, vp, vp]
        L.gf_layer_norm_backward_workspace_bytes.argtypes = [nd, ctypes.POINTER(sz)]
        L.gf_layer_norm_backward.argtypes = [nd, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gf_newton_schulz_workspace_bytes.argtypes = [sd, ctypes.POINTER(sz)]
        L.gf_newton_schulz.argtypes = [sd, vp, vp, vp, sz, vp, vp]
        L.gf_muon_workspace_bytes.argtypes = [md, ctypes.POINTER(sz)]
        L.gf_muon_step.argtypes = [md, vp, vp, vp, vp, vp, vp, sz, vp, vp]
        for name in ("gf_layer_norm_forward", "gf_layer_norm_backward_workspace_bytes", "gf_layer_norm_backward",
                     "gf_newton_schulz_workspace_bytes", "gf_newton_schulz", "gf_muon_workspace_bytes", "gf_muon_step"):
            getattr(L, name).restype = ctypes.c_int
        od, rd, qd, pd = (ctypes.POINTER(c) for c in (gf_dropout_desc, gf_rms_desc, gf_fp8_desc, gf_fp8_matmul_desc))
        L.gf_dropout_forward.argtypes = [od, vp, vp, vp, vp, vp]
        L.gf_dropout_backward.argtypes = [od, vp, vp, vp, vp]
        L.gf_rms_norm_forward.argtypes = [rd, vp, vp, vp, vp, vp, vp, vp, vp]
        L.gf_rms_norm_forward_fp8.argtypes = [rd, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.gf_rms_norm_backward_workspace_bytes.argtypes = [rd, ctypes.POINTER(sz)]
        L.gf_rms_norm_backward.argtypes = [rd, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gf_fp8_quantize_rows.argtypes = [qd, vp, vp, vp, vp]
        L.gf_fp8_quantize_blocks.argtypes = [qd, vp, vp, vp, vp]
        L.gf_fp8_matmul.argtypes = [pd, vp, vp, vp, vp, vp, vp, vp]
        for name in ("gf_dropout_forward", "gf_dropout_backward", "gf_rms_norm_forward", "gf_rms_norm_forward_fp8",
                     "gf_rms_norm_backward_workspace_bytes", "gf_rms_norm_backward", "gf_fp8_quantize_rows",
                     "gf_fp8_quantize_blocks", "gf_fp8_matmul"):
            getattr(L, name).restype = ctypes.c_int
        L.gf_selftest_fp8_form.argtypes, L.gf_selftest_fp8_form.restype = [pd], i32
        L.gf_selftest_bounded_wait.argtypes = [vp, ctypes.c_int64, vp]
        L.gf_selftest_bounded_wait.restype = ctypes.c_int
        L.gf_selftest_warp_wait.argtypes = [vp, ctypes.c_int64, vp]
        L.gf_selftest_warp_wait.restype = ctypes.c_int
        L.gf_selftest_end_of_turn.argtypes = [i32, i32, i32, i32]
        L.gf_selftest_end_of_turn.restype = i32
        L.gf_status_string.argtypes = [ctypes.c_int]
        L.gf_status_string.restype = ctypes.c_char_p
        for name in ("gf_stash_dims", "gf_stash_bytes", "gf_backward_workspace_bytes", "gf_stash_forward",
                     "gf_backward", "gf_last_async_status", "gf_host_step_arena_bytes", "gf_layer_step_host"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().gf_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != GF_OK:
        raise GfError(status, where)


def make_desc(N, C_in, C_out, H, W, KH, KW=None, *, r, groups=1, stride=1, pad_h=None, pad_w=None,
              dtype=GF_F32, layout=GF_NCHW) -> gf_conv_desc:
    KW = KH if KW is None else KW
    pad_h = (KH - 1) // 2 if pad_h is None else pad_h
    pad_w = (KW - 1) // 2 if pad_w is None else pad_w
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: GF_F32, torch.bfloat16: GF_BF16}[dtype]
    return gf_conv_desc(N, C_in, C_out, H, W, KH, KW, stride, pad_h, pad_w, groups, r, dtype, layout)


def desc_for(layer) -> gf_conv_desc:
    """Descriptor of a workloads.Layer."""
    return make_desc(layer.N, layer.C_in, layer.C_out, layer.H, layer.W, layer.K, r=layer.r,
                     groups=layer.groups, dtype=GF_F32 if layer.dtype == "f32" else GF_BF16)


def _ptr(t) -> ctypes.c_void_p:
    if t is None:
        return ctypes.c_void_p(0)
    if isinstance(t, torch.Tensor):
        # dense in either order; which one the bytes are in is the descriptor's `layout`
        if not (t.is_contiguous() or (t.dim() == 4 and t.is_contiguous(memory_format=torch.channels_last))):
            raise ValueError("tensors passed to the gf_* calls must be dense (contiguous, or channels_last for GF_NHWC)")
        return ctypes.c_void_p(t.data_ptr())
    return ctypes.c_void_p(int(t))


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


# ---- the C calls, same names ----------------------------------------------------

def gf_stash_dims(desc: gf_conv_desc) -> tuple[int, int, int, int]:
    dims = (ctypes.c_int64 * 4)()
    _check(lib().gf_stash_dims(ctypes.byref(desc), ctypes.byref(dims)), "gf_stash_dims")
    return tuple(int(v) for v in dims)


def gf_stash_bytes(desc: gf_conv_desc) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().gf_stash_bytes(ctypes.byref(desc), ctypes.byref(out)), "gf_stash_bytes")
    return int(out.value)


def gf_backward_workspace_bytes(desc: gf_conv_desc) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().gf_backward_workspace_bytes(ctypes.byref(desc), ctypes.byref(out)),
           "gf_backward_workspace_bytes")
    return int(out.value)


def gf_stash_forward(desc: gf_conv_desc, x, stash, stream=None) -> None:
    _check(lib().gf_stash_forward(ctypes.byref(desc), _ptr(x), _ptr(stash), _stream(stream)),
           "gf_stash_forward")


def gf_act_stash_forward(desc: gf_conv_desc, act: int, z, x, stash, stream=None) -> None:
    """x <- act(z) and stash <- patch sums of x, in one pass over z (x may be z)."""
    _check(lib().gf_act_stash_forward(ctypes.byref(desc), int(act), _ptr(z), _ptr(x), _ptr(stash), _stream(stream)),
           "gf_act_stash_forward")


def gf_backward(desc: gf_conv_desc, g_y, stash, W, g_W, g_X, workspace, workspace_bytes=None,
                stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(lib().gf_backward(ctypes.byref(desc), _ptr(g_y), _ptr(stash), _ptr(W), _ptr(g_W), _ptr(g_X),
                             _ptr(workspace), ctypes.c_size_t(workspace_bytes), _stream(stream)),
           "gf_backward")


def gf_backward_int8_workspace_bytes(desc: gf_conv_desc) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().gf_backward_int8_workspace_bytes(ctypes.byref(desc), ctypes.byref(out)), "gf_backward_int8_workspace_bytes")
    return int(out.value)


def gf_backward_int8(desc: gf_conv_desc, g_y, stash, W, g_W, g_X, workspace, workspace_bytes=None, stream=None) -> None:
    """gf_backward with the operands of the two reduced contractions quantised to INT8."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(lib().gf_backward_int8(ctypes.byref(desc), _ptr(g_y), _ptr(stash), _ptr(W), _ptr(g_W), _ptr(g_X), _ptr(workspace),
                                  ctypes.c_size_t(workspace_bytes), _stream(stream)), "gf_backward_int8")


GF_STATIC_SCRATCH_BYTES = 8 << 20


def gf_backward_static_scratch(desc: gf_conv_desc, g_y, stash, W, g_W, g_X, stream=None) -> None:
    """gf_backward without a workspace argument: the scratch is an array built into the
    library (GF_STATIC_SCRATCH_BYTES), for callers that may not allocate device memory.
    Calls must not overlap on the GPU; larger layers raise GfError(GF_ERR_WORKSPACE)."""
    _check(lib().gf_backward_static_scratch(ctypes.byref(desc), _ptr(g_y), _ptr(stash), _ptr(W), _ptr(g_W),
                                            _ptr(g_X), _stream(stream)), "gf_backward_static_scratch")


def gf_last_async_status(workspace, stream=None) -> int:
    return int(lib().gf_last_async_status(_ptr(workspace), _stream(stream)))


def gf_host_step_arena_bytes(desc: gf_conv_desc) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().gf_host_step_arena_bytes(ctypes.byref(desc), ctypes.byref(out)), "gf_host_step_arena_bytes")
    return int(out.value)


def gf_layer_step_host(desc: gf_conv_desc, h_x, h_gy, h_W, h_gW, h_gX, arena, arena_bytes=None,
                       stream=None) -> None:
    if arena_bytes is None:
        arena_bytes = arena.numel() * arena.element_size()
    _check(lib().gf_layer_step_host(ctypes.byref(desc), _ptr(h_x), _ptr(h_gy), _ptr(h_W), _ptr(h_gW),
                                    _ptr(h_gX), _ptr(arena), ctypes.c_size_t(arena_bytes), _stream(stream)),
           "gf_layer_step_host")


def gf_set_dense_path(path: int) -> None:
    """GF_PATH_AUTO (the library's choice per layer), GF_PATH_FUSED or GF_PATH_SPLIT, process-wide."""
    _check(lib().gf_set_dense_path(int(path)), "gf_set_dense_path")


def _gf_dtype(t: torch.Tensor) -> int:
    return {torch.float32: GF_F32, torch.bfloat16: GF_BF16}[t.dtype]


def gf_snr_terms(ref: torch.Tensor, approx: torch.Tensor, energies: torch.Tensor, stream=None) -> None:
    """energies (2 doubles on the device) <- sum ref^2, sum (ref - approx)^2."""
    assert ref.dtype == approx.dtype and ref.numel() == approx.numel() and energies.dtype == torch.float64
    _check(lib().gf_snr_terms(_ptr(ref), _ptr(approx), ctypes.c_int64(ref.numel()), _gf_dtype(ref), _ptr(energies),
                              _stream(stream)), "gf_snr_terms")


def gf_filter_snr_terms(g: torch.Tensor, r: int, energies: torch.Tensor, stream=None) -> None:
    """The SNR terms of the gradient filter with patch size r on g [..., H, W]."""
    assert energies.dtype == torch.float64 and g.dim() >= 2
    H, W = int(g.shape[-2]), int(g.shape[-1])
    _check(lib().gf_filter_snr_terms(_ptr(g), ctypes.c_int64(g.numel() // (H * W)), H, W, int(r), _gf_dtype(g),
                                     _ptr(energies), _stream(stream)), "gf_filter_snr_terms")


def gf_dcac_ratio(W: torch.Tensor, ratio: torch.Tensor, dft: tuple[int, int] = (0, 0), stream=None) -> None:
    """ratio [C_out, C_ig] (fp32, device) <- DC / largest AC energy of every kernel of W [C_out, C_ig, KH, KW]."""
    C_out, C_ig, KH, KW = (int(v) for v in W.shape)
    assert ratio.dtype == torch.float32 and ratio.numel() == C_out * C_ig
    _check(lib().gf_dcac_ratio(_ptr(W), C_out, C_ig, KH, KW, int(dft[0]), int(dft[1]), _gf_dtype(W), _ptr(ratio),
                               _stream(stream)), "gf_dcac_ratio")


# ---- operators of a fine-tuning step (gf_train.h) --------------------------------------------

def _dt(dtype) -> int:
    """gf_dtype of a torch dtype (an int is passed through)."""
    if isinstance(dtype, torch.dtype):
        try:
            return {torch.float32: GF_F32, torch.bfloat16: GF_BF16}[dtype]
        except KeyError:
            raise TypeError(f"float32 or bfloat16 expected, got {dtype}") from None
    return int(dtype)


def make_norm_desc(N, C, H=1, W=1, *, dtype=GF_F32, param_dtype=GF_F32, layout=GF_NHWC, eps=1e-5) -> gf_norm_desc:
    return gf_norm_desc(N, C, H, W, _dt(dtype), _dt(param_dtype), layout, eps)


def make_ns_desc(batch, rows, cols, *, in_dtype=GF_F32, out_dtype=GF_F32, precision=GF_NS_F32, steps=5, eps=1e-7) -> gf_ns_desc:
    return gf_ns_desc(batch, rows, cols, _dt(in_dtype), _dt(out_dtype), precision, steps, eps)


def make_muon_desc(count, rows, cols, taps=1, *, grad_dtype=GF_F32, weight_dtype=GF_F32, precision=GF_NS_F32, steps=5,
                   nesterov=True, eps=1e-7, momentum=0.95, lr=1e-3, weight_decay=0.0, scale=1.0) -> gf_muon_desc:
    return gf_muon_desc(count, rows, cols, taps, _dt(grad_dtype), _dt(weight_dtype), precision, steps, int(nesterov), eps,
                        momentum, lr, weight_decay, scale)


def _size(fn, desc, where: str) -> int:
    out = ctypes.c_size_t(0)
    _check(fn(ctypes.byref(desc), ctypes.byref(out)), where)
    return int(out.value)


def _nbytes(workspace) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def _addr(t):
    """Device address of a dense tensor, as ctypes takes it for a pointer (None: NULL).  These calls are short beside
    their marshalling, so that it is kept short: no intermediate objects."""
    if t is None:
        return None
    if not t.is_contiguous() and not (t.dim() == 4 and t.is_contiguous(memory_format=torch.channels_last)):
        raise ValueError("tensors passed to the gf_* calls must be dense")
    return t.data_ptr()


def _raw_stream(stream):
    if stream is None:      # what torch.cuda.current_stream().cuda_stream gives, without the stream object
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


def gf_layer_norm_forward(desc: gf_norm_desc, x, gamma, beta, y, mean=None, rstd=None, stream=None) -> None:
    """y <- (x - mean) rstd gamma + beta over the channels; mean and rstd (fp32, one per pixel) for the backward pass."""
    _check(lib().gf_layer_norm_forward(ctypes.byref(desc), _addr(x), _addr(gamma), _addr(beta), _addr(y), _addr(mean), _addr(rstd),
                                       _raw_stream(stream)), "gf_layer_norm_forward")


def gf_layer_norm_backward_workspace_bytes(desc: gf_norm_desc) -> int:
    return _size(lib().gf_layer_norm_backward_workspace_bytes, desc, "gf_layer_norm_backward_workspace_bytes")


def gf_layer_norm_backward(desc: gf_norm_desc, g_y, x, gamma, mean, rstd, g_x, g_gamma, g_beta, workspace,
                           workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = _nbytes(workspace)
    _check(lib().gf_layer_norm_backward(ctypes.byref(desc), _addr(g_y), _addr(x), _addr(gamma), _addr(mean), _addr(rstd), _addr(g_x),
                                        _addr(g_gamma), _addr(g_beta), _addr(workspace), workspace_bytes, _raw_stream(stream)),
           "gf_layer_norm_backward")


def _coeffs(coeffs, steps: int):
    """(a, b, c) per step as a host array, or NULL for the default ones."""
    if coeffs is None:
        return None
    flat = [float(v) for abc in coeffs for v in abc]
    if len(flat) != 3 * steps:
        raise ValueError(f"{steps} triples of coefficients expected, got {len(flat)} values")
    return (ctypes.c_float * len(flat))(*flat)


def gf_newton_schulz_workspace_bytes(desc: gf_ns_desc) -> int:
    return _size(lib().gf_newton_schulz_workspace_bytes, desc, "gf_newton_schulz_workspace_bytes")


def gf_newton_schulz(desc: gf_ns_desc, G, O, workspace, workspace_bytes=None, coeffs=None, stream=None) -> None:
    """O <- the Newton-Schulz iterates of the matrices G [batch, rows, cols]; coeffs: (a, b, c) for each step."""
    if workspace_bytes is None:
        workspace_bytes = _nbytes(workspace)
    _check(lib().gf_newton_schulz(ctypes.byref(desc), _addr(G), _addr(O), _addr(workspace), workspace_bytes,
                                  _coeffs(coeffs, desc.steps), _raw_stream(stream)), "gf_newton_schulz")


def gf_muon_workspace_bytes(desc: gf_muon_desc) -> int:
    return _size(lib().gf_muon_workspace_bytes, desc, "gf_muon_workspace_bytes")


def _ptrs(tensors, count: int):
    if len(tensors) != count:
        raise ValueError(f"{count} tensors expected, got {len(tensors)}")
    return (ctypes.c_void_p * count)(*map(_addr, tensors))


def gf_muon_step(desc: gf_muon_desc, grads, momenta, weights, momenta_out, weights_out, workspace, workspace_bytes=None,
                 coeffs=None, stream=None) -> None:
    """One Muon update of `count` layers of one shape (lists of tensors); the outputs may be the inputs."""
    if workspace_bytes is None:
        workspace_bytes = _nbytes(workspace)
    n = desc.count
    _check(lib().gf_muon_step(ctypes.byref(desc), _ptrs(grads, n), _ptrs(momenta, n), _ptrs(weights, n), _ptrs(momenta_out, n),
                              _ptrs(weights_out, n), _addr(workspace), workspace_bytes, _coeffs(coeffs, desc.steps),
                              _raw_stream(stream)), "gf_muon_step")


# ---- operators of a residual block with frozen layers (gf_block.h) ---------------------------------

def make_dropout_desc(count, *, dtype=GF_F32, out_dtype=None, p) -> gf_dropout_desc:
    return gf_dropout_desc(count, _dt(dtype), _dt(dtype if out_dtype is None else out_dtype), p)


def make_rms_desc(rows, cols, *, dtype=GF_F32, residual_dtype=None, param_dtype=GF_F32, eps=1e-5, p=0.0) -> gf_rms_desc:
    return gf_rms_desc(rows, cols, _dt(dtype), _dt(dtype if residual_dtype is None else residual_dtype), _dt(param_dtype), eps, p)


def make_fp8_desc(rows, cols, *, dtype=GF_F32) -> gf_fp8_desc:
    return gf_fp8_desc(rows, cols, _dt(dtype))


def make_fp8_matmul_desc(M, N, K, *, transposed=False, out_dtype=GF_BF16, bias_dtype=GF_F32) -> gf_fp8_matmul_desc:
    return gf_fp8_matmul_desc(M, N, K, int(transposed), _dt(out_dtype), _dt(bias_dtype))


def fp8_pitch(cols: int) -> int:
    """Bytes between the rows of an 8-bit matrix."""
    return (cols + 15) // 16 * 16


def fp8_scale_pitch(rows: int) -> int:
    """Places between the scales of one group of 128 columns and the next."""
    return (rows + 3) // 4 * 4


def gf_dropout_forward(desc: gf_dropout_desc, x, residual, seed, y, stream=None) -> None:
    """y <- residual + dropout(x); the mask is a function of seed (two 64-bit words on the device) and the element's index."""
    _check(lib().gf_dropout_forward(ctypes.byref(desc), _addr(x), _addr(residual), _addr(seed), _addr(y), _raw_stream(stream)),
           "gf_dropout_forward")


def gf_dropout_backward(desc: gf_dropout_desc, g_y, seed, g_x, stream=None) -> None:
    _check(lib().gf_dropout_backward(ctypes.byref(desc), _addr(g_y), _addr(seed), _addr(g_x), _raw_stream(stream)),
           "gf_dropout_backward")


def gf_rms_norm_forward(desc: gf_rms_desc, x, residual, seed, gamma, h, y, rstd=None, stream=None) -> None:
    """h <- residual + dropout(x), y <- h rstd gamma (h None: no residual and nothing dropped, h is x)."""
    _check(lib().gf_rms_norm_forward(ctypes.byref(desc), _addr(x), _addr(residual), _addr(seed), _addr(gamma), _addr(h), _addr(y),
                                     _addr(rstd), _raw_stream(stream)), "gf_rms_norm_forward")


def gf_rms_norm_forward_fp8(desc: gf_rms_desc, x, residual, seed, gamma, h, codes, scales, rstd=None, stream=None) -> None:
    """As gf_rms_norm_forward, with y as codes [rows, fp8_pitch(cols)] and scales [ceil(cols / 128), fp8_scale_pitch(rows)]."""
    _check(lib().gf_rms_norm_forward_fp8(ctypes.byref(desc), _addr(x), _addr(residual), _addr(seed), _addr(gamma), _addr(h),
                                         _addr(codes), _addr(scales), _addr(rstd), _raw_stream(stream)), "gf_rms_norm_forward_fp8")


def gf_rms_norm_backward_workspace_bytes(desc: gf_rms_desc) -> int:
    return _size(lib().gf_rms_norm_backward_workspace_bytes, desc, "gf_rms_norm_backward_workspace_bytes")


def gf_rms_norm_backward(desc: gf_rms_desc, g_y, g_h, h, rstd, gamma, seed, g_residual, g_x, g_gamma, workspace,
                         workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = _nbytes(workspace)
    _check(lib().gf_rms_norm_backward(ctypes.byref(desc), _addr(g_y), _addr(g_h), _addr(h), _addr(rstd), _addr(gamma), _addr(seed),
                                      _addr(g_residual), _addr(g_x), _addr(g_gamma), _addr(workspace), workspace_bytes,
                                      _raw_stream(stream)), "gf_rms_norm_backward")


def gf_fp8_quantize_rows(desc: gf_fp8_desc, x, codes, scales, stream=None) -> None:
    """codes [rows, fp8_pitch(cols)], scales [ceil(cols / 128), fp8_scale_pitch(rows)] <- x [rows, cols]."""
    _check(lib().gf_fp8_quantize_rows(ctypes.byref(desc), _addr(x), _addr(codes), _addr(scales), _raw_stream(stream)),
           "gf_fp8_quantize_rows")


def gf_fp8_quantize_blocks(desc: gf_fp8_desc, w, codes, scales, stream=None) -> None:
    """codes [rows, fp8_pitch(cols)], scales [ceil(rows / 128), ceil(cols / 128)] <- w [rows, cols]."""
    _check(lib().gf_fp8_quantize_blocks(ctypes.byref(desc), _addr(w), _addr(codes), _addr(scales), _raw_stream(stream)),
           "gf_fp8_quantize_blocks")


def gf_fp8_matmul(desc: gf_fp8_matmul_desc, a, a_scales, w, w_scales, bias, out, stream=None) -> None:
    """out [M, N] <- A W^T + bias, or with desc.transposed out [M, K] <- A W + bias."""
    _check(lib().gf_fp8_matmul(ctypes.byref(desc), _addr(a), _addr(a_scales), _addr(w), _addr(w_scales), _addr(bias), _addr(out),
                               _raw_stream(stream)), "gf_fp8_matmul")


def gf_selftest_fp8_form(desc: gf_fp8_matmul_desc) -> int:
    """Which kernel gf_fp8_matmul launches (include/gf_bench.h)."""
    return lib().gf_selftest_fp8_form(ctypes.byref(desc))


def gf_selftest_bounded_wait(workspace, limit_cycles: int, stream=None) -> None:
    """Launches a block whose bounded wait must expire; it records that in the workspace's error word."""
    _check(lib().gf_selftest_bounded_wait(_ptr(workspace), ctypes.c_int64(int(limit_cycles)), _stream(stream)),
           "gf_selftest_bounded_wait")


def gf_selftest_warp_wait(result, limit_cycles: int, stream=None) -> None:
    """A warp whose lanes wait with different limits; result (32 words on the device) <- what each lane went on with."""
    _check(lib().gf_selftest_warp_wait(_ptr(result), ctypes.c_int64(int(limit_cycles)), _stream(stream)), "gf_selftest_warp_wait")


def gf_selftest_end_of_turn(turn: int, turns: int, ok: bool, met: bool) -> bool:
    """Whether a role of the Newton-Schulz kernel goes on after turn `turn` of `turns` (evaluated on the host)."""
    return bool(lib().gf_selftest_end_of_turn(int(turn), int(turns), int(ok), int(met)))


def gf_kernel_launch_count() -> int:
    return int(lib().gf_kernel_launch_count())


def gf_kernel_id_count() -> int:
    return int(lib().gf_kernel_id_count())


def gf_kernel_name(kernel_id: int) -> str | None:
    n = lib().gf_kernel_name(int(kernel_id))
    return n.decode() if n else None


def kernel_id(name: str) -> int:
    for k in range(gf_kernel_id_count()):
        if gf_kernel_name(k) == name:
            return k
    raise KeyError(name)


def gf_profile_configure(mode: int, kernel_id: int = -1) -> None:
    _check(lib().gf_profile_configure(int(mode), int(kernel_id)), "gf_profile_configure")


def gf_profile_read() -> dict[str, tuple[int, float]]:
    """{kernel name: (timed launches, total ms)} since the last read."""
    n = gf_kernel_id_count()
    buf = (gf_kernel_time * n)()
    got = lib().gf_profile_read(buf, n)
    if got < 0:
        raise GfError(GF_ERR_CUDA, "gf_profile_read")
    return {gf_kernel_name(buf[i].kernel_id): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(got)}


# ---- conveniences that only allocate ---------------------------------------------

@dataclass
class LayerBuffers:
    desc: gf_conv_desc
    stash: torch.Tensor
    g_W: torch.Tensor
    g_X: torch.Tensor
    workspace: torch.Tensor


def alloc_layer(desc: gf_conv_desc, device="cuda") -> LayerBuffers:
    dt = torch.float32 if desc.dtype == GF_F32 else torch.bfloat16
    stash = torch.empty(gf_stash_dims(desc), dtype=dt, device=device)
    g_W = torch.empty((desc.C_out, desc.C_in // desc.groups, desc.KH, desc.KW), dtype=torch.float32,
                      device=device)
    g_X = torch.empty((desc.N, desc.C_in, desc.H, desc.W), dtype=dt, device=device)
    ws = torch.empty(gf_backward_workspace_bytes(desc), dtype=torch.uint8, device=device)
    return LayerBuffers(desc, stash, g_W, g_X, ws)
