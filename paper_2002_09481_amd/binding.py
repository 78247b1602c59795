"""ctypes binding of libaxconv.so: the same entry points as include/axconv.h and
include/axconv_probe.h.

Only argument marshalling happens here.  Tensors are torch CUDA tensors (torch provides
device memory and the stream); every step of the layer runs in the HIP kernels.  There is
no fallback: a missing library raises at first use.

The library itself keeps no options: tuning overrides travel with each call as an ax_tune_t.
ax_set_option / ax_get_option below only keep this module's default for that argument (the
tests use them to force every kernel path); calls made while a default is set go through the
entry points that accept a tune (ax_conv2d_ex, ax_conv2d_f32_ex, the layer handles).
"""

from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaxconv.so")

_lib = None


class AxError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("axconv error %d: %s" % (code, text))
        self.code = code


class ax_quant_t(ctypes.Structure):
    _fields_ = [
        ("x_scale", ctypes.c_float),
        ("x_zp", ctypes.c_int32),
        ("w_scale", ctypes.c_float),
        ("w_zp", ctypes.c_int32),
        ("pad_code", ctypes.c_int32),
    ]


EXPORTS = [  # include/axconv.h
    "ax_conv2d", "ax_conv2d_workspace_bytes", "ax_dense", "ax_dense_workspace_bytes", "ax_strerror",
    "ax_conv2d_transpose", "ax_conv2d_transpose_workspace_bytes", "ax_version", "ax_range_f32", "ax_range_workspace_bytes", "ax_quantize_f32", "ax_conv2d_f32",
    "ax_conv2d_f32_workspace_bytes", "ax_dense_f32", "ax_dense_f32_workspace_bytes", "ax_conv2d_ex",
    "ax_conv2d_ex_workspace_bytes", "ax_conv2d_multi_lut", "ax_conv2d_multi_lut_workspace_bytes", "ax_conv2d_f32_ex",
    "ax_conv2d_f32_ex_workspace_bytes", "ax_layer_create", "ax_layer_destroy", "ax_layer_prepared_bytes",
    "ax_layer_workspace_bytes", "ax_layer_prepare", "ax_layer_run", "ax_layer_plan", "ax_layer_plan_paths", "ax_layer_run_static",
    "ax_static_scratch_bytes", "ax_conv2d_backward", "ax_conv2d_backward_workspace_bytes",
    "ax_rmsnorm", "ax_rmsnorm_q8", "ax_rmsnorm_backward", "ax_rmsnorm_backward_workspace_bytes",
    "ax_matmul", "ax_matmul_workspace_bytes", "ax_matmul_q8", "ax_matmul_q8_workspace_bytes",
    "ax_matmul_backward", "ax_matmul_backward_workspace_bytes", "ax_gated", "ax_gated_workspace_bytes",
    "ax_gated_q8", "ax_gated_q8_workspace_bytes", "ax_gated_backward", "ax_gated_backward_workspace_bytes",
    "ax_adamw", "ax_adamw_states",
    "ax_route", "ax_route_workspace_bytes", "ax_route_backward", "ax_combine", "ax_combine_backward",
    "ax_matmul_experts", "ax_matmul_experts_workspace_bytes", "ax_gated_experts", "ax_gated_experts_workspace_bytes",
    "ax_matmul_experts_backward", "ax_matmul_experts_backward_workspace_bytes",
    "ax_gated_experts_backward", "ax_gated_experts_backward_workspace_bytes",
    "ax_quantize_q4", "ax_pack_q4", "ax_q4_values", "ax_q4_codes_bytes", "ax_q4_scales_bytes",
    "ax_matmul_q4", "ax_matmul_q4_workspace_bytes", "ax_gated_q4", "ax_gated_q4_workspace_bytes",
]
PROBE_EXPORTS = [  # include/axconv_probe.h
    "ax_probe_lds_gather", "ax_probe_copy", "ax_probe_mac", "ax_probe_layer_kernel_ms",
    "ax_probe_layer_route", "ax_probe_product_plan", "ax_probe_experts_plan", "ax_probe_q4_plan",
]


AX_PAD_DEFAULT = -(1 << 31)


class ax_tune_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("variant", "split_k", "tile", "row_tiles", "share_order", "combine", "tables")]


class ax_conv_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "N", "H", "W", "Cin", "KH", "KW", "Cout", "stride_h", "stride_w", "pad_h", "pad_w", "dilation_h", "dilation_w",
        "depthwise", "signed_codes", "groups")]


AX_F32, AX_BF16 = 0, 1
AX_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
AX_STATE_BLOCK = 256


class ax_norm_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "cols", "x_ld", "residual_ld", "sum_ld", "y_ld")] + [
        ("dtype", ctypes.c_int32), ("w_dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("normalize", ctypes.c_int32)]


class ax_matmul_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("M", "N", "K", "x_ld", "w_ld", "residual_ld", "y_ld")] + [
        (n, ctypes.c_int32) for n in ("dtype", "out_dtype", "act", "w_transposed", "unaligned")]


class ax_adamw_tensor_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("p", "g", "m", "v", "m_scale", "v_scale", "copy")] + [("n", ctypes.c_int64)]


class ax_adamw_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [
        ("step", ctypes.c_int64), ("grad_scale", ctypes.c_void_p)] + [
        (n, ctypes.c_int32) for n in ("p_dtype", "g_dtype", "state_bits", "reserved")]


class ax_route_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("tokens", "ld")] + [
        (n, ctypes.c_int32) for n in ("experts", "k", "dtype", "normalize")]


class ax_experts_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "x_rows", "N", "K", "x_ld", "w_ld", "y_ld", "gx_ld")] + [
        (n, ctypes.c_int32) for n in ("experts", "dtype", "act", "w_transposed", "indexed", "unaligned")]


class ax_combine_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("tokens", "h_rows", "cols", "h_ld", "residual_ld", "y_ld", "gh_ld")] + [
        (n, ctypes.c_int32) for n in ("k", "dtype")]


class ax_q4_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "x_rows", "N", "K", "x_ld", "residual_ld", "y_ld")] + [
        (n, ctypes.c_int32) for n in ("experts", "group", "dtype", "act", "indexed", "unaligned")]


def lib():
    """Load libaxconv.so (built beforehand by paper_2002_09481_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libaxconv.so is not built: run `python -m paper_2002_09481_amd.build` "
                           "(or __graft_entry__.build()) first; there is no fallback path")
    L = ctypes.CDLL(LIB_PATH)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    L.ax_conv2d.argtypes = [vp, ci, ci, ci, ci, vp, ci, ci, ci, vp, ci, ci, ci, ci,
                            ctypes.POINTER(ax_quant_t), vp, vp, vp, sz, vp]
    L.ax_conv2d.restype = ci
    L.ax_conv2d_workspace_bytes.argtypes = [ci] * 11
    L.ax_conv2d_workspace_bytes.restype = sz
    L.ax_dense.argtypes = [vp, ci, ci, vp, ci, vp, ctypes.POINTER(ax_quant_t), vp, vp, vp, sz, vp]
    L.ax_dense.restype = ci
    L.ax_dense_workspace_bytes.argtypes = [ci, ci, ci]
    L.ax_dense_workspace_bytes.restype = sz
    L.ax_strerror.argtypes = [ci]
    L.ax_strerror.restype = ctypes.c_char_p
    L.ax_version.argtypes = []
    L.ax_version.restype = ci
    dp = ctypes.POINTER(ctypes.c_double)
    L.ax_probe_lds_gather.argtypes = [ci, ci, ci, ci, ci, dp, dp, dp, ctypes.POINTER(ci), vp]
    L.ax_probe_lds_gather.restype = ci
    L.ax_probe_mac.argtypes = [ci, ci, ci, ci, dp, dp, vp]
    L.ax_probe_mac.restype = ci
    ip = ctypes.POINTER(ci)
    tp = ctypes.POINTER(ax_tune_t)
    descp = ctypes.POINTER(ax_conv_desc_t)
    L.ax_layer_create.argtypes = [descp, ci, ctypes.POINTER(ax_quant_t), tp, ctypes.POINTER(vp)]
    L.ax_layer_create.restype = ci
    L.ax_layer_destroy.argtypes = [vp]
    L.ax_layer_destroy.restype = None
    L.ax_layer_prepared_bytes.argtypes = [vp]
    L.ax_layer_prepared_bytes.restype = sz
    L.ax_layer_workspace_bytes.argtypes = [vp]
    L.ax_layer_workspace_bytes.restype = sz
    L.ax_layer_prepare.argtypes = [vp, vp, vp, vp, sz, vp]
    L.ax_layer_prepare.restype = ci
    L.ax_layer_run.argtypes = [vp, vp, vp, vp, vp, sz, vp]
    L.ax_layer_run.restype = ci
    L.ax_layer_plan.argtypes = [vp, ip, ip, ip, ip]
    L.ax_layer_plan.restype = ci
    L.ax_layer_plan_paths.argtypes = [vp, ip, ip]
    L.ax_layer_plan_paths.restype = ci
    L.ax_layer_run_static.argtypes = [vp, vp, vp, vp, vp]
    L.ax_layer_run_static.restype = ci
    L.ax_static_scratch_bytes.argtypes = []
    L.ax_static_scratch_bytes.restype = sz
    L.ax_conv2d_backward.argtypes = [descp, ctypes.POINTER(ax_quant_t), vp, vp, vp, vp, vp, vp, sz, vp]
    L.ax_conv2d_backward.restype = ci
    L.ax_conv2d_backward_workspace_bytes.argtypes = [descp]
    L.ax_conv2d_backward_workspace_bytes.restype = sz
    L.ax_probe_layer_kernel_ms.argtypes = [vp, vp, vp, vp, vp, sz, ci, ctypes.POINTER(ctypes.c_float), vp]
    L.ax_probe_layer_kernel_ms.restype = ci
    L.ax_probe_layer_route.argtypes = [vp] + [ip] * 6
    L.ax_probe_layer_route.restype = ci
    L.ax_probe_copy.argtypes = [vp, vp, sz, vp]
    L.ax_probe_copy.restype = ci
    L.ax_conv2d_multi_lut.argtypes = [vp, ci, ci, ci, ci, vp, ci, ci, ci, vp, ci, ci, ci, ci, ci,
                                      ctypes.POINTER(ax_quant_t), vp, vp, vp, sz, vp]
    L.ax_conv2d_multi_lut.restype = ci
    L.ax_conv2d_multi_lut_workspace_bytes.argtypes = [ci] * 12
    L.ax_conv2d_multi_lut_workspace_bytes.restype = sz
    L.ax_conv2d_f32_ex.argtypes = [descp, tp, vp, vp, vp, vp, vp, ci, ci, vp, vp, vp, sz, vp]
    L.ax_conv2d_f32_ex.restype = ci
    L.ax_conv2d_f32_ex_workspace_bytes.argtypes = [descp, tp]
    L.ax_conv2d_f32_ex_workspace_bytes.restype = sz
    L.ax_conv2d_ex.argtypes = [descp, tp, vp, vp, vp, ctypes.POINTER(ax_quant_t), vp, vp, vp, sz, vp]
    L.ax_conv2d_ex.restype = ci
    L.ax_conv2d_ex_workspace_bytes.argtypes = [descp, tp]
    L.ax_conv2d_ex_workspace_bytes.restype = sz
    L.ax_conv2d_transpose.argtypes = [descp, tp, vp, vp, vp, ctypes.POINTER(ax_quant_t), vp, vp, vp, sz, vp]
    L.ax_conv2d_transpose_workspace_bytes.argtypes = [descp, tp]
    L.ax_conv2d_transpose_workspace_bytes.restype = sz
    L.ax_range_f32.argtypes = [vp, sz, ci, vp, vp, sz, vp]
    L.ax_range_f32.restype = ci
    L.ax_range_workspace_bytes.argtypes = [sz]
    L.ax_range_workspace_bytes.restype = sz
    L.ax_quantize_f32.argtypes = [vp, sz, vp, ci, ci, vp, vp, vp]
    L.ax_quantize_f32.restype = ci
    L.ax_conv2d_f32.argtypes = [vp, ci, ci, ci, ci, vp, ci, ci, ci, vp, ci, ci, ci, ci, vp, vp, ci, ci, vp, vp, vp,
                                sz, vp]
    L.ax_conv2d_f32.restype = ci
    L.ax_conv2d_f32_workspace_bytes.argtypes = [ci] * 11
    L.ax_conv2d_f32_workspace_bytes.restype = sz
    L.ax_dense_f32.argtypes = [vp, ci, ci, vp, ci, vp, vp, vp, ci, ci, vp, vp, vp, sz, vp]
    L.ax_dense_f32.restype = ci
    L.ax_dense_f32_workspace_bytes.argtypes = [ci, ci, ci]
    L.ax_dense_f32_workspace_bytes.restype = sz
    nd, md = ctypes.POINTER(ax_norm_desc_t), ctypes.POINTER(ax_matmul_desc_t)
    for name, args in (
            ("ax_rmsnorm", [nd] + [vp] * 7), ("ax_rmsnorm_q8", [nd] + [vp] * 8),
            ("ax_rmsnorm_backward", [nd] + [vp] * 8 + [sz, vp]),
            ("ax_matmul", [md] + [vp] * 7 + [sz, vp]), ("ax_matmul_q8", [md] + [vp] * 8 + [sz, vp]),
            ("ax_matmul_backward", [md] + [vp] * 8 + [sz, vp]),
            ("ax_gated", [md] + [vp] * 7 + [sz, vp]), ("ax_gated_q8", [md] + [vp] * 8 + [sz, vp]),
            ("ax_gated_backward", [md] + [vp] * 10 + [sz, vp]),
            ("ax_adamw", [ctypes.POINTER(ax_adamw_desc_t), ctypes.POINTER(ax_adamw_tensor_t), ci, vp]),
            ("ax_adamw_states", [ctypes.POINTER(ax_adamw_tensor_t), ci, ctypes.POINTER(vp), ctypes.POINTER(vp), vp])):
        getattr(L, name).argtypes, getattr(L, name).restype = args, ci
    L.ax_probe_product_plan.argtypes, L.ax_probe_product_plan.restype = [md, ci] + [ip] * 4, ci
    L.ax_probe_experts_plan.argtypes, L.ax_probe_experts_plan.restype = [ctypes.POINTER(ax_experts_desc_t), ci] + [ip] * 5, ci
    L.ax_probe_q4_plan.argtypes, L.ax_probe_q4_plan.restype = [ctypes.POINTER(ax_q4_desc_t), ci] + [ip] * 4, ci
    L.ax_rmsnorm_backward_workspace_bytes.argtypes, L.ax_rmsnorm_backward_workspace_bytes.restype = [nd], sz
    for name in ("ax_matmul", "ax_matmul_q8", "ax_matmul_backward", "ax_gated", "ax_gated_q8", "ax_gated_backward"):
        f = getattr(L, name + "_workspace_bytes")
        f.argtypes, f.restype = [md], sz
    rd, ed, cd, qd = (ctypes.POINTER(t) for t in (ax_route_desc_t, ax_experts_desc_t, ax_combine_desc_t, ax_q4_desc_t))
    i64, i32 = ctypes.c_int64, ctypes.c_int32
    for name, args, workspace in (
            ("ax_route", [rd] + [vp] * 7 + [sz, vp], rd), ("ax_route_backward", [rd] + [vp] * 5 + [i64, vp], None),
            ("ax_matmul_experts", [ed] + [vp] * 7 + [sz, vp], ed), ("ax_gated_experts", [ed] + [vp] * 9 + [sz, vp], ed),
            ("ax_matmul_experts_backward", [ed] + [vp] * 9 + [sz, vp], ed),
            ("ax_gated_experts_backward", [ed] + [vp] * 12 + [sz, vp], ed),
            ("ax_combine", [cd] + [vp] * 6, None), ("ax_combine_backward", [cd] + [vp] * 7, None),
            ("ax_quantize_q4", [vp, i32] + [i64] * 4 + [i32] + [vp] * 3, None),
            ("ax_pack_q4", [vp] * 2 + [i64] * 3 + [i32] + [vp] * 3, None), ("ax_q4_values", [vp] * 2 + [i64] * 3 + [i32] + [vp] * 2, None),
            ("ax_matmul_q4", [qd] + [vp] * 9 + [sz, vp], qd), ("ax_gated_q4", [qd] + [vp] * 9 + [sz, vp], qd)):
        getattr(L, name).argtypes, getattr(L, name).restype = args, ci
        if workspace is not None:
            f = getattr(L, name + "_workspace_bytes")
            f.argtypes, f.restype = [workspace], sz
    L.ax_q4_codes_bytes.argtypes, L.ax_q4_codes_bytes.restype = [i64] * 3, sz
    L.ax_q4_scales_bytes.argtypes, L.ax_q4_scales_bytes.restype = [i64] * 3 + [i32], sz
    _lib = L
    return L


def _check(rc: int):
    if rc != 0:
        raise AxError(rc, lib().ax_strerror(rc).decode())


def ax_static_scratch_bytes() -> int:
    return int(lib().ax_static_scratch_bytes())


def ax_strerror(code: int) -> str:
    return lib().ax_strerror(code).decode()


def ax_version() -> int:
    return int(lib().ax_version())


_TUNE_FIELDS = ("variant", "split_k", "tile", "row_tiles", "share_order", "combine", "tables")
_tune = {n: 0 for n in _TUNE_FIELDS}  # this module's default ax_tune_t (all zero = automatic)


def _tune_arg(tune=None):
    """ctypes argument for a `const ax_tune_t*` parameter: NULL when everything is automatic."""
    if tune is None:
        if not any(_tune.values()):
            return None
        tune = _tune
    t = tune
    if not any(t.get(n, 0) for n in _TUNE_FIELDS):
        return None
    return ctypes.byref(ax_tune_t(*[int(t.get(n, 0)) for n in _TUNE_FIELDS]))


def ax_set_option(name: str, value: int) -> None:
    """Set one field of the module's default tune; the library checks the value's range."""
    if name not in _tune:
        raise AxError(-8, lib().ax_strerror(-8).decode())
    trial = dict(_tune)
    trial[name] = int(value)
    if not -(1 << 31) <= trial[name] < (1 << 31):
        raise AxError(-8, lib().ax_strerror(-8).decode())
    desc = ax_conv_desc_t(1, 1, 1, 1, 1, 1, 1, 1, 1, 0, 0, 1, 1, 0, 0)
    q = ax_quant_t(1.0, 0, 1.0, 0, -1)
    h = ctypes.c_void_p()
    _check(lib().ax_layer_create(ctypes.byref(desc), 1, ctypes.byref(q), _tune_arg(trial), ctypes.byref(h)))
    lib().ax_layer_destroy(h)
    _tune[name] = trial[name]


def ax_get_option(name: str) -> int:
    if name not in _tune:
        raise AxError(-8, lib().ax_strerror(-8).decode())
    return _tune[name]


def ax_conv2d_plan(x_shape, w_shape, stride=1, pad=0, num_luts=1) -> dict:
    """What a layer of this geometry runs under the module's default tune (host arithmetic)."""
    N, H, W, Cin = [int(v) for v in x_shape]
    KH, KW, _, Cout = [int(v) for v in w_shape]
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    desc = ax_conv_desc_t(N, H, W, Cin, KH, KW, Cout, sh, sw, ph, pw, 1, 1, 0, 0)
    with AxLayer(desc, ax_quant_t(1.0, 0, 1.0, 0, -1), num_luts) as layer:
        return layer.plan()


def _quant(q) -> ax_quant_t:
    pad_code = AX_PAD_DEFAULT if q.pad_code is None else int(q.pad_code)
    return ax_quant_t(float(q.x_scale), int(q.x_zp), float(q.w_scale), int(q.w_zp), pad_code)


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def _pair(v) -> Tuple[int, int]:
    return (int(v), int(v)) if isinstance(v, int) else (int(v[0]), int(v[1]))


def _stream_ptr(stream) -> int:
    if stream is None:  # (the handle alone: building torch's stream object takes longer than all checks of a small call)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


def _on_stream(call, stream, *args, held=()):
    """call(*args) on `stream`, which is not None: what it allocates comes from that stream's pool, whose blocks are free in
    that stream's order (one of the current stream's pool may have been freed with kernels still running there).  torch hands
    a block on when its tensor dies, so the tensors that the call takes are tied to `stream`, and its results to the stream
    that was current as well, where they will be used.  held: what the call uses besides its arguments, tensors of the object
    that it is a method of, which may be dropped with work under way as well."""
    before = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        try:
            out = call(*args)
        finally:  # (a call that fails at its second launch has enqueued the first)
            for t in _tensors_of((args, held)):
                if t.is_cuda:
                    t.record_stream(stream)
    for t in _tensors_of(out if isinstance(out, tuple) else (out,)):
        t.record_stream(before)
    return out


def _tensors_of(things):
    for t in things.values() if isinstance(things, dict) else things:
        if isinstance(t, torch.Tensor):
            yield t
        elif isinstance(t, AxQ4):
            yield t.codes
            yield t.scales
        elif isinstance(t, (tuple, list, dict)):
            yield from _tensors_of(t)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _workspace(need: int, device) -> torch.Tensor:
    """Temporary scratch for one call."""
    return torch.empty(max(int(need), 256), dtype=torch.uint8, device=device)


def _conv_desc(x_shape, w_shape, stride, pad, dilation=1, depthwise=False, signed=False, groups=1) -> ax_conv_desc_t:
    N, H, W, Cin = [int(v) for v in x_shape]
    KH, KW, _, last = [int(v) for v in w_shape]
    Cout = Cin * last if depthwise else last
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    dh, dw = _pair(dilation)
    return ax_conv_desc_t(N, H, W, Cin, KH, KW, Cout, sh, sw, ph, pw, dh, dw, int(bool(depthwise)), int(bool(signed)),
                          int(groups))


def _dense_desc(M: int, K: int, N: int) -> ax_conv_desc_t:
    return ax_conv_desc_t(int(M), 1, 1, int(K), 1, 1, int(N), 1, 1, 0, 0, 1, 1, 0, 0)


def _out_hw(d: ax_conv_desc_t) -> Tuple[int, int]:
    OH = (d.H + 2 * d.pad_h - d.dilation_h * (d.KH - 1) - 1) // d.stride_h + 1
    OW = (d.W + 2 * d.pad_w - d.dilation_w * (d.KW - 1) - 1) // d.stride_w + 1
    return OH, OW


def ax_conv2d_workspace_bytes(x_shape, w_shape, stride=1, pad=0) -> int:
    d = _conv_desc(x_shape, w_shape, stride, pad)
    t = _tune_arg()
    if t is not None:
        return int(lib().ax_conv2d_ex_workspace_bytes(ctypes.byref(d), t))
    return int(lib().ax_conv2d_workspace_bytes(d.N, d.H, d.W, d.Cin, d.KH, d.KW, d.Cout, d.stride_h, d.stride_w,
                                               d.pad_h, d.pad_w))


def ax_dense_workspace_bytes(M: int, K: int, N: int) -> int:
    t = _tune_arg()
    if t is not None:
        return int(lib().ax_conv2d_ex_workspace_bytes(ctypes.byref(_dense_desc(M, K, N)), t))
    return int(lib().ax_dense_workspace_bytes(int(M), int(K), int(N)))


def _check_lut(lut, n_entries=65536):
    if lut.dtype not in (torch.int16, torch.uint16):
        raise TypeError("lut must be a 16-bit integer tensor")
    _dev(lut, lut.dtype, "lut")
    if lut.numel() != n_entries:
        raise ValueError("lut must have %d entries" % n_entries)


def ax_conv2d(x, w, lut, stride, pad, q, acc_out=None, y_out=None, workspace=None, stream=None):
    """Enqueue one layer.  x: uint8 [N,H,W,Cin]; w: uint8 [KH,KW,Cin,Cout]; lut: int16/uint16
    [65536] (bit pattern of the uint16 entries); acc_out: int32 [N,OH,OW,Cout]; y_out: float32.
    Missing outputs / workspace are allocated with torch (the C call itself never allocates).
    Returns (acc_out, y_out)."""
    if stream is not None:
        return _on_stream(ax_conv2d, stream, x, w, lut, stride, pad, q, acc_out, y_out, workspace)
    # Small layers are bound by this function, not by the device: the plain entry point takes the sizes as they are, no
    # descriptor is filled in and read back (16 x 16 x 8, 3 x 3: 13.5 us a call, 11.4 now; 6.5 on the device).
    L = lib()
    _dev(x, torch.uint8, "x")
    _dev(w, torch.uint8, "w")
    _check_lut(lut)
    xs, ws = x.shape, w.shape
    if len(xs) != 4 or len(ws) != 4 or ws[2] != xs[3]:
        raise ValueError("x must be [N,H,W,Cin] and w [KH,KW,Cin,Cout]")
    N, H, W, Cin = xs
    KH, KW, _, Cout = ws
    (sh, sw), (ph, pw) = _pair(stride), _pair(pad)
    OH, OW = (H + 2 * ph - KH) // sh + 1, (W + 2 * pw - KW) // sw + 1
    if OH <= 0 or OW <= 0:
        _check(-2)
    acc_out, y_out = _outs((N, OH, OW, Cout), x.device, acc_out, y_out)
    if workspace is None:  # (a workspace handed in is checked by the C call itself)
        workspace = _workspace(ax_conv2d_workspace_bytes(xs, ws, stride, pad), x.device)
    _dev(workspace, torch.uint8, "workspace")
    tail = (ctypes.byref(_quant(q)), _ptr(None if acc_out is False else acc_out), _ptr(None if y_out is False else y_out),
            _ptr(workspace), workspace.numel(), _stream_ptr(None))
    t = _tune_arg()
    if t is None:
        rc = L.ax_conv2d(_ptr(x), N, H, W, Cin, _ptr(w), KH, KW, Cout, _ptr(lut), sh, sw, ph, pw, *tail)
    else:
        rc = L.ax_conv2d_ex(ctypes.byref(_conv_desc(xs, ws, stride, pad)), t, _ptr(x), _ptr(w), _ptr(lut), *tail)
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


def ax_dense(x, w, lut, q, acc_out=None, y_out=None, workspace=None, stream=None):
    """x: uint8 [M,K]; w: uint8 [K,N]; outputs [M,N]."""
    if stream is not None:
        return _on_stream(ax_dense, stream, x, w, lut, q, acc_out, y_out, workspace)
    L = lib()
    _dev(x, torch.uint8, "x")
    _dev(w, torch.uint8, "w")
    _check_lut(lut)
    if x.dim() != 2 or w.dim() != 2 or w.shape[0] != x.shape[1]:
        raise ValueError("x must be [M,K] and w [K,N]")
    M, K = x.shape
    N = w.shape[1]
    acc_out, y_out = _outs((M, N), x.device, acc_out, y_out)
    if workspace is None:
        workspace = _workspace(ax_dense_workspace_bytes(M, K, N), x.device)
    _dev(workspace, torch.uint8, "workspace")
    qs = _quant(q)
    t = _tune_arg()
    tail = (ctypes.byref(qs), _ptr(None if acc_out is False else acc_out), _ptr(None if y_out is False else y_out),
            _ptr(workspace), workspace.numel(), ctypes.c_void_p(_stream_ptr(None)))
    if t is None:
        rc = L.ax_dense(_ptr(x), M, K, _ptr(w), N, _ptr(lut), *tail)
    else:
        rc = L.ax_conv2d_ex(ctypes.byref(_dense_desc(M, K, N)), t, _ptr(x), _ptr(w), _ptr(lut), *tail)
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


def ax_conv2d_multi_lut_workspace_bytes(x_shape, w_shape, num_luts, stride=1, pad=0) -> int:
    d = _conv_desc(x_shape, w_shape, stride, pad)
    return int(lib().ax_conv2d_multi_lut_workspace_bytes(d.N, d.H, d.W, d.Cin, d.KH, d.KW, d.Cout, int(num_luts),
                                                         d.stride_h, d.stride_w, d.pad_h, d.pad_w))


def ax_conv2d_multi_lut(x, w, luts, stride, pad, q, acc_out=None, y_out=None, workspace=None, stream=None):
    """One layer against T tables.  luts: 16-bit integer CUDA tensor [T, 65536]; outputs
    [T, N, OH, OW, Cout].  Returns (acc_out, y_out); pass False to skip one of them.  With a
    default tune set the call goes through a layer handle (the one-call entry takes no tune)."""
    if stream is not None:
        return _on_stream(ax_conv2d_multi_lut, stream, x, w, luts, stride, pad, q, acc_out, y_out, workspace)
    L = lib()
    _dev(x, torch.uint8, "x")
    _dev(w, torch.uint8, "w")
    if luts.dim() != 2 or luts.shape[1] != 65536:
        raise ValueError("luts must be [T, 65536]")
    T = int(luts.shape[0])
    _check_lut(luts, T * 65536)
    if x.dim() != 4 or w.dim() != 4 or w.shape[2] != x.shape[3]:
        raise ValueError("x must be [N,H,W,Cin] and w [KH,KW,Cin,Cout]")
    d = _conv_desc(x.shape, w.shape, stride, pad)
    OH, OW = _out_hw(d)
    if OH <= 0 or OW <= 0:
        _check(-2)
    acc_out, y_out = _outs((T, d.N, OH, OW, d.Cout), x.device, acc_out, y_out)
    qs = _quant(q)
    if _tune_arg() is not None:
        with AxLayer(d, qs, T) as layer:
            layer.prepare(w, luts)
            layer.run(x, acc_out, y_out, workspace=workspace)
        return (None if acc_out is False else acc_out), (None if y_out is False else y_out)
    if workspace is None:
        workspace = _workspace(ax_conv2d_multi_lut_workspace_bytes(x.shape, w.shape, T, stride, pad), x.device)
    _dev(workspace, torch.uint8, "workspace")
    rc = L.ax_conv2d_multi_lut(_ptr(x), d.N, d.H, d.W, d.Cin, _ptr(w), d.KH, d.KW, d.Cout, _ptr(luts), T, d.stride_h,
                               d.stride_w, d.pad_h, d.pad_w, ctypes.byref(qs),
                               _ptr(None if acc_out is False else acc_out), _ptr(None if y_out is False else y_out),
                               _ptr(workspace), workspace.numel(), ctypes.c_void_p(_stream_ptr(None)))
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


def ax_conv2d_ex(x, w, lut, stride, pad, q, dilation=1, depthwise=False, acc_out=None, y_out=None, workspace=None,
                 stream=None, groups=1):
    """Operator variants.  Signed form: x, w int8 and lut int16 (chosen by x.dtype).  Depthwise:
    w is [KH,KW,Cin,mult].  Grouped: w is [KH,KW,Cin/groups,Cout].  q.pad_code None selects the
    zero point.  Returns (acc_out, y_out)."""
    if stream is not None:
        return _on_stream(ax_conv2d_ex, stream, x, w, lut, stride, pad, q, dilation, depthwise, acc_out, y_out, workspace, None,
                          groups)
    L = lib()
    signed = x.dtype == torch.int8
    cdt = torch.int8 if signed else torch.uint8
    _dev(x, cdt, "x")
    _dev(w, cdt, "w")
    _check_lut(lut)
    if x.dim() != 4 or w.dim() != 4 or w.shape[2] * int(groups) != x.shape[3]:
        raise ValueError("x must be [N,H,W,Cin] and w [KH,KW,Cin/groups,Cout] (or [KH,KW,Cin,mult])")
    desc = _conv_desc(x.shape, w.shape, stride, pad, dilation, depthwise, signed, groups)
    OH, OW = _out_hw(desc)
    if OH <= 0 or OW <= 0:
        _check(-2)
    acc_out, y_out = _outs((desc.N, OH, OW, desc.Cout), x.device, acc_out, y_out)
    t = _tune_arg()
    if workspace is None:
        workspace = _workspace(int(L.ax_conv2d_ex_workspace_bytes(ctypes.byref(desc), t)), x.device)
    _dev(workspace, torch.uint8, "workspace")
    qs = _quant(q)
    rc = L.ax_conv2d_ex(ctypes.byref(desc), t, _ptr(x), _ptr(w), _ptr(lut), ctypes.byref(qs),
                        _ptr(None if acc_out is False else acc_out), _ptr(None if y_out is False else y_out),
                        _ptr(workspace), workspace.numel(), ctypes.c_void_p(_stream_ptr(None)))
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


def ax_conv2d_transpose(x, w, lut, stride, pad, q, dilation=1, acc_out=None, y_out=None, workspace=None, stream=None):
    """Transposed convolution by zero insertion.  x: codes [N,H,W,Cin] (uint8, or int8 for the
    signed form), w: [KH,KW,Cin,Cout].  Returns (acc_out, y_out) of shape [N,OH,OW,Cout] with
    OH = (H-1)*stride + 1 + dilation*(KH-1) - 2*pad."""
    if stream is not None:
        return _on_stream(ax_conv2d_transpose, stream, x, w, lut, stride, pad, q, dilation, acc_out, y_out, workspace)
    L = lib()
    signed = x.dtype == torch.int8
    cdt = torch.int8 if signed else torch.uint8
    _dev(x, cdt, "x")
    _dev(w, cdt, "w")
    _check_lut(lut)
    if x.dim() != 4 or w.dim() != 4 or w.shape[2] != x.shape[3]:
        raise ValueError("x must be [N,H,W,Cin] and w [KH,KW,Cin,Cout]")
    desc = _conv_desc(x.shape, w.shape, stride, pad, dilation, False, signed)
    OH = (desc.H - 1) * desc.stride_h + 1 + desc.dilation_h * (desc.KH - 1) - 2 * desc.pad_h
    OW = (desc.W - 1) * desc.stride_w + 1 + desc.dilation_w * (desc.KW - 1) - 2 * desc.pad_w
    if OH <= 0 or OW <= 0:
        _check(-2)
    acc_out, y_out = _outs((desc.N, OH, OW, desc.Cout), x.device, acc_out, y_out)
    t = _tune_arg()
    if workspace is None:
        n = int(L.ax_conv2d_transpose_workspace_bytes(ctypes.byref(desc), t))
        if n == 0:
            _check(-2)
        workspace = _workspace(n, x.device)
    _dev(workspace, torch.uint8, "workspace")
    qs = _quant(q)
    rc = L.ax_conv2d_transpose(ctypes.byref(desc), t, _ptr(x), _ptr(w), _ptr(lut), ctypes.byref(qs),
                               _ptr(None if acc_out is False else acc_out), _ptr(None if y_out is False else y_out),
                               _ptr(workspace), workspace.numel(), ctypes.c_void_p(_stream_ptr(None)))
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


def ax_conv2d_backward(x, w, gy, stride, pad, q, dilation=1, gx_out=None, gw_out=None, workspace=None, stream=None):
    """Backward pass of a layer (straight-through).  x, w: codes (uint8, or int8 for the signed
    form); gy: float32 [N,OH,OW,Cout].  Returns (gx [N,H,W,Cin], gw [KH,KW,Cin,Cout]) as float32
    tensors; pass False to skip one of them."""
    if stream is not None:
        return _on_stream(ax_conv2d_backward, stream, x, w, gy, stride, pad, q, dilation, gx_out, gw_out, workspace)
    L = lib()
    signed = x.dtype == torch.int8
    cdt = torch.int8 if signed else torch.uint8
    _dev(x, cdt, "x")
    _dev(w, cdt, "w")
    _dev(gy, torch.float32, "gy")
    if x.dim() != 4 or w.dim() != 4 or w.shape[2] != x.shape[3]:
        raise ValueError("x must be [N,H,W,Cin] and w [KH,KW,Cin,Cout]")
    desc = _conv_desc(x.shape, w.shape, stride, pad, dilation, False, signed)
    OH, OW = _out_hw(desc)
    if OH <= 0 or OW <= 0:
        _check(-2)
    if tuple(gy.shape) != (desc.N, OH, OW, desc.Cout):
        raise ValueError("gy must be [N,OH,OW,Cout]")
    if gx_out is None:
        gx_out = torch.empty(x.shape, dtype=torch.float32, device=x.device)
    if gw_out is None:
        gw_out = torch.empty(w.shape, dtype=torch.float32, device=x.device)
    for o, ref, name in ((gx_out, x, "gx_out"), (gw_out, w, "gw_out")):
        if o is not False:
            _dev(o, torch.float32, name)
            if o.numel() != ref.numel():
                raise ValueError("%s has the wrong number of elements" % name)
    if workspace is None:
        workspace = _workspace(int(L.ax_conv2d_backward_workspace_bytes(ctypes.byref(desc))), x.device)
    _dev(workspace, torch.uint8, "workspace")
    qs = _quant(q)
    _check(L.ax_conv2d_backward(ctypes.byref(desc), ctypes.byref(qs), _ptr(x), _ptr(w), _ptr(gy),
                                _ptr(None if gx_out is False else gx_out), _ptr(None if gw_out is False else gw_out),
                                _ptr(workspace), workspace.numel(), ctypes.c_void_p(_stream_ptr(None))))
    return (None if gx_out is False else gx_out), (None if gw_out is False else gw_out)


class AxLayer:
    """A layer handle (ax_layer_*): filters and tables prepared once, then many calls.

    desc: ax_conv_desc_t; q: ax_quant_t or an object with x_scale, x_zp, w_scale, w_zp,
    pad_code (None = zero point); tune: dict with the fields of ax_tune_t (None = the module's
    default).  Device memory (prepared block, workspace) is torch tensors owned by this object
    unless the caller hands tensors in."""

    def __init__(self, desc: ax_conv_desc_t, q, num_luts: int = 1, tune=None):
        self._h = ctypes.c_void_p()
        self.desc = desc
        self.num_luts = int(num_luts)
        qs = q if isinstance(q, ax_quant_t) else _quant(q)
        _check(lib().ax_layer_create(ctypes.byref(desc), self.num_luts, ctypes.byref(qs), _tune_arg(tune),
                                     ctypes.byref(self._h)))
        self._keep = None  # tensors the handle's device pointers refer to
        self._ws = None

    def close(self):
        if self._h and _lib is not None:
            _lib.ax_layer_destroy(self._h)
        self._h = ctypes.c_void_p()
        self._keep = None
        self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:  # interpreter shutdown: the module's globals may be gone
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def prepared_bytes(self) -> int:
        return int(lib().ax_layer_prepared_bytes(self._h))

    @property
    def workspace_bytes(self) -> int:
        return int(lib().ax_layer_workspace_bytes(self._h))

    def out_shape(self):
        OH, OW = _out_hw(self.desc)
        shape = (self.desc.N, OH, OW, self.desc.Cout)
        return shape if self.num_luts == 1 else (self.num_luts,) + shape

    def plan(self) -> dict:
        out = [ctypes.c_int(0) for _ in range(4)]
        _check(lib().ax_layer_plan(self._h, *[ctypes.byref(o) for o in out]))
        paths = [ctypes.c_int(0) for _ in range(2)]
        _check(lib().ax_layer_plan_paths(self._h, *[ctypes.byref(o) for o in paths]))
        return {"variant": out[0].value, "tile": out[1].value, "workgroups": out[2].value, "pieces": out[3].value,
                "combine": paths[0].value, "tables": paths[1].value}

    def route(self) -> dict:
        """ax_probe_layer_route: which kernel the calls run ("tiles", "direct", "fewpix", "depthwise") and how
        it cuts the layer."""
        out = [ctypes.c_int(0) for _ in range(6)]
        _check(lib().ax_probe_layer_route(self._h, *[ctypes.byref(o) for o in out]))
        k, pixels, channels, tiles, workgroups, threads = [o.value for o in out]
        return {"kernel": ("tiles", "direct", "fewpix", "depthwise")[k], "pixels": pixels, "channels": channels,
                "tiles": tiles, "workgroups": workgroups, "threads": threads}

    def prepare(self, w, luts, prepared=None, stream=None):
        if stream is not None:
            return _on_stream(self.prepare, stream, w, luts, prepared)
        cdt = torch.int8 if self.desc.signed_codes else torch.uint8
        _dev(w, cdt, "w")
        _check_lut(luts, self.num_luts * 65536)
        if prepared is None:
            prepared = torch.empty(max(self.prepared_bytes, 256), dtype=torch.uint8, device=w.device)
        _dev(prepared, torch.uint8, "prepared")
        _check(lib().ax_layer_prepare(self._h, _ptr(w), _ptr(luts), _ptr(prepared), prepared.numel(),
                                      ctypes.c_void_p(_stream_ptr(None))))
        self._keep = (w, luts, prepared)
        return prepared

    def _held(self):
        return (self._keep or ()) + (self._ws,)

    def _args(self, x, acc_out, y_out, workspace):
        cdt = torch.int8 if self.desc.signed_codes else torch.uint8
        _dev(x, cdt, "x")
        acc_out, y_out = _outs(self.out_shape(), x.device, acc_out, y_out)
        if workspace is None:
            if self._ws is None or self._ws.device != x.device:
                self._ws = torch.empty(max(self.workspace_bytes, 256), dtype=torch.uint8, device=x.device)
            workspace = self._ws
        _dev(workspace, torch.uint8, "workspace")
        return acc_out, y_out, workspace

    def run(self, x, acc_out=None, y_out=None, workspace=None, stream=None):
        if stream is not None:
            out = _on_stream(self.run, stream, x, acc_out, y_out, workspace, held=self._held())
            if workspace is None:  # (of the pool of the first stream that runs the layer, this one or the current one among them)
                for s in (stream, torch.cuda.current_stream(stream.device)):
                    self._ws.record_stream(s)
            return out
        acc_out, y_out, workspace = self._args(x, acc_out, y_out, workspace)
        _check(lib().ax_layer_run(self._h, _ptr(x), _ptr(None if acc_out is False else acc_out),
                                  _ptr(None if y_out is False else y_out), _ptr(workspace), workspace.numel(),
                                  ctypes.c_void_p(_stream_ptr(None))))
        return (None if acc_out is False else acc_out), (None if y_out is False else y_out)

    def run_static(self, x, acc_out, y_out, stream=None):
        """ax_layer_run_static: scratch from the library's static device array; nothing is
        allocated, so the outputs must be handed in (False skips one of them)."""
        if stream is not None:
            return _on_stream(self.run_static, stream, x, acc_out, y_out, held=self._held())
        cdt = torch.int8 if self.desc.signed_codes else torch.uint8
        _dev(x, cdt, "x")
        if acc_out is None or y_out is None:
            raise ValueError("run_static allocates nothing: pass acc_out and y_out (False to skip one)")
        acc_out, y_out = _outs(self.out_shape(), x.device, acc_out, y_out)
        _check(lib().ax_layer_run_static(self._h, _ptr(x), _ptr(None if acc_out is False else acc_out),
                                         _ptr(None if y_out is False else y_out),
                                         ctypes.c_void_p(_stream_ptr(None))))
        return (None if acc_out is False else acc_out), (None if y_out is False else y_out)

    def kernel_ms(self, x, acc_out=None, y_out=None, workspace=None, reps: int = 8, stream=None) -> float:
        """ax_probe_layer_kernel_ms: duration of one launch of the layer's main kernel."""
        if stream is not None:
            return _on_stream(self.kernel_ms, stream, x, acc_out, y_out, workspace, reps, held=self._held())
        acc_out, y_out, workspace = self._args(x, acc_out, y_out, workspace)
        ms = ctypes.c_float(0.0)
        _check(lib().ax_probe_layer_kernel_ms(self._h, _ptr(x), _ptr(None if acc_out is False else acc_out),
                                              _ptr(None if y_out is False else y_out), _ptr(workspace),
                                              workspace.numel(), int(reps), ctypes.byref(ms),
                                              ctypes.c_void_p(_stream_ptr(None))))
        return float(ms.value)


def ax_range_workspace_bytes(n: int) -> int:
    return int(lib().ax_range_workspace_bytes(int(n)))


def ax_range_f32(x, relu=False, range_out=None, workspace=None, stream=None):
    """(min, max) of a float32 CUDA tensor into a float32 CUDA tensor of two."""
    if stream is not None:
        return _on_stream(ax_range_f32, stream, x, relu, range_out, workspace)
    L = lib()
    _dev(x, torch.float32, "x")
    if range_out is None:
        range_out = torch.empty(2, dtype=torch.float32, device=x.device)
    _dev(range_out, torch.float32, "range_out")
    if workspace is None:
        workspace = torch.empty(int(L.ax_range_workspace_bytes(x.numel())), dtype=torch.uint8, device=x.device)
    _dev(workspace, torch.uint8, "workspace")
    _check(L.ax_range_f32(_ptr(x), x.numel(), int(bool(relu)), _ptr(range_out), _ptr(workspace), workspace.numel(),
                          ctypes.c_void_p(_stream_ptr(None))))
    return range_out


def ax_quantize_f32(x, rng, relu=False, round_mode=0, codes_out=None, coeffs_out=None, stream=None):
    """Codes of a float32 CUDA tensor for the range `rng` (float32 CUDA tensor of two).
    coeffs_out: int32 CUDA tensor of two receiving the bit pattern of alpha and the value of
    beta (allocated when None).  Returns (codes_out, coeffs_out)."""
    if stream is not None:
        return _on_stream(ax_quantize_f32, stream, x, rng, relu, round_mode, codes_out, coeffs_out)
    L = lib()
    _dev(x, torch.float32, "x")
    _dev(rng, torch.float32, "range")
    if rng.numel() != 2:
        raise ValueError("range must hold two floats")
    if codes_out is None:
        codes_out = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    _dev(codes_out, torch.uint8, "codes_out")
    if codes_out.numel() != x.numel():
        raise ValueError("codes_out has the wrong number of elements")
    if coeffs_out is None:
        coeffs_out = torch.empty(2, dtype=torch.int32, device=x.device)
    _dev(coeffs_out, torch.int32, "coeffs_out")
    _check(L.ax_quantize_f32(_ptr(x), x.numel(), _ptr(rng), int(bool(relu)), int(round_mode), _ptr(codes_out),
                             _ptr(coeffs_out), ctypes.c_void_p(_stream_ptr(None))))
    return codes_out, coeffs_out


def ax_conv2d_f32_workspace_bytes(x_shape, w_shape, stride=1, pad=0) -> int:
    d = _conv_desc(x_shape, w_shape, stride, pad)
    t = _tune_arg()
    if t is not None:
        return int(lib().ax_conv2d_f32_ex_workspace_bytes(ctypes.byref(d), t))
    return int(lib().ax_conv2d_f32_workspace_bytes(d.N, d.H, d.W, d.Cin, d.KH, d.KW, d.Cout, d.stride_h, d.stride_w,
                                                   d.pad_h, d.pad_w))


def ax_dense_f32_workspace_bytes(M: int, K: int, N: int) -> int:
    t = _tune_arg()
    if t is not None:
        return int(lib().ax_conv2d_f32_ex_workspace_bytes(ctypes.byref(_dense_desc(M, K, N)), t))
    return int(lib().ax_dense_f32_workspace_bytes(int(M), int(K), int(N)))


def _f32_common(x, w, lut, x_range, w_range):
    _dev(x, torch.float32, "x")
    _dev(w, torch.float32, "w")
    for r, name in ((x_range, "x_range"), (w_range, "w_range")):
        if r is None:  # the layer takes the range itself
            continue
        _dev(r, torch.float32, name)
        if r.numel() != 2:
            raise ValueError("ranges must hold two floats")
    _check_lut(lut)


def _outs(shape, device, acc_out, y_out):
    if acc_out is None:
        acc_out = torch.empty(shape, dtype=torch.int32, device=device)
    if y_out is None:
        y_out = torch.empty(shape, dtype=torch.float32, device=device)
    n = 1
    for v in shape:
        n *= int(v)
    if acc_out is not False:
        _dev(acc_out, torch.int32, "acc_out")
    if y_out is not False:
        _dev(y_out, torch.float32, "y_out")
    for o in (acc_out, y_out):
        if o is not False and o.numel() != n:
            raise ValueError("output tensor has the wrong number of elements")
    return acc_out, y_out


def _f32_ex(desc, x, w, lut, x_range, w_range, relu, round_mode, acc_out, y_out, workspace, out_shape):
    L = lib()
    acc_out, y_out = _outs(out_shape, x.device, acc_out, y_out)
    t = _tune_arg()
    if workspace is None:
        workspace = _workspace(int(L.ax_conv2d_f32_ex_workspace_bytes(ctypes.byref(desc), t)), x.device)
    _dev(workspace, torch.uint8, "workspace")
    rc = L.ax_conv2d_f32_ex(ctypes.byref(desc), t, _ptr(x), _ptr(w), _ptr(lut), _ptr(x_range), _ptr(w_range),
                            int(bool(relu)), int(round_mode), _ptr(None if acc_out is False else acc_out),
                            _ptr(None if y_out is False else y_out), _ptr(workspace), workspace.numel(),
                            ctypes.c_void_p(_stream_ptr(None)))
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


def ax_conv2d_f32(x, w, lut, stride, pad, x_range=None, w_range=None, relu=False, round_mode=0, acc_out=None, y_out=None,
                  workspace=None, stream=None):
    """Float layer.  x: float32 [N,H,W,Cin]; w: float32 [KH,KW,Cin,Cout]; ranges: float32 CUDA
    tensors of two, or None to let the layer take the range of that tensor.  Returns (acc_out, y_out); pass False to skip one of them."""
    if stream is not None:
        return _on_stream(ax_conv2d_f32, stream, x, w, lut, stride, pad, x_range, w_range, relu, round_mode, acc_out,
                          y_out, workspace)
    L = lib()
    _f32_common(x, w, lut, x_range, w_range)
    if x.dim() != 4 or w.dim() != 4 or w.shape[2] != x.shape[3]:
        raise ValueError("x must be [N,H,W,Cin] and w [KH,KW,Cin,Cout]")
    d = _conv_desc(x.shape, w.shape, stride, pad)
    OH, OW = _out_hw(d)
    if OH <= 0 or OW <= 0:
        _check(-2)
    if _tune_arg() is not None:
        return _f32_ex(d, x, w, lut, x_range, w_range, relu, round_mode, acc_out, y_out, workspace,
                       (d.N, OH, OW, d.Cout))
    acc_out, y_out = _outs((d.N, OH, OW, d.Cout), x.device, acc_out, y_out)
    if workspace is None:
        workspace = _workspace(ax_conv2d_f32_workspace_bytes(x.shape, w.shape, stride, pad), x.device)
    _dev(workspace, torch.uint8, "workspace")
    rc = L.ax_conv2d_f32(_ptr(x), d.N, d.H, d.W, d.Cin, _ptr(w), d.KH, d.KW, d.Cout, _ptr(lut), d.stride_h, d.stride_w,
                         d.pad_h, d.pad_w, _ptr(x_range), _ptr(w_range), int(bool(relu)), int(round_mode),
                         _ptr(None if acc_out is False else acc_out), _ptr(None if y_out is False else y_out),
                         _ptr(workspace), workspace.numel(), ctypes.c_void_p(_stream_ptr(None)))
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


def ax_conv2d_f32_ex(x, w, lut, stride, pad, x_range=None, w_range=None, relu=False, round_mode=0, dilation=1,
                     depthwise=False, signed=False, acc_out=None, y_out=None, workspace=None, stream=None, groups=1):
    """Float layer with dilation / signed codes / depthwise filters (w [KH,KW,Cin,mult]) / grouped
    filters (w [KH,KW,Cin/groups,Cout]).  Returns (acc_out, y_out); pass False to skip one of them."""
    if stream is not None:
        return _on_stream(ax_conv2d_f32_ex, stream, x, w, lut, stride, pad, x_range, w_range, relu, round_mode, dilation,
                          depthwise, signed, acc_out, y_out, workspace, None, groups)
    _f32_common(x, w, lut, x_range, w_range)
    if x.dim() != 4 or w.dim() != 4 or w.shape[2] * int(groups) != x.shape[3]:
        raise ValueError("x must be [N,H,W,Cin] and w [KH,KW,Cin/groups,Cout] (or [KH,KW,Cin,mult])")
    desc = _conv_desc(x.shape, w.shape, stride, pad, dilation, depthwise, signed, groups)
    OH, OW = _out_hw(desc)
    if OH <= 0 or OW <= 0:
        _check(-2)
    return _f32_ex(desc, x, w, lut, x_range, w_range, relu, round_mode, acc_out, y_out, workspace,
                   (desc.N, OH, OW, desc.Cout))


def ax_dense_f32(x, w, lut, x_range=None, w_range=None, relu=False, round_mode=0, acc_out=None, y_out=None, workspace=None,
                 stream=None):
    """x: float32 [M,K]; w: float32 [K,N]; outputs [M,N]."""
    if stream is not None:
        return _on_stream(ax_dense_f32, stream, x, w, lut, x_range, w_range, relu, round_mode, acc_out, y_out, workspace)
    L = lib()
    _f32_common(x, w, lut, x_range, w_range)
    if x.dim() != 2 or w.dim() != 2 or w.shape[0] != x.shape[1]:
        raise ValueError("x must be [M,K] and w [K,N]")
    M, K = x.shape
    N = w.shape[1]
    if _tune_arg() is not None:
        return _f32_ex(_dense_desc(M, K, N), x, w, lut, x_range, w_range, relu, round_mode, acc_out, y_out, workspace,
                       (M, N))
    acc_out, y_out = _outs((M, N), x.device, acc_out, y_out)
    if workspace is None:
        workspace = _workspace(ax_dense_f32_workspace_bytes(M, K, N), x.device)
    _dev(workspace, torch.uint8, "workspace")
    rc = L.ax_dense_f32(_ptr(x), M, K, _ptr(w), N, _ptr(lut), _ptr(x_range), _ptr(w_range), int(bool(relu)),
                        int(round_mode), _ptr(None if acc_out is False else acc_out),
                        _ptr(None if y_out is False else y_out), _ptr(workspace), workspace.numel(),
                        ctypes.c_void_p(_stream_ptr(None)))
    _check(rc)
    return (None if acc_out is False else acc_out), (None if y_out is False else y_out)


# ---- feed-forward operators: norm, products, gated block, optimizer step -----------------------------------------------
#
# Matrices are torch tensors whose last dimension is contiguous; the leading dimensions are rows, at any pitch where there is
# one of them, contiguous where there are more.  Outputs that are not handed in are allocated with torch.  As with the lookup
# layers, nothing here is recorded by autograd: gradients are calls of their own.


_DT = {torch.float32: AX_F32, torch.bfloat16: AX_BF16}


def _float_dtype(t, name: str) -> int:
    dt = _DT.get(t.dtype)
    if dt is None:
        raise TypeError("%s must be float32 or bfloat16, got %s" % (name, t.dtype))
    return dt


# Descriptions of calls that were checked before, with what they need of workspace: every check of a call depends on the
# types, shapes and pitches of its tensors alone (and on whether they start on 16 bytes).  For a call of one token the
# checks would take longer than its kernels.
_checked = {}


def _remember(key, value):
    if len(_checked) >= 4096:
        _checked.clear()
    _checked[key] = value
    return value


def _sig(t):
    if t is None or t is False:
        return t
    return t.dtype, t.shape, t.stride(), t.device


def _mat(t, dtype, name: str) -> Tuple[int, int, int]:
    """(rows, columns, row pitch) of a matrix."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    n = t.dim()
    if n == 2:
        r, c = t.shape
        if c > 1 and t.stride(1) != 1:
            raise ValueError("%s must have contiguous rows" % name)
        if r <= 1:
            return r, c, c
        ld = t.stride(0)
        if ld < c:
            raise ValueError("%s must not overlap itself" % name)
        return r, c, ld
    if n == 0 or not t.is_contiguous():
        raise ValueError("%s must be a matrix with contiguous rows, or contiguous" % name)
    c = t.shape[-1]
    r = 1
    for v in t.shape[:-1]:
        r *= v
    return r, c, c


def _mat_of(t, dtype, rows: int, cols: int, name: str) -> int:
    """Row pitch of a matrix that has to be [rows, cols]."""
    r, c, ld = _mat(t, dtype, name)
    if r != rows or c != cols:
        raise ValueError("%s must be [%d, %d], got [%d, %d]" % (name, rows, cols, r, c))
    return ld


def _vec_of(t, dtype, n: int, name: str) -> None:
    _dev(t, dtype, name)
    if t.numel() != n:
        raise ValueError("%s must have %d elements" % (name, n))


def _act_code(act: str) -> int:
    if act not in AX_ACTS:
        raise ValueError("act must be one of %s" % ", ".join(AX_ACTS))
    return AX_ACTS[act]


def _norm_desc(x, residual, sum_out, weight, eps, normalize) -> ax_norm_desc_t:
    dt = _float_dtype(x, "x")
    rows, cols, ld = _mat(x, x.dtype, "x")
    d = ax_norm_desc_t(rows, cols, ld, cols, cols, cols, dt, dt, float(eps), int(bool(normalize)))
    if weight is not None:
        d.w_dtype = _float_dtype(weight, "weight")
        _vec_of(weight, weight.dtype, cols, "weight")
    if residual is not None:
        d.residual_ld = _mat_of(residual, x.dtype, rows, cols, "residual")
    elif sum_out is not None and sum_out is not False:
        raise ValueError("sum_out needs a residual")
    if sum_out is not None and sum_out is not False:
        d.sum_ld = _mat_of(sum_out, x.dtype, rows, cols, "sum_out")
    return d


def ax_rmsnorm(x, weight, residual=None, eps=1e-5, sum_out=None, y_out=None, rstd_out=None, stream=None):
    """Root-mean-square norm of rows: t = x + residual, y = t * rstd * weight.  Returns (y, t, rstd); t is None without
    a residual.  sum_out may be x or residual themselves; False skips t (or rstd)."""
    if stream is not None:
        return _on_stream(ax_rmsnorm, stream, x, weight, residual, eps, sum_out, y_out, rstd_out)
    key = ("rmsnorm", eps, _sig(x), _sig(weight), _sig(residual), _sig(sum_out), _sig(y_out), _sig(rstd_out))
    if residual is not None and sum_out is None:
        sum_out = torch.empty_like(x)
    if y_out is None:
        y_out = torch.empty_like(x)
    if rstd_out is None:
        rstd_out = x.new_empty(x.shape[:-1], dtype=torch.float32)
    d = _checked.get(key)
    if d is None:
        d = _norm_desc(x, residual, sum_out, weight, eps, True)
        d.y_ld = _mat_of(y_out, x.dtype, d.rows, d.cols, "y_out")
        if rstd_out is not False:
            _vec_of(rstd_out, torch.float32, d.rows, "rstd_out")
        _remember(key, d)
    sum_out, rstd_out = (None if o is False else o for o in (sum_out, rstd_out))
    _check(lib().ax_rmsnorm(d, _ptr(x), _ptr(residual), _ptr(weight), _ptr(sum_out), _ptr(y_out), _ptr(rstd_out),
                            _stream_ptr(None)))
    return y_out, sum_out, rstd_out


def ax_rmsnorm_q8(x, weight=None, residual=None, eps=1e-5, normalize=True, sum_out=None, codes_out=None, scales_out=None,
                  values_out=None, values=False, stream=None):
    """The norm's output as int8 codes with a scale a row: y = codes * scales[:, None].  normalize False: the rows
    themselves (times weight).  Returns (codes, scales, t, values); values, the float32 values that the codes stand for,
    is None unless asked for."""
    if stream is not None:
        return _on_stream(ax_rmsnorm_q8, stream, x, weight, residual, eps, normalize, sum_out, codes_out, scales_out,
                          values_out, values)
    key = ("rmsnorm_q8", eps, normalize, _sig(x), _sig(weight), _sig(residual), _sig(sum_out), _sig(codes_out), _sig(scales_out),
           _sig(values_out))
    if residual is not None and sum_out is None:
        sum_out = torch.empty_like(x)
    if codes_out is None:
        codes_out = torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format)
    if scales_out is None:
        scales_out = x.new_empty(x.shape[:-1], dtype=torch.float32)
    if values_out is None and values:
        values_out = torch.empty_like(x, dtype=torch.float32, memory_format=torch.contiguous_format)
    d = _checked.get(key)
    if d is None:
        d = _norm_desc(x, residual, sum_out, weight, eps, normalize)
        _vec_of(codes_out, torch.int8, d.rows * d.cols, "codes_out")
        _vec_of(scales_out, torch.float32, d.rows, "scales_out")
        if values_out is not None:
            _vec_of(values_out, torch.float32, d.rows * d.cols, "values_out")
        _remember(key, d)
    sum_out = None if sum_out is False else sum_out
    _check(lib().ax_rmsnorm_q8(d, _ptr(x), _ptr(residual), _ptr(weight), _ptr(sum_out), _ptr(codes_out), _ptr(scales_out),
                               _ptr(values_out), _stream_ptr(None)))
    return codes_out, scales_out, sum_out, values_out


def _scratch(need: int, workspace, device):
    if workspace is None:
        return _workspace(need, device) if need else None
    return _dev(workspace, torch.uint8, "workspace")


def _ws_args(ws):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel())


def ax_rmsnorm_backward(gy, t, weight, rstd, gsum=None, gx_out=None, gw_out=None, workspace=None, stream=None):
    """Gradients of ax_rmsnorm: (gx, gw), gx for x and residual alike, gw float32.  t, rstd: what the forward pass
    returned (t = x without a residual); gsum: the gradient that reaches t from the residual stream.  False skips one."""
    if stream is not None:
        return _on_stream(ax_rmsnorm_backward, stream, gy, t, weight, rstd, gsum, gx_out, gw_out, workspace)
    L = lib()
    key = ("rmsnorm_backward", _sig(gy), _sig(t), _sig(weight), _sig(rstd), _sig(gsum), _sig(gx_out), _sig(gw_out))
    if gx_out is None:
        gx_out = torch.empty_like(t)
    if gw_out is None:
        gw_out = torch.empty_like(weight, dtype=torch.float32)
    hit = _checked.get(key)
    if hit is None:
        rows, cols, ld = _mat(t, t.dtype, "t")
        d = ax_norm_desc_t(rows, cols, ld, cols, cols, _mat_of(gy, t.dtype, rows, cols, "gy"), _float_dtype(t, "t"),
                           _float_dtype(weight, "weight"), 0.0, 1)
        _vec_of(weight, weight.dtype, cols, "weight")
        _vec_of(rstd, torch.float32, rows, "rstd")
        if gsum is not None:
            d.residual_ld = _mat_of(gsum, t.dtype, rows, cols, "gsum")
        if gx_out is not False:
            d.sum_ld = _mat_of(gx_out, t.dtype, rows, cols, "gx_out")
        if gw_out is not False:
            _vec_of(gw_out, torch.float32, cols, "gw_out")
        hit = _remember(key, (d, int(L.ax_rmsnorm_backward_workspace_bytes(d))))
    d, need = hit
    gx_out, gw_out = (None if o is False else o for o in (gx_out, gw_out))
    ws = _scratch(need, workspace, t.device)
    _check(L.ax_rmsnorm_backward(d, _ptr(gy), _ptr(gsum), _ptr(t), _ptr(weight), _ptr(rstd), _ptr(gx_out), _ptr(gw_out),
                                 *_ws_args(ws), _stream_ptr(None)))
    return gx_out, gw_out


def _matmul_desc(x, w, act, transposed, out_dtype, aligned, names=("x", "w"), codes=False) -> ax_matmul_desc_t:
    dt = AX_BF16 if codes else _float_dtype(x, names[0])  # (of codes the library does not look at it)
    M, K, x_ld = _mat(x, x.dtype, names[0])
    wr, wc, w_ld = _mat(w, x.dtype, names[1])
    if w.dim() != 2 or (wc if transposed else wr) != K:
        raise ValueError("%s must be %s for %s [M,K]" % (names[1], "[N,K]" if transposed else "[K,N]", names[0]))
    N = wr if transposed else wc
    odt = _DT.get(out_dtype)
    if odt is None:
        raise TypeError("out_dtype must be float32 or bfloat16")
    return ax_matmul_desc_t(M, N, K, x_ld, w_ld, N, N, dt, odt, _act_code(act), int(bool(transposed)), int(not aligned))


def _columns(w, transposed) -> int:
    if w.dim() != 2:
        raise ValueError("weights must be matrices")
    return w.shape[0] if transposed else w.shape[1]


def _epilogue_args(d, bias, residual, y_out, z_out, dtype, name="y_out"):
    if bias is not None:
        _vec_of(bias, dtype, d.N, "bias")
    if residual is not None:
        d.residual_ld = _mat_of(residual, dtype, d.M, d.N, "residual")
    if z_out is not None:
        _vec_of(z_out, dtype, d.M * d.N, "z_out")
    d.y_ld = _mat_of(y_out, dtype, d.M, d.N, name)


def _codes_of(x, x_scales, w, w_scales, M, N):
    for t, name in ((x, "x"), (w, "w")):
        if t.dtype != torch.int8:
            raise TypeError("%s must have dtype torch.int8, got %s" % (name, t.dtype))
    _vec_of(x_scales, torch.float32, M, "x_scales")
    _vec_of(w_scales, torch.float32, N, "w_scales")


def ax_matmul(x, w, bias=None, residual=None, act="none", transposed=False, out_dtype=None, save=False, y_out=None, z_out=None,
              workspace=None, stream=None):
    """y = act(x w + bias) + residual.  x: [M,K]; w: [K,N], or [N,K] with transposed; float32 or bfloat16 both; bias,
    residual and the outputs have out_dtype (x's by default).  Returns (y, z): z, the value before the activation, with
    save or z_out, otherwise None."""
    if stream is not None:
        return _on_stream(ax_matmul, stream, x, w, bias, residual, act, transposed, out_dtype, save, y_out, z_out, workspace)
    L = lib()
    dev = x.device
    out_dtype = x.dtype if out_dtype is None else out_dtype
    xp, wp = x.data_ptr(), w.data_ptr()
    aligned = (xp | wp) % 16 == 0
    key = ("matmul", act, transposed, out_dtype, aligned, save, _sig(x), _sig(w), _sig(bias), _sig(residual), _sig(y_out),
           _sig(z_out))
    if y_out is None:
        y_out = x.new_empty(x.shape[:-1] + (_columns(w, transposed),), dtype=out_dtype)
    if z_out is None and save:
        z_out = torch.empty_like(y_out, memory_format=torch.contiguous_format)
    hit = _checked.get(key)
    if hit is None:
        d = _matmul_desc(x, w, act, transposed, out_dtype, aligned)
        _epilogue_args(d, bias, residual, y_out, z_out, out_dtype)
        hit = _remember(key, (d, int(L.ax_matmul_workspace_bytes(d))))
    d, need = hit
    ws = _scratch(need, workspace, dev)
    _check(L.ax_matmul(d, xp, wp, _ptr(bias), _ptr(residual), y_out.data_ptr(), _ptr(z_out), *_ws_args(ws), _stream_ptr(None)))
    return y_out, z_out


def ax_matmul_q8(x, x_scales, w, w_scales, bias=None, residual=None, act="none", out_dtype=torch.bfloat16, y_out=None,
                 workspace=None, stream=None):
    """y = act((x * x_scales) (w * w_scales)^T + bias) + residual on int8 codes: x [M,K] with a scale a row (what
    ax_rmsnorm_q8 returns), w [N,K] with a scale a row."""
    if stream is not None:
        return _on_stream(ax_matmul_q8, stream, x, x_scales, w, w_scales, bias, residual, act, out_dtype, y_out, workspace)
    L = lib()
    dev = x.device
    xp, wp = x.data_ptr(), w.data_ptr()
    aligned = (xp | wp) % 16 == 0
    key = ("matmul_q8", act, out_dtype, aligned, _sig(x), _sig(x_scales), _sig(w), _sig(w_scales), _sig(bias), _sig(residual),
           _sig(y_out))
    if y_out is None:
        y_out = x.new_empty(x.shape[:-1] + (_columns(w, True),), dtype=out_dtype)
    hit = _checked.get(key)
    if hit is None:
        d = _matmul_desc(x, w, act, True, out_dtype, aligned, codes=True)
        _codes_of(x, x_scales, w, w_scales, d.M, d.N)
        _epilogue_args(d, bias, residual, y_out, None, out_dtype)
        hit = _remember(key, (d, int(L.ax_matmul_q8_workspace_bytes(d))))
    d, need = hit
    ws = _scratch(need, workspace, dev)
    _check(L.ax_matmul_q8(d, xp, x_scales.data_ptr(), wp, w_scales.data_ptr(), _ptr(bias), _ptr(residual), y_out.data_ptr(),
                          *_ws_args(ws), _stream_ptr(None)))
    return y_out


def _grad_out(out, like):
    """A gradient with the shape and the row pitch of the tensor that it belongs to."""
    if out is None:
        return torch.empty_strided(like.shape, like.stride(), dtype=like.dtype, device=like.device)
    return out


def _check_grad(out, like, ld, name):
    if out is False:
        return
    r, c, _ = _mat(like, like.dtype, name)
    if _mat_of(out, like.dtype, r, c, name) != ld:
        raise ValueError("%s must have the row pitch of its tensor" % name)


def ax_matmul_backward(gy, x, w, z=None, act="none", transposed=False, gx_out=None, gw_out=None, gb_out=None, workspace=None,
                       stream=None):
    """Gradients of ax_matmul: (gx, gw, gb), gb float32; False skips one.  z: the value before the activation."""
    if stream is not None:
        return _on_stream(ax_matmul_backward, stream, gy, x, w, z, act, transposed, gx_out, gw_out, gb_out, workspace)
    L = lib()
    dev = x.device
    gp, xp, wp = gy.data_ptr(), x.data_ptr(), w.data_ptr()
    aligned = (xp | wp | (gp if act == "none" else 0)) % 16 == 0
    key = ("matmul_backward", act, transposed, aligned, _sig(gy), _sig(x), _sig(w), _sig(z), _sig(gx_out), _sig(gw_out), _sig(gb_out))
    gx_out, gw_out = _grad_out(gx_out, x), _grad_out(gw_out, w)
    if gb_out is None:
        gb_out = x.new_empty(_columns(w, transposed), dtype=torch.float32)
    hit = _checked.get(key)
    if hit is None:
        d = _matmul_desc(x, w, act, transposed, x.dtype, aligned)
        d.y_ld = _mat_of(gy, x.dtype, d.M, d.N, "gy")
        if z is not None:
            _vec_of(z, x.dtype, d.M * d.N, "z")
        elif d.act:
            raise ValueError("the gradient of an activation needs z")
        _check_grad(gx_out, x, d.x_ld, "gx_out")
        _check_grad(gw_out, w, d.w_ld, "gw_out")
        if gb_out is not False:
            _vec_of(gb_out, torch.float32, d.N, "gb_out")
        hit = _remember(key, (d, int(L.ax_matmul_backward_workspace_bytes(d))))
    d, need = hit
    gx_out, gw_out, gb_out = (None if o is False else o for o in (gx_out, gw_out, gb_out))
    ws = _scratch(need, workspace, dev)
    _check(L.ax_matmul_backward(d, gp, xp, wp, _ptr(z), _ptr(gx_out), _ptr(gw_out), _ptr(gb_out), *_ws_args(ws), _stream_ptr(None)))
    return gx_out, gw_out, gb_out


def _gated_desc(x, wg, wu, act, out_dtype, aligned, codes=False) -> ax_matmul_desc_t:
    d = _matmul_desc(x, wg, act, codes, out_dtype, aligned, ("x", "wg"), codes)  # (codes are [F,K])
    wr, wc, ld = _mat(wu, x.dtype, "wu")
    if wu.shape != wg.shape or ld != d.w_ld:
        raise ValueError("wg and wu must have one shape and one row pitch")
    return d


def ax_gated(x, wg, wu, act="silu", out_dtype=None, save=False, h_out=None, g_out=None, u_out=None, workspace=None, stream=None):
    """h = act(x wg) * (x wu).  x [M,K]; wg, wu [K,F]; float32 or bfloat16.  Returns (h, g, u): both projections with
    save (or g_out and u_out), otherwise None."""
    if stream is not None:
        return _on_stream(ax_gated, stream, x, wg, wu, act, out_dtype, save, h_out, g_out, u_out, workspace)
    L = lib()
    dev = x.device
    out_dtype = x.dtype if out_dtype is None else out_dtype
    xp, gp, up = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    aligned = (xp | gp | up) % 16 == 0
    key = ("gated", act, out_dtype, aligned, save, _sig(x), _sig(wg), _sig(wu), _sig(h_out), _sig(g_out), _sig(u_out))
    if h_out is None:
        h_out = x.new_empty(x.shape[:-1] + (_columns(wg, False),), dtype=out_dtype)
    if save:
        g_out, u_out = (torch.empty_like(h_out, memory_format=torch.contiguous_format) if o is None else o for o in (g_out, u_out))
    hit = _checked.get(key)
    if hit is None:
        d = _gated_desc(x, wg, wu, act, out_dtype, aligned)
        _epilogue_args(d, None, None, h_out, g_out, out_dtype, "h_out")
        if u_out is not None:
            _vec_of(u_out, out_dtype, d.M * d.N, "u_out")
        hit = _remember(key, (d, int(L.ax_gated_workspace_bytes(d))))
    d, need = hit
    ws = _scratch(need, workspace, dev)
    _check(L.ax_gated(d, xp, gp, up, h_out.data_ptr(), _ptr(g_out), _ptr(u_out), *_ws_args(ws), _stream_ptr(None)))
    return h_out, g_out, u_out


def ax_gated_q8(x, x_scales, wg, wg_scales, wu, wu_scales, act="silu", out_dtype=torch.bfloat16, h_out=None, workspace=None,
                stream=None):
    """The gated block on int8 codes: x [M,K] and wg, wu [F,K], each with a scale a row."""
    if stream is not None:
        return _on_stream(ax_gated_q8, stream, x, x_scales, wg, wg_scales, wu, wu_scales, act, out_dtype, h_out, workspace)
    L = lib()
    dev = x.device
    xp, gp, up = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    aligned = (xp | gp | up) % 16 == 0
    key = ("gated_q8", act, out_dtype, aligned, _sig(x), _sig(x_scales), _sig(wg), _sig(wg_scales), _sig(wu), _sig(wu_scales),
           _sig(h_out))
    if h_out is None:
        h_out = x.new_empty(x.shape[:-1] + (_columns(wg, True),), dtype=out_dtype)
    hit = _checked.get(key)
    if hit is None:
        d = _gated_desc(x, wg, wu, act, out_dtype, aligned, codes=True)
        _codes_of(x, x_scales, wg, wg_scales, d.M, d.N)
        _codes_of(x, x_scales, wu, wu_scales, d.M, d.N)
        _epilogue_args(d, None, None, h_out, None, out_dtype, "h_out")
        hit = _remember(key, (d, int(L.ax_gated_q8_workspace_bytes(d))))
    d, need = hit
    ws = _scratch(need, workspace, dev)
    _check(L.ax_gated_q8(d, xp, x_scales.data_ptr(), gp, wg_scales.data_ptr(), up, wu_scales.data_ptr(), h_out.data_ptr(),
                         *_ws_args(ws), _stream_ptr(None)))
    return h_out


def ax_gated_backward(gh, x, wg, wu, g, u, act="silu", gx_out=None, gwg_out=None, gwu_out=None, workspace=None, stream=None):
    """Gradients of ax_gated: (gx, gwg, gwu); gx_out False, or gwg_out and gwu_out False, skips them."""
    if stream is not None:
        return _on_stream(ax_gated_backward, stream, gh, x, wg, wu, g, u, act, gx_out, gwg_out, gwu_out, workspace)
    L = lib()
    dev = x.device
    xp, gp, up = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    aligned = (xp | gp | up) % 16 == 0
    key = ("gated_backward", act, aligned, _sig(gh), _sig(x), _sig(wg), _sig(wu), _sig(g), _sig(u), _sig(gx_out), _sig(gwg_out),
           _sig(gwu_out))
    gx_out, gwg_out, gwu_out = _grad_out(gx_out, x), _grad_out(gwg_out, wg), _grad_out(gwu_out, wu)
    hit = _checked.get(key)
    if hit is None:
        d = _gated_desc(x, wg, wu, act, x.dtype, aligned)
        d.y_ld = _mat_of(gh, x.dtype, d.M, d.N, "gh")
        _vec_of(g, x.dtype, d.M * d.N, "g")
        _vec_of(u, x.dtype, d.M * d.N, "u")
        for o, like, ld, name in ((gx_out, x, d.x_ld, "gx_out"), (gwg_out, wg, d.w_ld, "gwg_out"), (gwu_out, wu, d.w_ld, "gwu_out")):
            _check_grad(o, like, ld, name)
        hit = _remember(key, (d, int(L.ax_gated_backward_workspace_bytes(d))))
    d, need = hit
    gx_out, gwg_out, gwu_out = (None if o is False else o for o in (gx_out, gwg_out, gwu_out))
    ws = _scratch(need, workspace, dev)
    _check(L.ax_gated_backward(d, gh.data_ptr(), xp, gp, up, g.data_ptr(), u.data_ptr(), _ptr(gx_out), _ptr(gwg_out), _ptr(gwu_out),
                               *_ws_args(ws), _stream_ptr(None)))
    return gx_out, gwg_out, gwu_out


# ---- feed-forward blocks of experts ------------------------------------------------------------------------------------
#
# Rows are grouped by expert: offsets [experts + 1] and tokens [rows], both int32 on the device, are what ax_route returns.
# Weights are [experts, inputs, outputs] (or [experts, outputs, inputs] with transposed), the experts' matrices one behind the
# other.  Tensors of a call share a device, the current one.


def _same_device(*tensors):
    dev = tensors[0].device
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.device != dev:
            raise ValueError("all tensors must be on one device")


def _current_device(t):
    if t.is_cuda and t.device.type == "cuda" and t.device.index != torch._C._cuda_getDevice():
        raise ValueError("the tensors are on %s, which is not the current device" % t.device)


def _whole(t, n: int, name: str) -> None:
    """A vector of n whole numbers."""
    _dev(t, torch.int32, name)
    if n >= 0 and t.numel() != n:
        raise ValueError("%s must have %d elements" % (name, n))


def _weights(t, dtype, name: str):
    """(experts, rows, columns, row pitch) of the experts' matrices."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 3:
        raise ValueError("%s must be [experts, rows, columns]" % name)
    e, r, c = t.shape
    ld = t.stride(1) if r > 1 else t.stride(0) if e > 1 else c
    if (c > 1 and t.stride(2) != 1) or ld < c or (e > 1 and t.stride(0) != r * ld):
        raise ValueError("%s must have contiguous rows at one pitch, the experts' matrices one behind the other" % name)
    return e, r, c, ld


def ax_route(logits, k, normalize=True, experts_out=None, weights_out=None, offsets_out=None, rows_out=None, tokens_out=None,
             workspace=None, stream=None):
    """Each token's k largest logits and the order of its choices by expert.  logits: [tokens, experts].  Returns (experts
    [tokens, k], weights [tokens, k], offsets [experts + 1], rows [tokens, k], tokens [tokens * k]): weights float32, the softmax
    over the chosen experts (normalize) or over all; the others int32.  Where none of those for the choices is given they are from one
    allocation."""
    if stream is not None:
        return _on_stream(ax_route, stream, logits, k, normalize, experts_out, weights_out, offsets_out, rows_out, tokens_out, workspace)
    L = lib()
    key = ("route", k, normalize, _sig(logits), _sig(experts_out), _sig(weights_out), _sig(offsets_out), _sig(rows_out), _sig(tokens_out))
    hit = _checked.get(key)
    if hit is None:
        T, E, ld = _mat(logits, logits.dtype, "logits")
        d = ax_route_desc_t(T, ld, E, int(k), _float_dtype(logits, "logits"), int(bool(normalize)))
        if not 1 <= d.k <= E:
            raise ValueError("k must be between 1 and the number of experts")
        for t, n, dt, name in ((experts_out, T * d.k, torch.int32, "experts_out"), (weights_out, T * d.k, torch.float32, "weights_out"),
                               (offsets_out, E + 1, torch.int32, "offsets_out"), (rows_out, T * d.k, torch.int32, "rows_out"),
                               (tokens_out, T * d.k, torch.int32, "tokens_out")):
            if t is not None:
                _vec_of(t, dt, n, name)
        _same_device(logits, experts_out, weights_out, offsets_out, rows_out, tokens_out)
        hit = _remember(key, (d, int(L.ax_route_workspace_bytes(d)), logits.shape[:-1] + (d.k,), T * d.k))
    d, need, shape, n = hit
    _current_device(logits)
    if experts_out is weights_out is rows_out is tokens_out is None:  # (one allocation: for a token or two they are most of a call)
        experts_out, rows_out, tokens_out, weights_out = logits.new_empty((4,) + shape, dtype=torch.int32).unbind(0)
        tokens_out, weights_out = tokens_out.view(-1), weights_out.view(torch.float32)
    if experts_out is None:
        experts_out = logits.new_empty(shape, dtype=torch.int32)
    if weights_out is None:
        weights_out = logits.new_empty(shape, dtype=torch.float32)
    if offsets_out is None:
        offsets_out = logits.new_empty(d.experts + 1, dtype=torch.int32)
    if rows_out is None:
        rows_out = logits.new_empty(shape, dtype=torch.int32)
    if tokens_out is None:
        tokens_out = logits.new_empty(n, dtype=torch.int32)
    ws = _scratch(need, workspace, logits.device)
    _check(L.ax_route(d, _ptr(logits), _ptr(experts_out), _ptr(weights_out), _ptr(offsets_out), _ptr(rows_out), _ptr(tokens_out),
                      *_ws_args(ws), _stream_ptr(None)))
    return experts_out, weights_out, offsets_out, rows_out, tokens_out


def ax_route_backward(gweights, logits, experts, weights, normalize=True, glogits_out=None, stream=None):
    """The gradient of the logits from that of the weights [tokens, k] (float32); experts and weights as ax_route returned them."""
    if stream is not None:
        return _on_stream(ax_route_backward, stream, gweights, logits, experts, weights, normalize, glogits_out)
    L = lib()
    key = ("route_backward", normalize, _sig(gweights), _sig(logits), _sig(experts), _sig(weights), _sig(glogits_out))
    if glogits_out is None:
        glogits_out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    hit = _checked.get(key)
    if hit is None:
        T, E, ld = _mat(logits, logits.dtype, "logits")
        if experts.dim() < 1 or experts.numel() != T * experts.shape[-1]:
            raise ValueError("experts must be [tokens, k]")
        k = experts.shape[-1]
        d = ax_route_desc_t(T, ld, E, k, _float_dtype(logits, "logits"), int(bool(normalize)))
        _whole(experts, T * k, "experts")
        _vec_of(weights, torch.float32, T * k, "weights")
        _vec_of(gweights, torch.float32, T * k, "gweights")
        _same_device(logits, gweights, experts, weights, glogits_out)
        hit = _remember(key, (d, _mat_of(glogits_out, logits.dtype, T, E, "glogits_out")))
    d, ld = hit
    _current_device(logits)
    _check(L.ax_route_backward(d, _ptr(gweights), _ptr(logits), _ptr(experts), _ptr(weights), _ptr(glogits_out), ld, _stream_ptr(None)))
    return glogits_out


def _experts_desc(x, weights, names, offsets, tokens, act, transposed, aligned) -> ax_experts_desc_t:
    n, K, x_ld = _mat(x, x.dtype, "x")
    w = weights[0]
    E, wr, wc, w_ld = _weights(w, x.dtype, names[0])
    for other, name in zip(weights[1:], names[1:]):
        if _weights(other, x.dtype, name) != (E, wr, wc, w_ld):
            raise ValueError("%s and %s must have one shape and one row pitch" % (names[0], name))
    if (wc if transposed else wr) != K:
        raise ValueError("%s must be %s for x [rows,K]" % (names[0], "[experts,N,K]" if transposed else "[experts,K,N]"))
    _whole(offsets, E + 1, "offsets")
    if tokens is not None:
        _whole(tokens, -1, "tokens")
    N = wr if transposed else wc
    return ax_experts_desc_t(n if tokens is None else tokens.numel(), n, N, K, x_ld, w_ld, N, K, E, _float_dtype(x, "x"), _act_code(act),
                             int(bool(transposed)), int(tokens is not None), int(not aligned))


def _expert_columns(w, transposed) -> int:
    if w.dim() != 3:
        raise ValueError("the experts' weights must be [experts, rows, columns]")
    return w.shape[1] if transposed else w.shape[2]


def _rows_of(x, tokens):
    return x.shape[:-1] if tokens is None else (tokens.numel(),)


def ax_matmul_experts(x, w, offsets, tokens=None, act="none", transposed=False, save=False, y_out=None, z_out=None, workspace=None,
                      stream=None):
    """y = act(x w_e) for rows grouped by expert: row r is row tokens[r] of x (row r without tokens).  w: [experts,K,N], or
    [experts,N,K] with transposed; float32 or bfloat16.  Returns (y, z): z, the value before the activation, with save or z_out,
    otherwise None.  Rows that belong to no expert are not written."""
    if stream is not None:
        return _on_stream(ax_matmul_experts, stream, x, w, offsets, tokens, act, transposed, save, y_out, z_out, workspace)
    L = lib()
    xp, wp = x.data_ptr(), w.data_ptr()
    aligned = (wp | xp) % 16 == 0
    key = ("matmul_experts", act, transposed, aligned, save, _sig(x), _sig(w), _sig(offsets), _sig(tokens), _sig(y_out), _sig(z_out))
    if y_out is None:
        y_out = x.new_empty(_rows_of(x, tokens) + (_expert_columns(w, transposed),))
    if z_out is None and save:
        z_out = torch.empty_like(y_out, memory_format=torch.contiguous_format)
    hit = _checked.get(key)
    if hit is None:
        d = _experts_desc(x, (w,), ("w",), offsets, tokens, act, transposed, aligned)
        d.y_ld = _mat_of(y_out, x.dtype, d.rows, d.N, "y_out")
        if z_out is not None:
            _vec_of(z_out, x.dtype, d.rows * d.N, "z_out")
        _same_device(x, w, offsets, tokens, y_out, z_out)
        hit = _remember(key, (d, int(L.ax_matmul_experts_workspace_bytes(d))))
    d, need = hit
    _current_device(x)
    ws = _scratch(need, workspace, x.device)
    _check(L.ax_matmul_experts(d, xp, _ptr(tokens), offsets.data_ptr(), wp, y_out.data_ptr(), _ptr(z_out), *_ws_args(ws), _stream_ptr(None)))
    return y_out, z_out


def _rows_grad(out, rows, x):
    return x.new_empty((rows, x.shape[-1])) if out is None else out


def _check_weight_grad(out, like, name):
    if out is not False and _weights(out, like.dtype, name) != _weights(like, like.dtype, name):
        raise ValueError("%s must have the shape and the row pitch of its tensor" % name)


def ax_matmul_experts_backward(gy, x, w, offsets, tokens=None, z=None, act="none", transposed=False, gx_out=None, gw_out=None,
                               workspace=None, stream=None):
    """Gradients of ax_matmul_experts: (gx, gw); False skips one.  gx is that of the rows of the products, [rows,K] (with tokens,
    x's own is their sum: ax_combine without weights); z: the value before the activation."""
    if stream is not None:
        return _on_stream(ax_matmul_experts_backward, stream, gy, x, w, offsets, tokens, z, act, transposed, gx_out, gw_out, workspace)
    L = lib()
    gp, xp, wp = gy.data_ptr(), x.data_ptr(), w.data_ptr()
    aligned = (wp | xp | (gp if act == "none" else 0)) % 16 == 0
    key = ("matmul_experts_backward", act, transposed, aligned, _sig(gy), _sig(x), _sig(w), _sig(offsets), _sig(tokens), _sig(z),
           _sig(gx_out), _sig(gw_out))
    hit = _checked.get(key)
    if hit is None:
        d = _experts_desc(x, (w,), ("w",), offsets, tokens, act, transposed, aligned)
        d.y_ld = _mat_of(gy, x.dtype, d.rows, d.N, "gy")
        if z is not None:
            _vec_of(z, x.dtype, d.rows * d.N, "z")
        elif d.act:
            raise ValueError("the gradient of an activation needs z")
        if gx_out is not None and gx_out is not False:
            d.gx_ld = _mat_of(gx_out, x.dtype, d.rows, d.K, "gx_out")
        if gw_out is not None:
            _check_weight_grad(gw_out, w, "gw_out")
        _same_device(x, gy, w, offsets, tokens, z, gx_out, gw_out)
        hit = _remember(key, (d, int(L.ax_matmul_experts_backward_workspace_bytes(d))))
    d, need = hit
    _current_device(x)
    gx_out, gw_out = _rows_grad(gx_out, d.rows, x), _grad_out(gw_out, w)
    gx_out, gw_out = (None if o is False else o for o in (gx_out, gw_out))
    ws = _scratch(need, workspace, x.device)
    _check(L.ax_matmul_experts_backward(d, gp, xp, _ptr(tokens), offsets.data_ptr(), wp, _ptr(z), _ptr(gx_out), _ptr(gw_out),
                                        *_ws_args(ws), _stream_ptr(None)))
    return gx_out, gw_out


def ax_gated_experts(x, wg, wu, offsets, tokens=None, act="silu", save=False, h_out=None, g_out=None, u_out=None, workspace=None,
                     stream=None):
    """h = act(x wg_e) * (x wu_e) for rows grouped by expert, as ax_matmul_experts; wg, wu [experts,K,F].  Returns (h, g, u): both
    projections with save (or g_out and u_out), otherwise None."""
    if stream is not None:
        return _on_stream(ax_gated_experts, stream, x, wg, wu, offsets, tokens, act, save, h_out, g_out, u_out, workspace)
    L = lib()
    xp, gp, up = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    aligned = (gp | up | xp) % 16 == 0
    key = ("gated_experts", act, aligned, save, _sig(x), _sig(wg), _sig(wu), _sig(offsets), _sig(tokens), _sig(h_out), _sig(g_out), _sig(u_out))
    if h_out is None:
        h_out = x.new_empty(_rows_of(x, tokens) + (_expert_columns(wg, False),))
    if save:
        g_out, u_out = (torch.empty_like(h_out, memory_format=torch.contiguous_format) if o is None else o for o in (g_out, u_out))
    hit = _checked.get(key)
    if hit is None:
        d = _experts_desc(x, (wg, wu), ("wg", "wu"), offsets, tokens, act, False, aligned)
        d.y_ld = _mat_of(h_out, x.dtype, d.rows, d.N, "h_out")
        for t, name in ((g_out, "g_out"), (u_out, "u_out")):
            if t is not None:
                _vec_of(t, x.dtype, d.rows * d.N, name)
        _same_device(x, wg, wu, offsets, tokens, h_out, g_out, u_out)
        hit = _remember(key, (d, int(L.ax_gated_experts_workspace_bytes(d))))
    d, need = hit
    _current_device(x)
    ws = _scratch(need, workspace, x.device)
    _check(L.ax_gated_experts(d, xp, _ptr(tokens), offsets.data_ptr(), gp, up, h_out.data_ptr(), _ptr(g_out), _ptr(u_out), *_ws_args(ws),
                              _stream_ptr(None)))
    return h_out, g_out, u_out


def ax_gated_experts_backward(gh, x, wg, wu, g, u, offsets, tokens=None, act="silu", gx_out=None, gwg_out=None, gwu_out=None,
                              workspace=None, stream=None):
    """Gradients of ax_gated_experts: (gx, gwg, gwu), gx that of the rows as in ax_matmul_experts_backward; gx_out False, or gwg_out
    and gwu_out False, skips them."""
    if stream is not None:
        return _on_stream(ax_gated_experts_backward, stream, gh, x, wg, wu, g, u, offsets, tokens, act, gx_out, gwg_out, gwu_out, workspace)
    L = lib()
    xp, gp, up = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    aligned = (gp | up | xp) % 16 == 0
    key = ("gated_experts_backward", act, aligned, _sig(gh), _sig(x), _sig(wg), _sig(wu), _sig(g), _sig(u), _sig(offsets), _sig(tokens),
           _sig(gx_out), _sig(gwg_out), _sig(gwu_out))
    hit = _checked.get(key)
    if hit is None:
        d = _experts_desc(x, (wg, wu), ("wg", "wu"), offsets, tokens, act, False, aligned)
        d.y_ld = _mat_of(gh, x.dtype, d.rows, d.N, "gh")
        _vec_of(g, x.dtype, d.rows * d.N, "g")
        _vec_of(u, x.dtype, d.rows * d.N, "u")
        if gx_out is not None and gx_out is not False:
            d.gx_ld = _mat_of(gx_out, x.dtype, d.rows, d.K, "gx_out")
        for o, like, name in ((gwg_out, wg, "gwg_out"), (gwu_out, wu, "gwu_out")):
            if o is not None:
                _check_weight_grad(o, like, name)
        _same_device(x, gh, wg, wu, g, u, offsets, tokens, gx_out, gwg_out, gwu_out)
        hit = _remember(key, (d, int(L.ax_gated_experts_backward_workspace_bytes(d))))
    d, need = hit
    _current_device(x)
    gx_out, gwg_out, gwu_out = _rows_grad(gx_out, d.rows, x), _grad_out(gwg_out, wg), _grad_out(gwu_out, wu)
    gx_out, gwg_out, gwu_out = (None if o is False else o for o in (gx_out, gwg_out, gwu_out))
    ws = _scratch(need, workspace, x.device)
    _check(L.ax_gated_experts_backward(d, gh.data_ptr(), xp, _ptr(tokens), offsets.data_ptr(), gp, up, g.data_ptr(), u.data_ptr(),
                                       _ptr(gx_out), _ptr(gwg_out), _ptr(gwu_out), *_ws_args(ws), _stream_ptr(None)))
    return gx_out, gwg_out, gwu_out


def _combine_desc(h, rows, weights, y, name) -> ax_combine_desc_t:
    """y: what has a row for every token."""
    n, cols, ld = _mat(h, h.dtype, "h")
    _whole(rows, -1, "rows")
    if rows.dim() < 2:
        raise ValueError("rows must be [tokens, k]")
    k = rows.shape[-1]
    T = math.prod(rows.shape[:-1])
    if weights is not None:
        _vec_of(weights, torch.float32, T * k, "weights")
    y_ld = _mat_of(y, h.dtype, T, cols, name)
    return ax_combine_desc_t(T, n, cols, ld, cols, y_ld, cols, k, _float_dtype(h, "h"))


def ax_combine(h, rows, weights=None, residual=None, y_out=None, stream=None):
    """y[t] = residual[t] + sum over j of weights[t,j] * h[rows[t,j]]: the tokens' sums of their experts' rows.  rows [tokens,k] int32
    as ax_route returned them (one outside h is left out), weights [tokens,k] float32 (one each without them).  y_out may be the residual
    itself."""
    if stream is not None:
        return _on_stream(ax_combine, stream, h, rows, weights, residual, y_out)
    key = ("combine", _sig(h), _sig(rows), _sig(weights), _sig(residual), _sig(y_out))
    if y_out is None:
        y_out = h.new_empty(rows.shape[:-1] + h.shape[-1:])
    d = _checked.get(key)
    if d is None:
        d = _combine_desc(h, rows, weights, y_out, "y_out")
        if residual is not None:
            d.residual_ld = _mat_of(residual, h.dtype, d.tokens, d.cols, "residual")
        _same_device(h, rows, weights, residual, y_out)
        _remember(key, d)
    _current_device(h)
    _check(lib().ax_combine(d, h.data_ptr(), rows.data_ptr(), _ptr(weights), _ptr(residual), y_out.data_ptr(), _stream_ptr(None)))
    return y_out


def ax_combine_backward(gy, h, rows, weights=None, gh_out=None, gweights_out=None, stream=None):
    """Gradients of ax_combine: (gh, gweights); False skips one.  Rows of gh that no choice names are not written; the residual's
    gradient is gy."""
    if stream is not None:
        return _on_stream(ax_combine_backward, stream, gy, h, rows, weights, gh_out, gweights_out)
    key = ("combine_backward", _sig(gy), _sig(h), _sig(rows), _sig(weights), _sig(gh_out), _sig(gweights_out))
    if gh_out is None:
        gh_out = torch.empty_like(h, memory_format=torch.contiguous_format)
    if gweights_out is None:
        gweights_out = rows.new_empty(rows.shape, dtype=torch.float32)
    d = _checked.get(key)
    if d is None:
        d = _combine_desc(h, rows, weights, gy, "gy")
        if gh_out is not False:
            d.gh_ld = _mat_of(gh_out, h.dtype, d.h_rows, d.cols, "gh_out")
        if gweights_out is not False:
            _vec_of(gweights_out, torch.float32, d.tokens * d.k, "gweights_out")
        _same_device(h, gy, rows, weights, gh_out, gweights_out)
        _remember(key, d)
    _current_device(h)
    gh_out, gweights_out = (None if o is False else o for o in (gh_out, gweights_out))
    _check(lib().ax_combine_backward(d, gy.data_ptr(), h.data_ptr(), rows.data_ptr(), _ptr(weights), _ptr(gh_out), _ptr(gweights_out),
                                     _stream_ptr(None)))
    return gh_out, gweights_out


# ---- weights of 4 bits -------------------------------------------------------------------------------------------------


class AxQ4:
    """Weights of 4 bits with a scale for every group of a row, in the library's layout: made once by ax_quantize_q4 or
    ax_pack_q4, read by ax_matmul_q4 and ax_gated_q4.  rows and cols are those of one matrix (outputs and inputs); experts is
    None for a single one."""

    def __init__(self, rows, cols, group, experts, device):
        L = lib()
        self.rows, self.cols, self.group, self.experts = int(rows), int(cols), int(group), experts
        if self.group not in (32, 64, 128):
            raise ValueError("group must be 32, 64 or 128")
        n = (experts or 1, self.rows, self.cols)
        c, s = int(L.ax_q4_codes_bytes(*n)), int(L.ax_q4_scales_bytes(*n, self.group))
        if not c or not s:
            _check(-2)
        self.codes = torch.empty(c, dtype=torch.uint8, device=device)
        self.scales = torch.empty(s // 2, dtype=torch.bfloat16, device=device)

    @property
    def shape(self):
        """[outputs, inputs], or [experts, outputs, inputs]."""
        return ((self.experts,) if self.experts else ()) + (self.rows, self.cols)

    def _sizes(self):
        return self.experts or 1, self.rows, self.cols, self.group

    def values(self, stream=None):
        """The weights that the codes and scales stand for, float32."""
        return _q4_values(self) if stream is None else _on_stream(_q4_values, stream, self)


def _q4_values(w):
    _current_device(w.codes)
    out = torch.empty(w.shape, dtype=torch.float32, device=w.codes.device)
    _check(lib().ax_q4_values(w.codes.data_ptr(), w.scales.data_ptr(), *w._sizes(), out.data_ptr(), _stream_ptr(None)))
    return out


def ax_quantize_q4(w, group=128, stream=None) -> AxQ4:
    """Float weights [outputs, inputs], or [experts, outputs, inputs], in 4 bits: of every `group` inputs of a row the scale is the
    largest |w| / 7 (bfloat16), the codes w / scale rounded, -8 .. 7."""
    if stream is not None:
        return _on_stream(ax_quantize_q4, stream, w, group)
    dt = _float_dtype(w, "w")
    if w.dim() == 3:
        E, r, c, ld = _weights(w, w.dtype, "w")
    else:
        E, (r, c, ld) = None, _mat(w, w.dtype, "w")
        if w.dim() != 2:
            raise ValueError("w must be [outputs, inputs] or [experts, outputs, inputs]")
    _current_device(w)
    q = AxQ4(r, c, group, E, w.device)
    _check(lib().ax_quantize_q4(w.data_ptr(), dt, ld, *q._sizes(), q.codes.data_ptr(), q.scales.data_ptr(), _stream_ptr(None)))
    return q


def ax_pack_q4(codes, scales, group=128, stream=None) -> AxQ4:
    """Codes and scales from elsewhere: codes int8 [outputs, inputs] or [experts, outputs, inputs], -8 .. 7; scales bfloat16 of the
    same shape with one for every `group` inputs."""
    if stream is not None:
        return _on_stream(ax_pack_q4, stream, codes, scales, group)
    _dev(codes, torch.int8, "codes")
    _dev(scales, torch.bfloat16, "scales")
    if codes.dim() not in (2, 3) or group not in (32, 64, 128):
        raise ValueError("codes must be [outputs, inputs] or [experts, outputs, inputs], group 32, 64 or 128")
    if scales.shape != codes.shape[:-1] + (-(-codes.shape[-1] // group),):
        raise ValueError("scales must have one for every group of a row")
    _same_device(codes, scales)
    _current_device(codes)
    q = AxQ4(codes.shape[-2], codes.shape[-1], group, codes.shape[0] if codes.dim() == 3 else None, codes.device)
    _check(lib().ax_pack_q4(codes.data_ptr(), scales.data_ptr(), *q._sizes(), q.codes.data_ptr(), q.scales.data_ptr(), _stream_ptr(None)))
    return q


def _q4_desc(x, weights, offsets, tokens, act, aligned) -> ax_q4_desc_t:
    w = weights[0]
    n, K, x_ld = _mat(x, x.dtype, "x")
    for other in weights:
        if not isinstance(other, AxQ4):
            raise TypeError("weights must be AxQ4")
        if other.shape != w.shape or other.group != w.group:
            raise ValueError("both weights must have one shape and one group")
    if K != w.cols:
        raise ValueError("x must be [rows, %d] for these weights" % w.cols)
    E = w.experts or 1
    if offsets is not None:
        _whole(offsets, E + 1, "offsets")
    elif E > 1:
        raise ValueError("weights of several experts need offsets")
    if tokens is not None:
        _whole(tokens, -1, "tokens")
    return ax_q4_desc_t(n if tokens is None else tokens.numel(), n, w.rows, K, x_ld, w.rows, w.rows, E, w.group, _float_dtype(x, "x"),
                        _act_code(act), int(tokens is not None), int(not aligned))


def _q4_sig(w):
    return (w.experts, w.rows, w.cols, w.group, w.codes.device) if isinstance(w, AxQ4) else None


def ax_matmul_q4(x, w, bias=None, residual=None, act="none", offsets=None, tokens=None, y_out=None, workspace=None, stream=None):
    """y = act(x w^T + bias) + residual with weights of 4 bits (AxQ4).  x: [rows, inputs], float32 or bfloat16, as bias, residual and
    y are.  Weights of several experts: rows grouped by them, as in ax_matmul_experts."""
    if stream is not None:
        return _on_stream(ax_matmul_q4, stream, x, w, bias, residual, act, offsets, tokens, y_out, workspace)
    L = lib()
    xp = x.data_ptr()
    aligned = xp % 16 == 0
    key = ("matmul_q4", act, aligned, _sig(x), _q4_sig(w), _sig(bias), _sig(residual), _sig(offsets), _sig(tokens), _sig(y_out))
    hit = _checked.get(key)
    if hit is None:
        d = _q4_desc(x, (w,), offsets, tokens, act, aligned)
        if bias is not None:
            _vec_of(bias, x.dtype, d.N, "bias")
        if residual is not None:
            d.residual_ld = _mat_of(residual, x.dtype, d.rows, d.N, "residual")
        if y_out is not None:
            d.y_ld = _mat_of(y_out, x.dtype, d.rows, d.N, "y_out")
        _same_device(x, w.codes, bias, residual, offsets, tokens, y_out)
        hit = _remember(key, (d, int(L.ax_matmul_q4_workspace_bytes(d))))
    d, need = hit
    _current_device(x)
    if y_out is None:
        y_out = x.new_empty(_rows_of(x, tokens) + (w.rows,))
    ws = _scratch(need, workspace, x.device)
    _check(L.ax_matmul_q4(d, xp, _ptr(tokens), _ptr(offsets), w.codes.data_ptr(), w.scales.data_ptr(), _ptr(bias), _ptr(residual),
                          y_out.data_ptr(), *_ws_args(ws), _stream_ptr(None)))
    return y_out


def ax_gated_q4(x, wg, wu, act="silu", offsets=None, tokens=None, h_out=None, workspace=None, stream=None):
    """h = act(x wg^T) * (x wu^T) with weights of 4 bits (AxQ4), as ax_matmul_q4."""
    if stream is not None:
        return _on_stream(ax_gated_q4, stream, x, wg, wu, act, offsets, tokens, h_out, workspace)
    L = lib()
    xp = x.data_ptr()
    aligned = xp % 16 == 0
    key = ("gated_q4", act, aligned, _sig(x), _q4_sig(wg), _q4_sig(wu), _sig(offsets), _sig(tokens), _sig(h_out))
    hit = _checked.get(key)
    if hit is None:
        d = _q4_desc(x, (wg, wu), offsets, tokens, act, aligned)
        if h_out is not None:
            d.y_ld = _mat_of(h_out, x.dtype, d.rows, d.N, "h_out")
        _same_device(x, wg.codes, wu.codes, offsets, tokens, h_out)
        hit = _remember(key, (d, int(L.ax_gated_q4_workspace_bytes(d))))
    d, need = hit
    _current_device(x)
    if h_out is None:
        h_out = x.new_empty(_rows_of(x, tokens) + (wg.rows,))
    ws = _scratch(need, workspace, x.device)
    _check(L.ax_gated_q4(d, xp, _ptr(tokens), _ptr(offsets), wg.codes.data_ptr(), wg.scales.data_ptr(), wu.codes.data_ptr(),
                         wu.scales.data_ptr(), h_out.data_ptr(), *_ws_args(ws), _stream_ptr(None)))
    return h_out


class AxAdamW:
    """The AdamW step over a list of tensors (ax_adamw), with the list checked and marshalled once.

    params, grads: lists of contiguous tensors, each list of one type (float32 or bfloat16).  States: None, None allocates
    them (bits = 32 or 8); otherwise lists m and v, float32, or int8 and uint8 codes together with their scales m_scales and
    v_scales (ceil(n / 256) float32 a tensor).  copies: bfloat16 tensors that receive the updated parameters as well.
    The tensors are held, and their addresses used, until the object is dropped; set_grads exchanges the gradients."""

    def __init__(self, params, grads, m=None, v=None, m_scales=None, v_scales=None, copies=None, bits=32):
        self._streams = set()  # that steps were enqueued on
        self.params, self.copies = list(params), None if copies is None else list(copies)
        n = len(self.params)
        if not n:
            raise ValueError("no parameters")
        dev, pdt = self.params[0].device, self.params[0].dtype
        sizes = [t.numel() for t in self.params]
        blocks = [-(-k // AX_STATE_BLOCK) for k in sizes]
        if (m is None) != (v is None) or (m_scales is None) != (v_scales is None):
            raise ValueError("both states or neither, both lists of scales or neither")
        if m is None:
            if bits not in (32, 8) or m_scales is not None:
                raise ValueError("bits must be 32 or 8, and scales come with their codes")
            make = lambda shapes, dt: [torch.zeros(s, dtype=dt, device=dev) for s in shapes]  # noqa: E731
            shapes = [t.shape for t in self.params]
            if bits == 8:
                m, v = make(shapes, torch.int8), make(shapes, torch.uint8)
                m_scales, v_scales = make(blocks, torch.float32), make(blocks, torch.float32)
            else:
                m, v = make(shapes, torch.float32), make(shapes, torch.float32)
        self.bits = 32 if m_scales is None else 8
        self.m, self.v = list(m), list(v)
        self.m_scales, self.v_scales = (None if s is None else list(s) for s in (m_scales, v_scales))
        mt, vt = (torch.int8, torch.uint8) if self.bits == 8 else (torch.float32, torch.float32)
        for what, ts, dt, counts in (("params", self.params, pdt, sizes), ("m", self.m, mt, sizes), ("v", self.v, vt, sizes),
                                     ("m_scales", self.m_scales, torch.float32, blocks),
                                     ("v_scales", self.v_scales, torch.float32, blocks),
                                     ("copies", self.copies, torch.bfloat16, sizes)):
            if ts is None:
                continue
            if len(ts) != n:
                raise ValueError("%s must hold %d tensors" % (what, n))
            for t, k in zip(ts, counts):
                _vec_of(t, dt, k, what)
        self._d = ax_adamw_desc_t()
        self._d.p_dtype, self._d.state_bits = _float_dtype(self.params[0], "params"), self.bits
        self._t = (ax_adamw_tensor_t * n)()
        for i, e in enumerate(self._t):
            e.p, e.m, e.v, e.n = self.params[i].data_ptr(), self.m[i].data_ptr(), self.v[i].data_ptr(), sizes[i]
            if self.bits == 8:
                e.m_scale, e.v_scale = self.m_scales[i].data_ptr(), self.v_scales[i].data_ptr()
            if self.copies is not None:
                e.copy = self.copies[i].data_ptr()
        # states(): the tensors' places in one buffer, whole lines apart
        self._places, self._whole = [], 0
        for t, k in zip(self.params, sizes):
            self._places.append((t.shape, t.stride(), self._whole))
            self._whole += -(-k // 64) * 64
        self.set_grads(grads)

    def _held(self):
        return self.params, self.m, self.v, self.m_scales or (), self.v_scales or (), self.copies or ()

    def __del__(self):
        # (tied here, not in every step: hundreds of tensors, and until now nobody could drop the last of any)
        try:
            for s in self._streams:
                for t in _tensors_of(self._held()):
                    t.record_stream(s)
        except Exception:  # interpreter shutdown: the module's globals may be gone
            pass

    def set_grads(self, grads):
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError("grads must hold %d tensors" % len(self.params))
        for t, p in zip(grads, self.params):
            _vec_of(t, grads[0].dtype, p.numel(), "grads")
        self._d.g_dtype = _float_dtype(grads[0], "grads")
        for e, t in zip(self._t, grads):
            e.g = t.data_ptr()
        self.grads = grads

    def step(self, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=None, stream=None):
        """One step, the step-th (from 1).  grad_scale: None, or a float32 CUDA tensor of one element that multiplies the
        gradients (what clipping by a norm that was computed on the device gives).  lr and the factors of the step-th step are
        the launch's arguments: a graph that holds it repeats that step."""
        d = self._d
        d.lr, d.beta1, d.beta2, d.eps, d.weight_decay, d.step = lr, beta1, beta2, eps, weight_decay, int(step)
        if grad_scale is not None:
            _vec_of(grad_scale, torch.float32, 1, "grad_scale")
        d.grad_scale = _ptr(grad_scale)
        if stream is not None:  # (the gradients may be exchanged, and the factor dropped, before the step has run)
            for t in self.grads if grad_scale is None else self.grads + [grad_scale]:
                t.record_stream(stream)
            self._streams.add(stream)
        _check(lib().ax_adamw(d, self._t, len(self._t), _stream_ptr(stream)))

    def states(self, stream=None):
        """(m, v) as lists of float32 tensors: the values that 8-bit states stand for (views of one new buffer for m and one
        for v), or the 32-bit states themselves."""
        if self.bits == 32:
            return self.m, self.v
        bufs = self._states() if stream is None else _on_stream(self._states, stream, held=self._held())
        m, v = ([b.as_strided(*place) for place in self._places] for b in bufs)
        return m, v

    def _states(self):
        bufs = tuple(torch.empty(self._whole, dtype=torch.float32, device=self.params[0].device) for _ in range(2))
        ptrs = [(ctypes.c_void_p * len(self._places))(*[b.data_ptr() + 4 * at for _, _, at in self._places]) for b in bufs]
        _check(lib().ax_adamw_states(self._t, len(self._t), ptrs[0], ptrs[1], _stream_ptr(None)))
        return bufs


def ax_probe_lds_gather(width_bytes: int, pattern: int, table_bytes: int, threads: int = 1024, iters: int = 2000,
                        stream=None) -> dict:
    wr, cy, sec = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    wgs = ctypes.c_int()
    rc = lib().ax_probe_lds_gather(width_bytes, pattern, table_bytes, threads, iters, ctypes.byref(wr),
                                   ctypes.byref(cy), ctypes.byref(sec), ctypes.byref(wgs),
                                   ctypes.c_void_p(_stream_ptr(stream)))
    _check(rc)
    return {"wave_reads": wr.value, "cycles": cy.value, "seconds": sec.value, "workgroups": wgs.value}


def ax_probe_mac(mode: int, pattern: int = 1, iters: int = 200, wgs_per_cu: int = 1, stream=None) -> dict:
    ops, sec = ctypes.c_double(), ctypes.c_double()
    _check(lib().ax_probe_mac(mode, pattern, iters, wgs_per_cu, ctypes.byref(ops), ctypes.byref(sec),
                              ctypes.c_void_p(_stream_ptr(stream))))
    return {"ops": ops.value, "seconds": sec.value, "ops_per_s": ops.value / sec.value}


PRODUCTS = ("matmul", "matmul_q8", "gated", "gated_q8", "matmul_gx", "matmul_gw", "gated_gx", "gated_gw")


def ax_probe_product_plan(product: str, M: int, K: int, N: int, dtype=torch.bfloat16, out_dtype=None, transposed=False) -> dict:
    """Which kernel a product of contiguous aligned matrices runs ("tiles", "few", "outer"), its tile and the slices of its
    contraction.  M, K, N: of the call, also where the product is one of its gradients (matmul_gx, ...)."""
    q8 = product.endswith("q8")
    out_dtype = (torch.bfloat16 if q8 else dtype) if out_dtype is None else out_dtype
    transposed = transposed or q8
    d = ax_matmul_desc_t(M, N, K, K, K if transposed else N, N, N, AX_BF16 if q8 else _DT[dtype], _DT[out_dtype], 0, int(transposed), 0)
    out = [ctypes.c_int(0) for _ in range(4)]
    _check(lib().ax_probe_product_plan(d, PRODUCTS.index(product), *[ctypes.byref(o) for o in out]))
    k, rows, cols, slices = [o.value for o in out]
    return {"kernel": ("tiles", "few", "outer")[k], "tile": (rows, cols), "slices": slices}


def _plan(f, results, desc, *args) -> list:
    out = [ctypes.c_int(0) for _ in range(results)]
    _check(f(ctypes.byref(desc), *args, *[ctypes.byref(o) for o in out]))
    return [o.value for o in out]


def ax_probe_experts_plan(product: str, rows: int, experts: int, K: int, N: int, dtype=torch.bfloat16, transposed=False, x_rows=None,
                          unaligned=False) -> dict:
    """Which kernel a product grouped by expert runs ("tiles", "few"), its tile, its workgroups a compute unit, and whether it looks up the
    rows of an index (of x_rows rows) itself.  Contiguous operands."""
    d = ax_experts_desc_t(rows, rows if x_rows is None else x_rows, N, K, K, K if transposed else N, N, K, experts, _DT[dtype], 0,
                          int(transposed), int(x_rows is not None), int(unaligned))
    k, r, c, per_cu, found = _plan(lib().ax_probe_experts_plan, 5, d, PRODUCTS.index(product))
    return {"kernel": ("tiles", "few")[k], "tile": (r, c), "per_cu": per_cu, "found": bool(found)}


def ax_probe_q4_plan(gated: bool, rows: int, experts: int, K: int, N: int, group=128, dtype=torch.bfloat16, x_rows=None) -> dict:
    """Which kernel a product with 4-bit weights runs ("few", "tiles", "written"), rows and columns of its workgroups, and of "few" their
    waves.  Contiguous aligned operands."""
    d = ax_q4_desc_t(rows, rows if x_rows is None else x_rows, N, K, K, N, N, experts, group, _DT[dtype], 0, int(x_rows is not None), 0)
    k, r, c, waves = _plan(lib().ax_probe_q4_plan, 4, d, int(gated))
    return {"kernel": ("few", "tiles", "written")[k], "tile": (r, c), "waves": waves}


def ax_probe_copy(dst: torch.Tensor, src: torch.Tensor, stream=None) -> None:
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("size mismatch")
    _check(lib().ax_probe_copy(_ptr(dst), _ptr(src), nbytes, ctypes.c_void_p(_stream_ptr(stream))))


def lut_to_device(lut_np, device="cuda") -> torch.Tensor:
    """uint16 (or, for signed multipliers, int16) numpy table -> device tensor holding the same
    bit patterns."""
    import numpy as np

    a = np.ascontiguousarray(lut_np)
    if a.dtype != np.int16:
        a = np.ascontiguousarray(a, dtype=np.uint16).view(np.int16)
    return torch.from_numpy(a.reshape(-1).copy()).to(device)
