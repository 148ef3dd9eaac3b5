"""Thin Python binding of libdstd (include/dstd.h): argument marshalling only.

Every function takes CUDA float32 torch tensors (int32 for labels, any dtype
for opaque byte buffers), checks shapes and dtypes, and calls the C entry
point of the same name on the given stream (default: torch's current
stream). All arithmetic happens in the library's kernels; there is no
fallback of any kind. A missing library raises at load time.
"""

import ctypes
import os

from .build import LIB_PATH

MATH = {"f32": 0, "x3": 1, "bf16": 2}

ERRORS = {0: "ok", -1: "invalid argument", -2: "unsupported size or mode", -3: "workspace too small",
          -4: "CUDA call or kernel launch failed", -5: "a bounded device-side wait expired",
          -6: "no usable sm_103 device"}

EXPORTS = ("dstd_dense_saved_bytes", "dstd_dense_workspace_bytes", "dstd_binning", "dstd_dense_what",
           "dstd_scan_solve", "dstd_dense_fwd", "dstd_dense_fwd_ce", "dstd_dense_bwd", "dstd_ce_loss", "dstd_sum_t_loss",
           "dstd_adamw", "dstd_adamw_multi", "dstd_device_status", "dstd_error_string", "dstd_version", "dstd_timing_enable",
           "dstd_timing_read", "dstd_timing_collect", "dstd_set_pair_policy", "dstd_conv_set_chunk_images", "dstd_conv_set_operand_policy", "dstd_kernel_kind_count", "dstd_kernel_kind_name", "dstd_selftest_wait_timeout",
           "dstd_dense_fwd_noalloc", "dstd_conv_workspace_bytes", "dstd_conv_fwd", "dstd_conv_bwd",
           "dstd_exact_workspace_bytes", "dstd_exact_fwd", "dstd_exact_bwd", "dstd_concat_channels", "dstd_split_channels",
           "dstd_ms_saved_bytes", "dstd_ms_workspace_bytes", "dstd_dense_fwd_ms", "dstd_dense_bwd_ms",
           "dstd_quantize_rows", "dstd_int8_matmul_workspace_bytes", "dstd_int8_matmul_aligned_workspace_bytes",
           "dstd_int8_matmul", "dstd_dense_q8_workspace_bytes",
           "dstd_dense_fwd_q8", "dstd_grad_norm_workspace_bytes", "dstd_grad_norm", "dstd_clip_grads", "dstd_adamw_clip")


class DstdError(RuntimeError):
    def __init__(self, code, where):
        super().__init__(f"{where}: {ERRORS.get(code, 'unknown error')} (code {code})")
        self.code = code


class Params(ctypes.Structure):
    """dstd_params of include/dstd.h."""
    _fields_ = [("tau_m", ctypes.c_float), ("tau_s", ctypes.c_float), ("v_th", ctypes.c_float),
                ("t_first", ctypes.c_float), ("t_end", ctypes.c_float), ("M", ctypes.c_int32),
                ("t_offset", ctypes.c_float), ("t_head", ctypes.c_float), ("t_tail", ctypes.c_float),
                ("gamma_head", ctypes.c_float), ("gamma_tail", ctypes.c_float), ("gamma_q", ctypes.c_float),
                ("penalty_norm", ctypes.c_float)]


def params(layer, penalty_norm=0.0):
    """dstd_params from a layer dict (see configs.py)."""
    return Params(float(layer["tau_v"]), float(layer["tau_I"]), float(layer["v_th"]), float(layer["t_first"]),
                  float(layer["t_end"]), int(layer["M"]), float(layer.get("t_offset", 0.0)),
                  float(layer.get("t_head_l", 0.0)), float(layer.get("t_tail_l", 0.0)),
                  float(layer.get("gamma_head", 0.0)), float(layer.get("gamma_tail", 0.0)),
                  float(layer.get("gamma_q", 0.0)), float(penalty_norm))


_LIB = None
_P = ctypes.c_void_p
_I = ctypes.c_int
_F = ctypes.c_float
_D = ctypes.c_double
_SZ = ctypes.c_size_t
_I64 = ctypes.c_int64
_PP = ctypes.POINTER(Params)


def load(path=None):
    """Load libdstd.so (built by ``build.build()``); raises if it is missing."""
    global _LIB
    if _LIB is not None:
        return _LIB
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"libdstd.so not found at {p}: build it first (python -m paper_2607_14672_gb300.build)")
    lib = ctypes.CDLL(p)
    sig = {
        "dstd_dense_saved_bytes": (_SZ, [_I, _I]),
        "dstd_dense_workspace_bytes": (_SZ, [_I, _I, _I, _PP, _I]),
        "dstd_binning": (_I, [_P, _I, _I, _PP, _P, _P, _P]),
        "dstd_dense_what": (_I, [_P, _P, _I, _I, _I, _PP, _I, _P, _P, _SZ, _P]),
        "dstd_scan_solve": (_I, [_P, _I, _I, _PP, _P, _P, _P, _P, _P]),
        "dstd_dense_fwd": (_I, [_P, _P, _I, _I, _I, _PP, _I, _P, _P, _P, _P, _SZ, _P]),
        "dstd_dense_fwd_ce": (_I, [_P, _P, _I, _I, _I, _PP, _I, _P, _P, _P, _P, _SZ, _P, _F, _F, _P, _P, _P]),
        "dstd_dense_bwd": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _PP, _I, _P, _P, _P, _SZ, _P]),
        "dstd_ce_loss": (_I, [_P, _P, _I, _I, _F, _F, _P, _P, _P]),
        "dstd_sum_t_loss": (_I, [_P, _I64, _P, _P, _P]),
        "dstd_adamw": (_I, [_P, _P, _P, _P, _I64, _F, _F, _F, _F, _F, _I, _P]),
        "dstd_adamw_multi": (_I, [_I, _P, _P, _P, _P, _P, _F, _F, _F, _F, _F, _P, _P, _P]),
        "dstd_device_status": (_I, [_I]),
        "dstd_error_string": (ctypes.c_char_p, [_I]),
        "dstd_version": (_I, []),
        "dstd_timing_enable": (_I, [_I]),
        "dstd_timing_read": (_I, [_I, ctypes.POINTER(_F), ctypes.POINTER(_I64)]),
        "dstd_timing_collect": (_I, []),
        "dstd_set_pair_policy": (_I, [_I]),
        "dstd_conv_set_chunk_images": (_I, [_I]),
        "dstd_conv_set_operand_policy": (_I, [_I]),
        "dstd_exact_workspace_bytes": (_SZ, [_I, _I, _I]),
        "dstd_exact_fwd": (_I, [_P, _P, _I, _I, _I, _PP, _P, _P, _SZ, _P]),
        "dstd_exact_bwd": (_I, [_P, _P, _P, _P, _I, _I, _I, _PP, _P, _P, _P, _SZ, _P]),
        "dstd_kernel_kind_count": (_I, []),
        "dstd_kernel_kind_name": (ctypes.c_char_p, [_I]),
        "dstd_selftest_wait_timeout": (_I, [ctypes.c_uint32, _P]),
        "dstd_dense_fwd_noalloc": (_I, [_P, _P, _I, _I, _I, _PP, _I, _P, _P, _P, _P]),
        "dstd_conv_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I, _I, _I, _PP, _I]),
        "dstd_conv_fwd": (_I, [_P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _PP, _I, _P, _P, _P, _P, _SZ, _P]),
        "dstd_conv_bwd": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _PP, _I, _P, _P, _P, _SZ, _P]),
        "dstd_concat_channels": (_I, [_P, _I, _F, _P, _I, _I64, _P, _P]),
        "dstd_ms_saved_bytes": (_SZ, [_I, _I, _I]),
        "dstd_ms_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _PP, _I]),
        "dstd_dense_fwd_ms": (_I, [_P, _P, _I, _I, _I, _I, _I, _PP, _I, _P, _P, _P, _SZ, _P]),
        "dstd_dense_bwd_ms": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _PP, _I, _P, _P, _P, _SZ, _P]),
        "dstd_quantize_rows": (_I, [_P, _I, _I, _I, _I64, _P, _I64, _P, _P, _I64, _P]),
        "dstd_int8_matmul_workspace_bytes": (_SZ, [_I, _I, _I]),
        "dstd_int8_matmul_aligned_workspace_bytes": (_SZ, [_I, _I, _I]),
        "dstd_int8_matmul": (_I, [_P, _I64, _P, _P, _I64, _P, _I, _I, _I, _P, _I, _I64, _P, _SZ, _P]),
        "dstd_dense_q8_workspace_bytes": (_SZ, [_I, _I, _I, _PP]),
        "dstd_dense_fwd_q8": (_I, [_P, _P, _P, _I, _I, _I, _PP, _P, _P, _P, _P, _SZ, _P]),
        "dstd_grad_norm_workspace_bytes": (_SZ, [_I, _P]),
        "dstd_grad_norm": (_I, [_I, _P, _P, _P, _P, _P, _P, _SZ, _P]),
        "dstd_clip_grads": (_I, [_I, _P, _P, _P, _P, _D, _P, _P, _SZ, _P]),
        "dstd_adamw_clip": (_I, [_I, _P, _P, _P, _P, _P, _P, _D, _D, _D, _D, _D, _D, _P, _P, _P, _P, _SZ, _P]),
        "dstd_split_channels": (_I, [_P, _I, _I, _I64, _P, _I, _P, _I, _P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _LIB = lib
    return lib


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    import torch
    return torch.cuda.current_stream().cuda_stream


def _check(code, where):
    if code != 0:
        raise DstdError(code, where)


def _f32(x, name, shape=None):
    import torch
    if x.dtype != torch.float32 or not x.is_cuda or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA float32 tensor")
    if shape is not None and tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(x.shape)}, expected {tuple(shape)}")


def version():
    return load().dstd_version()


def error_string(code):
    return load().dstd_error_string(code).decode()


def dense_saved_bytes(B, N_out):
    return load().dstd_dense_saved_bytes(B, N_out)


def dense_workspace_bytes(B, N_in, N_out, p, math_mode):
    return load().dstd_dense_workspace_bytes(B, N_in, N_out, ctypes.byref(p), MATH[math_mode])


def binning(t_in, p, s, ds=None, stream=None):
    B, N = t_in.shape
    _f32(t_in, "t_in")
    _f32(s, "s", (B, p.M, N))
    if ds is not None:
        _f32(ds, "ds", (B, p.M, N))
    _check(load().dstd_binning(_ptr(t_in), B, N, ctypes.byref(p), _ptr(s), _ptr(ds), _stream(stream)),
           "dstd_binning")


def dense_what(t_in, W, p, math_mode, what, workspace, stream=None):
    B, N_in = t_in.shape
    N_out = W.shape[0]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(what, "what", (B, N_out, p.M))
    _check(load().dstd_dense_what(_ptr(t_in), _ptr(W), B, N_in, N_out, ctypes.byref(p), MATH[math_mode],
                                  _ptr(what), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _stream(stream)), "dstd_dense_what")


def scan_solve(what, p, w_rowsum, t_out, saved=None, penalty=None, stream=None):
    B, N_out, M = what.shape
    _f32(what, "what")
    _f32(t_out, "t_out", (B, N_out))
    _check(load().dstd_scan_solve(_ptr(what), B, N_out, ctypes.byref(p), _ptr(w_rowsum), _ptr(t_out), _ptr(saved),
                                  _ptr(penalty), _stream(stream)), "dstd_scan_solve")


def dense_fwd(t_in, W, p, math_mode, t_out, saved, penalty, workspace, stream=None):
    B, N_in = t_in.shape
    N_out = W.shape[0]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(t_out, "t_out", (B, N_out))
    _check(load().dstd_dense_fwd(_ptr(t_in), _ptr(W), B, N_in, N_out, ctypes.byref(p), MATH[math_mode], _ptr(t_out),
                                 _ptr(saved), _ptr(penalty), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "dstd_dense_fwd")


def dense_fwd_ce(t_in, W, p, math_mode, t_out, saved, penalty, workspace, labels, tau_soft, t_silent, loss,
                 g_t_out, stream=None):
    """dense_fwd of the output layer, then the CE loss of its spike times
    (fused into one kernel on the few-output path). loss: float32[2] device
    tensor, loss[1] zero before the first call (left zero)."""
    B, N_in = t_in.shape
    N_out = W.shape[0]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(t_out, "t_out", (B, N_out))
    _f32(g_t_out, "g_t_out", (B, N_out))
    if loss.numel() < 2:
        raise ValueError("dense_fwd_ce: loss must hold 2 floats (value, scratch)")
    _check(load().dstd_dense_fwd_ce(_ptr(t_in), _ptr(W), B, N_in, N_out, ctypes.byref(p), MATH[math_mode],
                                    _ptr(t_out), _ptr(saved), _ptr(penalty), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _ptr(labels), float(tau_soft),
                                    float(t_silent), _ptr(loss), _ptr(g_t_out), _stream(stream)), "dstd_dense_fwd_ce")


def dense_fwd_noalloc(t_in, W, p, math_mode, t_out, saved, penalty=None, stream=None):
    """dstd_dense_fwd without a workspace: for callers that cannot allocate
    device memory; scratch is the library's fixed 64 MiB device array, shared
    by every call (do not overlap calls on the GPU)."""
    B, N_in = t_in.shape
    N_out = W.shape[0]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(t_out, "t_out", (B, N_out))
    _check(load().dstd_dense_fwd_noalloc(_ptr(t_in), _ptr(W), B, N_in, N_out, ctypes.byref(p), MATH[math_mode],
                                         _ptr(t_out), _ptr(saved), _ptr(penalty), _stream(stream)),
           "dstd_dense_fwd_noalloc")


def dense_bwd(t_in, W, t_out, saved, g_t_out, p, math_mode, g_t_in, g_W, workspace, stream=None):
    B, N_in = t_in.shape
    N_out = W.shape[0]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(g_W, "g_W", (N_out, N_in))
    if g_t_in is not None:
        _f32(g_t_in, "g_t_in", (B, N_in))
    _check(load().dstd_dense_bwd(_ptr(t_in), _ptr(W), _ptr(t_out), _ptr(saved), _ptr(g_t_out), B, N_in, N_out,
                                 ctypes.byref(p), MATH[math_mode], _ptr(g_t_in), _ptr(g_W), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "dstd_dense_bwd")


def conv_out_hw(H, W, k, stride, pad):
    return (H + 2 * pad - k) // stride + 1, (W + 2 * pad - k) // stride + 1


def conv_workspace_bytes(B, H, W, C_in, C_out, k, stride, pad, p, math_mode):
    return load().dstd_conv_workspace_bytes(B, H, W, C_in, C_out, k, stride, pad, ctypes.byref(p), MATH[math_mode])


def conv_fwd(t_in, W, stride, pad, p, math_mode, t_out, saved, penalty, workspace, stream=None):
    """t_in [B, H, W, C_in] NHWC, W [C_out, k, k, C_in] -> t_out [B, Ho, Wo, C_out]."""
    B, H, Wd, C = t_in.shape
    C_out, k = W.shape[0], W.shape[1]
    Ho, Wo = conv_out_hw(H, Wd, k, stride, pad)
    _f32(t_in, "t_in")
    _f32(W, "W", (C_out, k, k, C))
    _f32(t_out, "t_out", (B, Ho, Wo, C_out))
    _check(load().dstd_conv_fwd(_ptr(t_in), _ptr(W), B, H, Wd, C, C_out, k, stride, pad, ctypes.byref(p),
                                MATH[math_mode], _ptr(t_out), _ptr(saved), _ptr(penalty), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream)), "dstd_conv_fwd")


def conv_bwd(t_in, W, t_out, saved, g_t_out, stride, pad, p, math_mode, g_t_in, g_W, workspace, stream=None):
    B, H, Wd, C = t_in.shape
    C_out, k = W.shape[0], W.shape[1]
    _f32(t_in, "t_in")
    _f32(W, "W", (C_out, k, k, C))
    _f32(g_W, "g_W", (C_out, k, k, C))
    if g_t_in is not None:
        _f32(g_t_in, "g_t_in", (B, H, Wd, C))
    _check(load().dstd_conv_bwd(_ptr(t_in), _ptr(W), _ptr(t_out), _ptr(saved), _ptr(g_t_out), B, H, Wd, C, C_out, k,
                                stride, pad, ctypes.byref(p), MATH[math_mode], _ptr(g_t_in), _ptr(g_W),
                                _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "dstd_conv_bwd")


def ce_loss(t_L, labels, tau_soft, t_silent, loss, g_t_L, stream=None):
    B, C = t_L.shape
    _f32(t_L, "t_L")
    _check(load().dstd_ce_loss(_ptr(t_L), _ptr(labels), B, C, float(tau_soft), float(t_silent), _ptr(loss),
                               _ptr(g_t_L), _stream(stream)), "dstd_ce_loss")


def ms_saved_bytes(B, N_out, F_out):
    return load().dstd_ms_saved_bytes(B, N_out, F_out)


def ms_workspace_bytes(B, N_in, N_out, F_in, F_out, p, math="x3"):
    return load().dstd_ms_workspace_bytes(B, N_in, N_out, F_in, F_out, ctypes.byref(p), MATH[math])


def dense_fwd_ms(t_in, W, p, math, t_out, saved, workspace, stream=None):
    """Multi-spike layer forward: t_in [B, N_in, F_in] -> t_out [B, N_out, F_out]."""
    B, N_in, F_in = t_in.shape
    N_out, F_out = t_out.shape[1], t_out.shape[2]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(t_out, "t_out", (B, N_out, F_out))
    _check(load().dstd_dense_fwd_ms(_ptr(t_in), _ptr(W), B, N_in, N_out, F_in, F_out, ctypes.byref(p), MATH[math],
                                    _ptr(t_out), _ptr(saved), _ptr(workspace), workspace.numel(), _stream(stream)),
           "dstd_dense_fwd_ms")


def dense_bwd_ms(t_in, W, t_out, saved, g_t_out, p, math, g_t_in, g_W, workspace, stream=None):
    """Multi-spike layer backward (g_t_in may be None)."""
    B, N_in, F_in = t_in.shape
    N_out, F_out = t_out.shape[1], t_out.shape[2]
    _check(load().dstd_dense_bwd_ms(_ptr(t_in), _ptr(W), _ptr(t_out), _ptr(saved), _ptr(g_t_out), B, N_in, N_out,
                                    F_in, F_out, ctypes.byref(p), MATH[math], _ptr(g_t_in), _ptr(g_W),
                                    _ptr(workspace), workspace.numel(), _stream(stream)), "dstd_dense_bwd_ms")


def concat_channels(a, b, delay_a, out, stream=None):
    """out[..., :C_a] = a + delay_a, out[..., C_a:] = b (channels innermost)."""
    for x, nm in ((a, "a"), (b, "b"), (out, "out")):
        _f32(x, nm)
    Ca, Cb = a.shape[-1], b.shape[-1]
    P = a.numel() // Ca
    if b.numel() != P * Cb or out.numel() != P * (Ca + Cb):
        raise ValueError("concat_channels: a, b and out disagree on the number of positions")
    _check(load().dstd_concat_channels(_ptr(a), Ca, float(delay_a), _ptr(b), Cb, P, _ptr(out),
                                       _stream(stream)), "dstd_concat_channels")


def split_channels(g, C_a, g_a=None, accumulate_a=False, g_b=None, accumulate_b=False, stream=None):
    """Adjoint of concat_channels: g[..., :C_a] into g_a, g[..., C_a:] into g_b
    (overwriting, or adding with accumulate_*); either target may be None."""
    _f32(g, "g")
    Ct = g.shape[-1]
    Cb = Ct - C_a
    P = g.numel() // Ct
    _check(load().dstd_split_channels(_ptr(g), int(C_a), int(Cb), P, _ptr(g_a) if g_a is not None else None,
                                      int(bool(accumulate_a)), _ptr(g_b) if g_b is not None else None,
                                      int(bool(accumulate_b)), _stream(stream)), "dstd_split_channels")


def sum_t_loss(t, loss, g, stream=None):
    _f32(t, "t")
    _check(load().dstd_sum_t_loss(_ptr(t), t.numel(), _ptr(loss), _ptr(g), _stream(stream)), "dstd_sum_t_loss")


def adamw(w, g, m, v, lr, beta1, beta2, eps, weight_decay, step, stream=None):
    _f32(w, "w")
    _check(load().dstd_adamw(_ptr(w), _ptr(g), _ptr(m), _ptr(v), w.numel(), float(lr), float(beta1), float(beta2),
                             float(eps), float(weight_decay), int(step), _stream(stream)), "dstd_adamw")


def adamw_multi(ws, gs, ms, vs, lr, beta1, beta2, eps, weight_decay, step, lr_dev=None, stream=None):
    """One AdamW launch over the tensors ws (in place, with gs, ms, vs alike);
    step is a device int32[2] tensor holding (updates done, 0)."""
    k = len(ws)
    if not (len(gs) == len(ms) == len(vs) == k):
        raise ValueError("adamw_multi: tensor lists differ in length")
    for w in ws:
        _f32(w, "w")
    import torch
    if step.dtype != torch.int32 or step.numel() != 2 or not step.is_cuda:
        raise ValueError("adamw_multi: step must be a device int32 tensor of 2 elements")
    arr = lambda xs: (ctypes.c_void_p * k)(*[x.data_ptr() for x in xs])
    n = (ctypes.c_int64 * k)(*[w.numel() for w in ws])
    _check(load().dstd_adamw_multi(k, arr(ws), arr(gs), arr(ms), arr(vs), n, float(lr), float(beta1), float(beta2),
                                   float(eps), float(weight_decay), _ptr(step), _ptr(lr_dev), _stream(stream)),
           "dstd_adamw_multi")


# -- training and serving in 8 bits ------------------------------------------
_TORCH = None       # torch, once one of these calls has needed it
_CODES = {}         # torch dtype -> dstd_type
_RAW_STREAM = None  # device index -> the current stream's handle
_DEVICE = None      # index of the current device
_ONLY = -2          # 0 where there is one device: it is the current one


def _torch():
    global _TORCH, _RAW_STREAM, _DEVICE, _ONLY
    if _TORCH is None:
        import torch
        _CODES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
        _RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        _DEVICE = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _ONLY = 0 if torch.cuda.device_count() == 1 else -2
        _TORCH = torch
    return _TORCH


def _here(x, dev, name):
    """Refuses x of device dev unless that is the current one: kernels run there,
    and another device's memory is out of their reach. The other tensors of a
    call are checked against dev. (With one device there is nothing to ask.)"""
    if dev < 0 or dev != _DEVICE():
        raise ValueError(f"{name} must be a tensor on the current CUDA device, not on {x.device}")


def _stream_of(stream, dev):
    """The stream to launch on: the given one, or the device's current one."""
    if stream is None:
        return _RAW_STREAM(dev)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _type_code(dtype, name):
    """dstd_type of a torch dtype (include/dstd.h)."""
    code = _CODES.get(dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, not {dtype}")
    return code


def _rows(x, name, R, K, dev, dtype=None):
    """Row stride of a matrix [R, K] on the device whose rows are contiguous (they may be padded, not overlap)."""
    if x.shape == (R, K) and x.get_device() == dev and (dtype is None or x.dtype == dtype):
        ld, one = x.stride()
        if (one == 1 or K <= 1) and ld >= K:
            return ld
        if (one == 1 or K <= 1) and R <= 1:
            return K
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    raise ValueError(f"{name} must be a matrix of shape {(R, K)} on cuda:{dev}" +
                     (f" and {dtype}" if dtype is not None else "") + f", not {tuple(x.shape)}, {x.dtype}, {x.device}")


def _floats(x, name, n, dev):
    if x.shape != (n,) or x.dtype != _TORCH.float32 or x.get_device() != dev or (n > 1 and x.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous float32 tensor of {n} on cuda:{dev}")


def _scratch(ws, where, dev):
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"{where}: workspace must be a contiguous tensor on cuda:{dev}")
    return ws.numel() * ws.element_size()


def quantize_rows(x, q, scale, values=None, stream=None):
    """Rows of x [R, K] (float32, bfloat16 or float16) to int8 codes q [R, K]
    and scales [R]: scale = max |x| / 127, q = x / scale to the nearest.
    ``values`` [R, K] float32 receives what the codes stand for. A row that is
    not finite gets scale NaN. Rows may be padded."""
    torch = _torch()
    R, K = x.shape
    dev = x.get_device()
    if dev != _ONLY:
        _here(x, dev, "x")
    ld_x = _rows(x, "x", R, K, dev)
    ld_q = _rows(q, "q", R, K, dev, torch.int8)
    _floats(scale, "scale", R, dev)
    ld_v, v = 0, None
    if values is not None:
        ld_v, v = _rows(values, "values", R, K, dev, torch.float32), values.data_ptr()
    code = load().dstd_quantize_rows(x.data_ptr(), _type_code(x.dtype, "x"), R, K, ld_x, q.data_ptr(), ld_q,
                                     scale.data_ptr(), v, ld_v, _stream_of(stream, dev))
    if code:
        raise DstdError(code, "dstd_quantize_rows")


def int8_matmul_workspace_bytes(T, N, K, aligned=False):
    """Scratch of int8_matmul for T tokens, N channels, K inputs: from 9 tokens
    on the tokens in 16 bits and room for a copy of the weights; without the
    latter where the rows of x and w start at multiples of 16 bytes (aligned)."""
    f = load().dstd_int8_matmul_aligned_workspace_bytes if aligned else load().dstd_int8_matmul_workspace_bytes
    return f(T, N, K)


def int8_matmul(x, x_scale, w, w_scale, out, workspace, stream=None):
    """out [T, N] = x_scale[:, None] * w_scale * (x @ w^T) of int8 rows x [T, K]
    and w [N, K]; the sum over K is exact. out is float32, bfloat16 or float16;
    rows may be padded."""
    torch = _torch()
    T, K = x.shape
    N = w.shape[0]
    dev = x.get_device()
    if dev != _ONLY:
        _here(x, dev, "x")
    ld_x = _rows(x, "x", T, K, dev, torch.int8)
    ld_w = _rows(w, "w", N, K, dev, torch.int8)
    ld_out = _rows(out, "out", T, N, dev)
    _floats(x_scale, "x_scale", T, dev)
    _floats(w_scale, "w_scale", N, dev)
    code = load().dstd_int8_matmul(x.data_ptr(), ld_x, x_scale.data_ptr(), w.data_ptr(), ld_w, w_scale.data_ptr(), T,
                                   N, K, out.data_ptr(), _type_code(out.dtype, "out"), ld_out, workspace.data_ptr(),
                                   _scratch(workspace, "int8_matmul", dev), _stream_of(stream, dev))
    if code:
        raise DstdError(code, "dstd_int8_matmul")


def dense_q8_workspace_bytes(B, N_in, N_out, p):
    return load().dstd_dense_q8_workspace_bytes(B, N_in, N_out, ctypes.byref(p))


def dense_fwd_q8(t_in, w_q, w_scale, p, t_out, saved, penalty, workspace, stream=None):
    """dense_fwd with an 8-bit contraction: w_q [N_out, N_in] int8 codes and
    w_scale [N_out] from quantize_rows; the grid weights are quantised for each
    (sample, grid point). Backward: dense_bwd with the weights' values."""
    torch = _torch()
    B, N_in = t_in.shape
    N_out = w_q.shape[0]
    _f32(t_in, "t_in")
    _f32(w_scale, "w_scale", (N_out,))
    _f32(t_out, "t_out", (B, N_out))
    dev = t_in.get_device()
    if dev != _ONLY:
        _here(t_in, dev, "t_in")
    if w_scale.get_device() != dev or t_out.get_device() != dev:
        raise ValueError(f"w_scale and t_out must be on cuda:{dev}")
    if w_q.dtype != torch.int8 or w_q.get_device() != dev or not w_q.is_contiguous() or tuple(w_q.shape) != (N_out, N_in):
        raise ValueError(f"w_q must be a contiguous int8 tensor [N_out, N_in] on cuda:{dev}")
    _check(load().dstd_dense_fwd_q8(t_in.data_ptr(), w_q.data_ptr(), w_scale.data_ptr(), B, N_in, N_out,
                                    ctypes.byref(p), t_out.data_ptr(), _ptr(saved), _ptr(penalty),
                                    workspace.data_ptr(), _scratch(workspace, "dense_fwd_q8", dev),
                                    _stream_of(stream, dev)), "dstd_dense_fwd_q8")


class TensorList:
    """Pointers, sizes and types of many tensors, checked and laid out once for
    the calls that take lists (grad_norm, clip_grads, adamw_clip). Keeps the
    tensors alive; their storage must stay where it is."""

    def __init__(self, tensors):
        _torch()
        self.tensors = list(tensors)
        for i, t in enumerate(self.tensors):
            if not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"tensor {i} of the list must be a contiguous CUDA tensor")
        devices = set(t.get_device() for t in self.tensors)
        if len(devices) > 1:
            raise ValueError("the tensors of a list must be on one device")
        self.device = devices.pop() if devices else None
        k = len(self.tensors)
        self.sizes = tuple(t.numel() for t in self.tensors)
        self.codes = tuple(_type_code(t.dtype, f"tensor {i} of the list") for i, t in enumerate(self.tensors))
        self.f32 = not any(self.codes)
        self.ptr = (ctypes.c_void_p * k)(*[t.data_ptr() for t in self.tensors])
        self.n = (ctypes.c_int64 * k)(*self.sizes)
        self.type = (ctypes.c_int32 * k)(*self.codes)

    def __len__(self):
        return len(self.tensors)


def _list(x):
    return x if isinstance(x, TensorList) else TensorList(x)


def _elsewhere(dev, where):
    raise ValueError(f"{where}: the lists' tensors must be on cuda:{dev}")


def grad_norm_workspace_bytes(gs):
    """Bytes of the workspace that grad_norm, clip_grads and adamw_clip share
    for these gradients: a tensor of zeros at first, left ready by each call.
    Asks for nothing but the sizes: tensors of any device will do."""
    sizes = gs.sizes if isinstance(gs, TensorList) else [t.numel() for t in gs]
    return load().dstd_grad_norm_workspace_bytes(len(sizes), (ctypes.c_int64 * len(sizes))(*sizes))


def grad_norm(gs, norm, workspace, tensor_norms=None, stream=None):
    """norm[0] = the 2-norm over all gradients of the list (float32, bfloat16 or
    float16 tensors, or a TensorList); tensor_norms [len(gs)]: of each."""
    _torch()
    gs = _list(gs)
    dev = norm.get_device()
    if dev != _ONLY:
        _here(norm, dev, "norm")
    if gs.device not in (dev, None):
        _elsewhere(dev, "grad_norm")
    _floats(norm, "norm", 1, dev)
    if tensor_norms is not None:
        _floats(tensor_norms, "tensor_norms", len(gs.sizes), dev)
    code = load().dstd_grad_norm(len(gs.sizes), gs.ptr, gs.n, gs.type, norm.data_ptr(), _ptr(tensor_norms),
                                 workspace.data_ptr(), _scratch(workspace, "grad_norm", dev), _stream_of(stream, dev))
    if code:
        raise DstdError(code, "dstd_grad_norm")


def clip_grads(gs, max_norm, norm, workspace, outs=None, stream=None):
    """Gradients times min(1, max_norm / norm), in place or into ``outs``;
    norm[0] receives the norm before clipping. Where a gradient is infinite or
    NaN all pass unchanged. Finite gradients whose norm passes float32 are
    clipped, although norm[0] is inf."""
    _torch()
    gs = _list(gs)
    outs = gs if outs is None else _list(outs)
    if gs.sizes != outs.sizes or gs.codes != outs.codes:
        raise ValueError("clip_grads: outs must have the gradients' sizes and types")
    dev = norm.get_device()
    if dev != _ONLY:
        _here(norm, dev, "norm")
    if not (gs.device == outs.device and gs.device in (dev, None)):
        _elsewhere(dev, "clip_grads")
    _floats(norm, "norm", 1, dev)
    code = load().dstd_clip_grads(len(gs.sizes), gs.ptr, outs.ptr, gs.n, gs.type, max_norm, norm.data_ptr(),
                                  workspace.data_ptr(), _scratch(workspace, "clip_grads", dev), _stream_of(stream, dev))
    if code:
        raise DstdError(code, "dstd_clip_grads")


def adamw_clip(ws, gs, ms, vs, lr, beta1, beta2, eps, weight_decay, step, max_norm, norm, workspace, lr_dev=None,
               stream=None):
    """One AdamW step of the tensors ws (in place, with ms, vs) on gradients
    clipped to the global norm max_norm; gs is only read. step: device int32
    tensor whose first element counts the updates done. Where a gradient is
    infinite or NaN nothing changes but norm[0], and the count tells so:
    norm[0] is also inf where the norm of finite gradients passes float32, and
    those are clipped and the step is done."""
    torch = _torch()
    ws, gs, ms, vs = _list(ws), _list(gs), _list(ms), _list(vs)
    if not (ws.sizes == gs.sizes == ms.sizes == vs.sizes):
        raise ValueError("adamw_clip: tensor lists differ in length or sizes")
    if not (ws.f32 and ms.f32 and vs.f32):
        raise ValueError("adamw_clip: weights and moments must be float32")
    dev = norm.get_device()
    if dev != _ONLY:
        _here(norm, dev, "norm")
    if not (ws.device == gs.device == ms.device == vs.device and gs.device in (dev, None)):
        _elsewhere(dev, "adamw_clip")
    if step.dtype != torch.int32 or step.numel() < 1 or step.get_device() != dev:
        raise ValueError(f"adamw_clip: step must be an int32 tensor on cuda:{dev}")
    if lr_dev is not None:
        _f32(lr_dev, "lr_dev")
        if lr_dev.get_device() != dev:
            raise ValueError(f"adamw_clip: lr_dev must be on cuda:{dev}")
    _floats(norm, "norm", 1, dev)
    code = load().dstd_adamw_clip(len(gs.sizes), ws.ptr, gs.ptr, ms.ptr, vs.ptr, gs.n, gs.type, lr, beta1, beta2, eps,
                                  weight_decay, max_norm, step.data_ptr(), _ptr(lr_dev), norm.data_ptr(),
                                  workspace.data_ptr(), _scratch(workspace, "adamw_clip", dev), _stream_of(stream, dev))
    if code:
        raise DstdError(code, "dstd_adamw_clip")


def device_status(clear=True):
    """DSTD_OK (0) or DSTD_E_TIMEOUT after synchronising the device."""
    return load().dstd_device_status(1 if clear else 0)



def timing_enable(on=True):
    """Turn per-kernel event timing on/off (clears the counters)."""
    _check(load().dstd_timing_enable(1 if on else 0), "dstd_timing_enable")


def exact_workspace_bytes(B, N_in, N_out):
    return load().dstd_exact_workspace_bytes(B, N_in, N_out)


def exact_fwd(t_in, W, p, t_out, workspace, stream=None):
    """Exact (event-driven, Alg. 1) first-spike times of a dense layer."""
    B, N_in = t_in.shape
    N_out = W.shape[0]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(t_out, "t_out", (B, N_out))
    _check(load().dstd_exact_fwd(_ptr(t_in), _ptr(W), B, N_in, N_out, ctypes.byref(p), _ptr(t_out), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "dstd_exact_fwd")


def exact_bwd(t_in, W, t_out, g_t_out, p, g_t_in, g_W, workspace, stream=None):
    """Backward of the exact layer (implicit function theorem at each exact
    spike time): g_W [N_out, N_in] and g_t_in [B, N_in] (or None), overwritten."""
    B, N_in = t_in.shape
    N_out = W.shape[0]
    _f32(t_in, "t_in")
    _f32(W, "W", (N_out, N_in))
    _f32(t_out, "t_out", (B, N_out))
    _f32(g_t_out, "g_t_out", (B, N_out))
    _f32(g_W, "g_W", (N_out, N_in))
    if g_t_in is not None:
        _f32(g_t_in, "g_t_in", (B, N_in))
    _check(load().dstd_exact_bwd(_ptr(t_in), _ptr(W), _ptr(t_out), _ptr(g_t_out), B, N_in, N_out, ctypes.byref(p),
                                 _ptr(g_t_in) if g_t_in is not None else None, _ptr(g_W), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "dstd_exact_bwd")


def set_pair_policy(policy):
    """Forward contraction scheduling: 0 cost model (default), 1 SM pairs
    wherever they apply, 2 single CTAs only. Returns the previous policy."""
    r = load().dstd_set_pair_policy(int(policy))
    if r < 0:
        raise DstdError(r, "dstd_set_pair_policy")
    return r


def conv_set_chunk_images(max_images):
    """Cap the images per chunk of the implicit-GEMM conv layers (0 = from
    the scratch budget). Returns the previous cap; query the workspace size
    again afterwards."""
    return int(load().dstd_conv_set_chunk_images(int(max_images)))


def conv_set_operand_policy(policy):
    """Operand of the implicit-GEMM conv forward and dW: 0 by layer shape,
    1 generated on chip, 2 the binned input written out and read through
    TMA. Returns the previous policy; query the workspace size again."""
    return int(load().dstd_conv_set_operand_policy(int(policy)))


def timing_collect():
    """Add the last replay of a graph captured with timing on to the totals."""
    _check(load().dstd_timing_collect(), "dstd_timing_collect")


def timing_read():
    """{kernel kind: (total ms, launches)} accumulated since timing_enable."""
    lib = load()
    out = {}
    for k in range(lib.dstd_kernel_kind_count()):
        ms = _F()
        n = _I64()
        _check(lib.dstd_timing_read(k, ctypes.byref(ms), ctypes.byref(n)), "dstd_timing_read")
        out[lib.dstd_kernel_kind_name(k).decode()] = (ms.value, n.value)
    return out


def selftest_wait_timeout(timeout_us, stream=None):
    """Launch the bounded-wait self-test (see include/dstd.h)."""
    _check(load().dstd_selftest_wait_timeout(int(timeout_us), _stream(stream)), "dstd_selftest_wait_timeout")
