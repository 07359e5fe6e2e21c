"""Thin Python binding of the DSTD-LIF C ABI (``include/dstd_lif.h``).

The functions named like the C entry points take plain integers (device
pointers, sizes, stream handles) and return the status code. The tensor
helpers below them only marshal arguments: they allocate outputs and
workspace with PyTorch on the tensors' device, pass ``data_ptr()`` and the
current stream, and raise on a non-OK status. Every step of the layer runs in
the HIP library; if ``libdstd_lif.so`` is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Optional, Tuple

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdstd_lif.so")

DSTD_OK = 0
DSTD_ERR_NULL = -1
DSTD_ERR_SHAPE = -2
DSTD_ERR_PARAM = -3
DSTD_ERR_UNSUPPORTED = -4
DSTD_ERR_WORKSPACE = -5
DSTD_ERR_HIP = -6
DSTD_F32 = 0
DSTD_BF16 = 1
DSTD_MAX_M = 256
DSTD_NOALLOC_SCRATCH_BYTES = 32 << 20
DSTD_FLAG_CONTRACT_SPARSE = 0x2
DSTD_FLAG_CONTRACT_MFMA = 0x4
DSTD_FLAG_CONV_KEEP = 0x8
DSTD_FLAG_CONV_REUSE = 0x10


class dstd_lif_params(C.Structure):
    _fields_ = [("tau_m", C.c_float), ("tau_s", C.c_float), ("threshold", C.c_float),
                ("M", C.c_int32), ("t0", C.c_float), ("dt", C.c_float), ("t_max", C.c_float),
                ("flags", C.c_int32)]


class dstd_conv_shape(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("C_in", "H", "W", "C_out", "KH", "KW", "stride", "pad",
                                         "pool_in")]


class dstd_synfire_params(C.Structure):
    _fields_ = [(k, C.c_float) for k in ("gamma_head", "gamma_tail", "t_head", "t_tail", "gamma_q",
                                         "scale")]


class dstd_tensor(C.Structure):
    _fields_ = ([(k, C.c_void_p) for k in ("g", "out", "w", "w32", "m", "v")] + [("n", C.c_int64)] +
                [(k, C.c_int32) for k in ("g_dtype", "out_dtype", "w_dtype")] +
                [(k, C.c_float) for k in ("lr_scale", "decay_scale")])


class dstd_tensor_list(C.Structure):
    _fields_ = [("mem", C.c_void_p), ("n_tensors", C.c_int64), ("n_chunks", C.c_int64),
                ("g_bytes", C.c_int64), ("out_bytes", C.c_int64), ("w_bytes", C.c_int64),
                ("magic", C.c_uint32), ("has_weights", C.c_uint32), ("g_types", C.c_uint32)]


class dstd_adamw_params(C.Structure):
    _fields_ = [(k, C.c_double) for k in ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm")]


class DSTDError(RuntimeError):
    def __init__(self, fn: str, status: int):
        lib = _load()
        self.status = status
        msg = lib.dstd_status_string(status).decode()
        detail = lib.dstd_last_error().decode()
        super().__init__(f"{fn}: {msg} ({status}): {detail}")


_lib = None
_P = C.c_void_p
_L = C.c_int64
_S = C.c_size_t
_I = C.c_int
_F = C.c_float
_D = C.c_double

# name -> (restype, argtypes)
_SIGS = {
    "dstd_lif_forward_workspace_size": (_S, [_P, _L, _L, _L]),
    "dstd_lif_backward_workspace_size": (_S, [_P, _L, _L, _L]),
    "dstd_lif_forward": (_I, [_P, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P, _S, _P]),
    "dstd_lif_forward_noalloc": (_I, [_P, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P]),
    "dstd_lif_backward": (_I, [_P, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P, _P, _P, _P, _S, _P]),
    "dstd_lif_conv_forward_workspace_size": (_S, [_P, _P, _L]),
    "dstd_lif_conv_backward_workspace_size": (_S, [_P, _P, _L]),
    "dstd_lif_conv_forward": (_I, [_P, _P, _L, _P, _P, _I, _P, _P, _P, _P, _S, _P]),
    "dstd_lif_conv_backward": (_I, [_P, _P, _L, _P, _P, _I, _P, _P, _P, _P, _P, _P, _P, _S, _P]),
    "dstd_lif_backward_synfire": (_I, [_P, _P, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P, _P, _P, _P,
                                       _S, _P]),
    "dstd_lif_conv_backward_synfire": (_I, [_P, _P, _P, _L, _P, _P, _I, _P, _P, _P, _P, _P, _P, _P,
                                            _S, _P]),
    "dstd_synfire_penalty_workspace_size": (_S, [_L, _L, _L]),
    "dstd_synfire_penalty": (_I, [_P, _L, _L, _L, _L, _P, _P, _I, _P, _P, _S, _P]),
    "dstd_exact_forward_workspace_size": (_S, [_P, _L, _L, _L]),
    "dstd_exact_backward_workspace_size": (_S, [_P, _L, _L, _L]),
    "dstd_exact_forward": (_I, [_P, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P, _S, _P]),
    "dstd_exact_backward": (_I, [_P, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P, _P, _P, _P, _S, _P]),
    "dstd_lif_multispike_forward_workspace_size": (_S, [_P, _L, _L, _L, _L, _L]),
    "dstd_lif_multispike_backward_workspace_size": (_S, [_P, _L, _L, _L, _L, _L]),
    "dstd_lif_multispike_forward": (_I, [_P, _L, _L, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P, _P,
                                         _S, _P]),
    "dstd_lif_multispike_backward": (_I, [_P, _L, _L, _L, _L, _L, _P, _P, _I, _P, _P, _P, _P, _P,
                                          _P, _P, _P, _S, _P]),
    "dstd_skip_delay_concat": (_I, [_L, _L, _L, _L, _P, _F, _P, _P, _P]),
    "dstd_skip_delay_concat_backward": (_I, [_L, _L, _L, _L, _P, _P, C.c_int32, _P, _P]),
    "dstd_softmax_ce_grad": (_I, [_L, _L, _P, _P, _F, _F, _P, _P, _P]),
    "dstd_mse_grad": (_I, [_L, _L, _P, _P, _P, _P, _P]),
    "dstd_tensor_list_size": (_S, [_L, _P]),
    "dstd_tensor_list_build": (_I, [_L, _P, _P, _S, _P, _P]),
    "dstd_tensor_list_workspace_size": (_S, [_P]),
    "dstd_grad_norm": (_I, [_P, _P, _P, _S, _P]),
    "dstd_grad_clip": (_I, [_P, _D, _P, C.c_int32, _P, _S, _P]),
    "dstd_adamw_step": (_I, [_P, _P, _P, _P, _P, C.c_int32, _P, _S, _P]),
    "dstd_profile_enable": (C.c_int32, [C.c_int32]),
    "dstd_profile_collect": (_I, []),
    "dstd_profile_count": (C.c_int32, []),
    "dstd_profile_entry": (_I, [C.c_int32, C.POINTER(C.c_char_p), C.POINTER(C.c_int64),
                                C.POINTER(C.c_double)]),
    "dstd_profile_reset": (None, []),
    "dstd_status_string": (C.c_char_p, [_I]),
    "dstd_last_error": (C.c_char_p, []),
    "dstd_version": (C.c_int32, []),
}


def _load():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2607_14672_amd.build`")
        lib = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def exported_symbols():
    return list(_SIGS)


def _ref(s):
    return None if s is None else C.addressof(s)


# ------------------------------------------------------------ raw C ABI --
def dstd_lif_forward_workspace_size(p, B, N_in, N_out):
    return _load().dstd_lif_forward_workspace_size(_ref(p), B, N_in, N_out)


def dstd_lif_backward_workspace_size(p, B, N_in, N_out):
    return _load().dstd_lif_backward_workspace_size(_ref(p), B, N_in, N_out)


def dstd_lif_forward(p, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx, ws, ws_bytes, stream):
    return _load().dstd_lif_forward(_ref(p), B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx,
                                    ws, ws_bytes, stream)


def dstd_lif_forward_noalloc(p, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx, stream):
    return _load().dstd_lif_forward_noalloc(_ref(p), B, N_in, N_out, t_in, W, w_dtype, t_out,
                                            slope, q_idx, stream)


def dstd_lif_backward(p, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx, grad_t_out,
                      grad_W, grad_t_in, ws, ws_bytes, stream):
    return _load().dstd_lif_backward(_ref(p), B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx,
                                     grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream)


def dstd_exact_forward_workspace_size(p, B, N_in, N_out):
    return _load().dstd_exact_forward_workspace_size(_ref(p), B, N_in, N_out)


def dstd_exact_backward_workspace_size(p, B, N_in, N_out):
    return _load().dstd_exact_backward_workspace_size(_ref(p), B, N_in, N_out)


def dstd_exact_forward(p, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, k_idx, ws, ws_bytes,
                       stream):
    return _load().dstd_exact_forward(_ref(p), B, N_in, N_out, t_in, W, w_dtype, t_out, slope,
                                      k_idx, ws, ws_bytes, stream)


def dstd_exact_backward(p, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, k_idx, grad_t_out,
                        grad_W, grad_t_in, ws, ws_bytes, stream):
    return _load().dstd_exact_backward(_ref(p), B, N_in, N_out, t_in, W, w_dtype, t_out, slope,
                                       k_idx, grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream)


def dstd_lif_multispike_forward_workspace_size(p, B, N_in, F_in, N_out, F_out):
    return _load().dstd_lif_multispike_forward_workspace_size(_ref(p), B, N_in, F_in, N_out, F_out)


def dstd_lif_multispike_backward_workspace_size(p, B, N_in, F_in, N_out, F_out):
    return _load().dstd_lif_multispike_backward_workspace_size(_ref(p), B, N_in, F_in, N_out, F_out)


def dstd_lif_multispike_forward(p, B, N_in, F_in, N_out, F_out, t_in, W, w_dtype, t_out, slope,
                                q_idx, cur, ws, ws_bytes, stream):
    return _load().dstd_lif_multispike_forward(_ref(p), B, N_in, F_in, N_out, F_out, t_in, W,
                                               w_dtype, t_out, slope, q_idx, cur, ws, ws_bytes,
                                               stream)


def dstd_lif_multispike_backward(p, B, N_in, F_in, N_out, F_out, t_in, W, w_dtype, t_out, slope,
                                 q_idx, cur, grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream):
    return _load().dstd_lif_multispike_backward(_ref(p), B, N_in, F_in, N_out, F_out, t_in, W,
                                                w_dtype, t_out, slope, q_idx, cur, grad_t_out,
                                                grad_W, grad_t_in, ws, ws_bytes, stream)


def dstd_skip_delay_concat(B, C1, C2, HW, t1, delay, t2, out, stream):
    return _load().dstd_skip_delay_concat(B, C1, C2, HW, t1, delay, t2, out, stream)


def dstd_skip_delay_concat_backward(B, C1, C2, HW, g, g1, accumulate, g2, stream):
    return _load().dstd_skip_delay_concat_backward(B, C1, C2, HW, g, g1, accumulate, g2, stream)


def dstd_lif_conv_forward_workspace_size(p, cs, B):
    return _load().dstd_lif_conv_forward_workspace_size(_ref(p), _ref(cs), B)


def dstd_lif_conv_backward_workspace_size(p, cs, B):
    return _load().dstd_lif_conv_backward_workspace_size(_ref(p), _ref(cs), B)


def dstd_lif_conv_forward(p, cs, B, t_in, W, w_dtype, t_out, slope, q_idx, ws, ws_bytes, stream):
    return _load().dstd_lif_conv_forward(_ref(p), _ref(cs), B, t_in, W, w_dtype, t_out, slope, q_idx,
                                         ws, ws_bytes, stream)


def dstd_lif_conv_backward(p, cs, B, t_in, W, w_dtype, t_out, slope, q_idx, grad_t_out, grad_W,
                           grad_t_in, ws, ws_bytes, stream):
    return _load().dstd_lif_conv_backward(_ref(p), _ref(cs), B, t_in, W, w_dtype, t_out, slope,
                                          q_idx, grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream)


def dstd_lif_backward_synfire(p, sp, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx,
                              grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream):
    return _load().dstd_lif_backward_synfire(_ref(p), _ref(sp), B, N_in, N_out, t_in, W, w_dtype,
                                             t_out, slope, q_idx, grad_t_out, grad_W, grad_t_in,
                                             ws, ws_bytes, stream)


def dstd_lif_conv_backward_synfire(p, sp, cs, B, t_in, W, w_dtype, t_out, slope, q_idx,
                                   grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream):
    return _load().dstd_lif_conv_backward_synfire(_ref(p), _ref(sp), _ref(cs), B, t_in, W, w_dtype,
                                                  t_out, slope, q_idx, grad_t_out, grad_W,
                                                  grad_t_in, ws, ws_bytes, stream)


def dstd_synfire_penalty_workspace_size(B, rows, spatial):
    return _load().dstd_synfire_penalty_workspace_size(B, rows, spatial)


def dstd_synfire_penalty(sp, B, rows, spatial, row_len, t_out, W, w_dtype, value, ws, ws_bytes,
                         stream):
    return _load().dstd_synfire_penalty(_ref(sp), B, rows, spatial, row_len, t_out, W, w_dtype,
                                        value, ws, ws_bytes, stream)


def dstd_softmax_ce_grad(B, N, t_out, labels, tau_soft, t_cap, grad_t, loss, stream):
    return _load().dstd_softmax_ce_grad(B, N, t_out, labels, tau_soft, t_cap, grad_t, loss, stream)


def dstd_mse_grad(B, N, t_out, target, grad_t, loss, stream):
    return _load().dstd_mse_grad(B, N, t_out, target, grad_t, loss, stream)


def dstd_tensor_list_size(n_tensors, tensors):
    return _load().dstd_tensor_list_size(n_tensors, _ref(tensors))


def dstd_tensor_list_build(n_tensors, tensors, mem, mem_bytes, lst, stream):
    return _load().dstd_tensor_list_build(n_tensors, _ref(tensors), mem, mem_bytes, _ref(lst), stream)


def dstd_tensor_list_workspace_size(lst):
    return _load().dstd_tensor_list_workspace_size(_ref(lst))


def dstd_grad_norm(lst, norm, ws, ws_bytes, stream):
    return _load().dstd_grad_norm(_ref(lst), norm, ws, ws_bytes, stream)


def dstd_grad_clip(lst, max_norm, norm, norm_given, ws, ws_bytes, stream):
    return _load().dstd_grad_clip(_ref(lst), max_norm, norm, norm_given, ws, ws_bytes, stream)


def dstd_adamw_step(lst, p, lr, step, norm, norm_given, ws, ws_bytes, stream):
    return _load().dstd_adamw_step(_ref(lst), _ref(p), lr, step, norm, norm_given, ws, ws_bytes,
                                   stream)


def dstd_status_string(s):
    return _load().dstd_status_string(s).decode()


def dstd_last_error():
    return _load().dstd_last_error().decode()


def dstd_version():
    return _load().dstd_version()


def dstd_profile_enable(on):
    return _load().dstd_profile_enable(1 if on else 0)


def dstd_profile_collect():
    return _load().dstd_profile_collect()


def dstd_profile_count():
    return _load().dstd_profile_count()


def dstd_profile_entry(idx):
    name = C.c_char_p()
    n = C.c_int64()
    ms = C.c_double()
    st = _load().dstd_profile_entry(idx, C.byref(name), C.byref(n), C.byref(ms))
    _check("dstd_profile_entry", st)
    return name.value.decode(), n.value, ms.value


def dstd_profile_reset():
    _load().dstd_profile_reset()


def profile_table():
    """{kernel name: (launches, total ms)} of the library's own timer."""
    dstd_profile_collect()
    return {e[0]: (e[1], e[2]) for e in (dstd_profile_entry(i) for i in range(dstd_profile_count()))}


# -------------------------------------------------------- tensor helpers --
def make_params(tau_m, tau_s, threshold, M, t0, dt, t_max=math.inf, flags=0) -> dstd_lif_params:
    return dstd_lif_params(float(tau_m), float(tau_s), float(threshold), int(M), float(t0),
                           float(dt), float(t_max), int(flags))


def make_synfire(gamma_head, gamma_tail, t_head, t_tail, gamma_q, scale) -> dstd_synfire_params:
    """One layer's synfire-term parameters (window ends t_head, t_tail already
    shifted for the layer; scale = 1/B, conv 1/(B*H_out*W_out))."""
    return dstd_synfire_params(gamma_head, gamma_tail, t_head, t_tail, gamma_q, scale)


def make_conv_shape(C_in, H, W, C_out, KH=3, KW=3, stride=1, pad=1, pool_in=1) -> dstd_conv_shape:
    return dstd_conv_shape(C_in, H, W, C_out, KH, KW, stride, pad, pool_in)


def conv_out_hw(cs: dstd_conv_shape) -> Tuple[int, int]:
    H, W = cs.H, cs.W
    if cs.pool_in == 2:
        H, W = H // 2, W // 2
    elif cs.pool_in == 0:
        H, W = 1, 1
    return (H + 2 * cs.pad - cs.KH) // cs.stride + 1, (W + 2 * cs.pad - cs.KW) // cs.stride + 1


def _torch():
    import torch
    return torch


def _stream(dev):
    return _torch().cuda.current_stream(dev).cuda_stream


def _wdtype(W):
    torch = _torch()
    if W.dtype == torch.float32:
        return DSTD_F32
    if W.dtype == torch.bfloat16:
        return DSTD_BF16
    raise TypeError(f"W must be float32 or bfloat16, got {W.dtype}")


def _check(name, st):
    if st != DSTD_OK:
        raise DSTDError(name, st)


def _cont(x, dtype=None):
    if dtype is not None:
        assert x.dtype == dtype, f"expected {dtype}, got {x.dtype}"
    assert x.is_cuda, "tensors must live on the GPU"
    return x.contiguous()


def _ptr(x):
    return None if x is None else x.data_ptr()


def workspace(nbytes: int, device):
    torch = _torch()
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def _grad_dest(torch, grad_W, W, shape, dev, need_W):
    """Where a backward writes dL/dW (f32): `grad_W`, checked, a new tensor, or
    None where it is not wanted."""
    if grad_W is None:
        return torch.empty(shape, dtype=torch.float32, device=dev) if need_W else None
    if not need_W:
        raise ValueError("grad_W is given, but need_W is False")
    if not isinstance(grad_W, torch.Tensor) or grad_W.dtype != torch.float32:
        raise TypeError("grad_W must be a float32 tensor")
    if grad_W.device != dev:
        raise ValueError(f"grad_W must be on {dev}")
    if grad_W.shape != torch.Size(shape):
        raise ValueError(f"grad_W has shape {tuple(grad_W.shape)}, not {tuple(shape)}")
    if not grad_W.is_contiguous():
        raise ValueError("grad_W must be contiguous")
    a, b = grad_W.data_ptr(), W.data_ptr()
    if a < b + W.numel() * W.element_size() and b < a + grad_W.numel() * 4:
        raise ValueError("grad_W and W share the same memory")
    return grad_W


def forward(p: dstd_lif_params, t_in, W, ws=None):
    """Dense layer forward. t_in [B, N_in] f32, W [N_out, N_in] f32|bf16 (CUDA tensors)."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B, N_in = t_in.shape
    N_out = W.shape[0]
    assert W.shape[1] == N_in
    dev = t_in.device
    t_out = torch.empty((B, N_out), dtype=torch.float32, device=dev)
    slope = torch.empty_like(t_out)
    q = torch.empty((B, N_out), dtype=torch.int32, device=dev)
    need = dstd_lif_forward_workspace_size(p, B, N_in, N_out)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    _check("dstd_lif_forward",
           dstd_lif_forward(p, B, N_in, N_out, _ptr(t_in), _ptr(W), _wdtype(W), _ptr(t_out),
                            _ptr(slope), _ptr(q), _ptr(ws), ws.numel(), _stream(dev)))
    return t_out, slope, q


def forward_noalloc(p: dstd_lif_params, t_in, W, outputs=None):
    """Dense layer forward through the allocation-free entry point (the
    library's static scratch). `outputs` = (t_out, slope, q) preallocated
    tensors, or None to allocate them here."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B, N_in = t_in.shape
    N_out = W.shape[0]
    assert W.shape[1] == N_in
    dev = t_in.device
    if outputs is None:
        t_out = torch.empty((B, N_out), dtype=torch.float32, device=dev)
        outputs = (t_out, torch.empty_like(t_out), torch.empty((B, N_out), dtype=torch.int32, device=dev))
    t_out, slope, q = outputs
    _check("dstd_lif_forward_noalloc",
           dstd_lif_forward_noalloc(p, B, N_in, N_out, _ptr(t_in), _ptr(W), _wdtype(W), _ptr(t_out),
                                    _ptr(slope), _ptr(q), _stream(dev)))
    return t_out, slope, q


def backward(p: dstd_lif_params, t_in, W, t_out, slope, q, grad_t_out, need_W=True,
             need_t_in=True, ws=None, synfire: Optional[dstd_synfire_params] = None, grad_W=None):
    """Dense layer backward; returns (grad_W or None, grad_t_in or None). With
    `synfire`, the layer's temporal-penalty and dead-neuron gradients are
    included. dL/dW is written to `grad_W` if given (f32, as all four
    backward helpers take it), else to a new tensor at each call: a tensor list
    needs the former."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B, N_in = t_in.shape
    N_out = W.shape[0]
    dev = t_in.device
    gW = _grad_dest(torch, grad_W, W, (N_out, N_in), dev, need_W)
    gt = torch.empty((B, N_in), dtype=torch.float32, device=dev) if need_t_in else None
    need = dstd_lif_backward_workspace_size(p, B, N_in, N_out)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    args = (B, N_in, N_out, _ptr(t_in), _ptr(W), _wdtype(W), _ptr(_cont(t_out, torch.float32)),
            _ptr(_cont(slope, torch.float32)), _ptr(_cont(q, torch.int32)),
            _ptr(_cont(grad_t_out, torch.float32)), _ptr(gW), _ptr(gt), _ptr(ws), ws.numel(),
            _stream(dev))
    if synfire is None:
        _check("dstd_lif_backward", dstd_lif_backward(p, *args))
    else:
        _check("dstd_lif_backward_synfire", dstd_lif_backward_synfire(p, synfire, *args))
    return gW, gt


def multispike_forward(p: dstd_lif_params, t_in, W, F_out: int, ws=None):
    """Multi-spike dense forward. t_in [B, N_in, F_in]; returns (t_out, slope, q, cur),
    each [B, N_out, F_out]."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B, N_in, F_in = t_in.shape
    N_out = W.shape[0]
    dev = t_in.device
    shp = (B, N_out, F_out)
    t_out = torch.empty(shp, dtype=torch.float32, device=dev)
    slope = torch.empty_like(t_out)
    cur = torch.empty_like(t_out)
    q = torch.empty(shp, dtype=torch.int32, device=dev)
    need = dstd_lif_multispike_forward_workspace_size(p, B, N_in, F_in, N_out, F_out)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    _check("dstd_lif_multispike_forward",
           dstd_lif_multispike_forward(p, B, N_in, F_in, N_out, F_out, _ptr(t_in), _ptr(W),
                                       _wdtype(W), _ptr(t_out), _ptr(slope), _ptr(q), _ptr(cur),
                                       _ptr(ws), ws.numel(), _stream(dev)))
    return t_out, slope, q, cur


def multispike_backward(p: dstd_lif_params, t_in, W, t_out, slope, q, cur, grad_t_out,
                        need_W=True, need_t_in=True, ws=None, grad_W=None):
    """Multi-spike dense backward; returns (grad_W or None, grad_t_in [B, N_in, F_in] or None)."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B, N_in, F_in = t_in.shape
    N_out = W.shape[0]
    F_out = t_out.shape[2]
    dev = t_in.device
    gW = _grad_dest(torch, grad_W, W, (N_out, N_in), dev, need_W)
    gt = torch.empty((B, N_in, F_in), dtype=torch.float32, device=dev) if need_t_in else None
    need = dstd_lif_multispike_backward_workspace_size(p, B, N_in, F_in, N_out, F_out)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    _check("dstd_lif_multispike_backward",
           dstd_lif_multispike_backward(p, B, N_in, F_in, N_out, F_out, _ptr(t_in), _ptr(W),
                                        _wdtype(W), _ptr(_cont(t_out, torch.float32)),
                                        _ptr(_cont(slope, torch.float32)),
                                        _ptr(_cont(q, torch.int32)), _ptr(_cont(cur, torch.float32)),
                                        _ptr(_cont(grad_t_out, torch.float32)), _ptr(gW), _ptr(gt),
                                        _ptr(ws), ws.numel(), _stream(dev)))
    return gW, gt


def skip_delay_concat(t1, delay: float, t2):
    """SD-block skip input: cat([t1 + delay, t2], channels). t1 [B, C1, H, W], t2 [B, C2, H, W]."""
    torch = _torch()
    t1 = _cont(t1, torch.float32)
    t2 = _cont(t2, torch.float32)
    B, C1 = t1.shape[:2]
    C2 = t2.shape[1]
    assert t2.shape[0] == B and t1.shape[2:] == t2.shape[2:]
    HW = int(math.prod(t1.shape[2:]))
    out = torch.empty((B, C1 + C2) + tuple(t1.shape[2:]), dtype=torch.float32, device=t1.device)
    _check("dstd_skip_delay_concat",
           dstd_skip_delay_concat(B, C1, C2, HW, _ptr(t1), float(delay), _ptr(t2), _ptr(out),
                                  _stream(t1.device)))
    return out


def skip_delay_concat_backward(g, C1: int, g1=None, want_g2=True):
    """Split dL/d(concat) [B, C1 + C2, H, W]: adds the first C1 channels into g1
    (written when g1 is None) and returns (g1, g2)."""
    torch = _torch()
    g = _cont(g, torch.float32)
    B, C = g.shape[:2]
    C2 = C - C1
    HW = int(math.prod(g.shape[2:]))
    acc = 1
    if g1 is None:
        g1 = torch.empty((B, C1) + tuple(g.shape[2:]), dtype=torch.float32, device=g.device)
        acc = 0
    else:
        assert g1.is_contiguous() and g1.dtype == torch.float32 and g1.shape[:2] == (B, C1)
    g2 = torch.empty((B, C2) + tuple(g.shape[2:]), dtype=torch.float32, device=g.device) if want_g2 else None
    _check("dstd_skip_delay_concat_backward",
           dstd_skip_delay_concat_backward(B, C1, C2, HW, _ptr(g), _ptr(g1), acc, _ptr(g2),
                                           _stream(g.device)))
    return g1, g2


def exact_forward(p: dstd_lif_params, t_in, W, ws=None):
    """Exact (sorted-input) forward of a dense layer; returns (t_out, slope,
    k_idx). Only tau_m, tau_s, threshold and t_max of `p` are used."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B, N_in = t_in.shape
    N_out = W.shape[0]
    assert W.shape[1] == N_in
    dev = t_in.device
    t_out = torch.empty((B, N_out), dtype=torch.float32, device=dev)
    slope = torch.empty_like(t_out)
    k = torch.empty((B, N_out), dtype=torch.int32, device=dev)
    need = dstd_exact_forward_workspace_size(p, B, N_in, N_out)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    _check("dstd_exact_forward",
           dstd_exact_forward(p, B, N_in, N_out, _ptr(t_in), _ptr(W), _wdtype(W), _ptr(t_out),
                              _ptr(slope), _ptr(k), _ptr(ws), ws.numel(), _stream(dev)))
    return t_out, slope, k


def exact_backward(p: dstd_lif_params, t_in, W, t_out, slope, k, grad_t_out, need_W=True,
                   need_t_in=True, ws=None, grad_W=None):
    """Exact backward of a dense layer; returns (grad_W or None, grad_t_in or None)."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B, N_in = t_in.shape
    N_out = W.shape[0]
    dev = t_in.device
    gW = _grad_dest(torch, grad_W, W, (N_out, N_in), dev, need_W)
    gt = torch.empty((B, N_in), dtype=torch.float32, device=dev) if need_t_in else None
    need = dstd_exact_backward_workspace_size(p, B, N_in, N_out)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    _check("dstd_exact_backward",
           dstd_exact_backward(p, B, N_in, N_out, _ptr(t_in), _ptr(W), _wdtype(W),
                               _ptr(_cont(t_out, torch.float32)), _ptr(_cont(slope, torch.float32)),
                               _ptr(_cont(k, torch.int32)), _ptr(_cont(grad_t_out, torch.float32)),
                               _ptr(gW), _ptr(gt), _ptr(ws), ws.numel(), _stream(dev)))
    return gW, gt


def conv_forward(p: dstd_lif_params, cs: dstd_conv_shape, t_in, W, ws=None):
    """Conv layer forward. t_in [B, C_in, H, W] f32, W [C_out, C_in, KH, KW]."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B = t_in.shape[0]
    Ho, Wo = conv_out_hw(cs)
    dev = t_in.device
    t_out = torch.empty((B, cs.C_out, Ho, Wo), dtype=torch.float32, device=dev)
    slope = torch.empty_like(t_out)
    q = torch.empty((B, cs.C_out, Ho, Wo), dtype=torch.int32, device=dev)
    need = dstd_lif_conv_forward_workspace_size(p, cs, B)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    _check("dstd_lif_conv_forward",
           dstd_lif_conv_forward(p, cs, B, _ptr(t_in), _ptr(W), _wdtype(W), _ptr(t_out),
                                 _ptr(slope), _ptr(q), _ptr(ws), ws.numel(), _stream(dev)))
    return t_out, slope, q


def conv_backward(p, cs, t_in, W, t_out, slope, q, grad_t_out, need_W=True, need_t_in=True,
                  ws=None, synfire: Optional[dstd_synfire_params] = None, grad_W=None):
    """Conv layer backward; returns (grad_W or None, grad_t_in or None), as
    `backward`."""
    torch = _torch()
    t_in = _cont(t_in, torch.float32)
    W = _cont(W)
    B = t_in.shape[0]
    dev = t_in.device
    gW = _grad_dest(torch, grad_W, W, W.shape, dev, need_W)
    gt = torch.empty(t_in.shape, dtype=torch.float32, device=dev) if need_t_in else None
    need = dstd_lif_conv_backward_workspace_size(p, cs, B)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    args = (B, _ptr(t_in), _ptr(W), _wdtype(W), _ptr(_cont(t_out, torch.float32)),
            _ptr(_cont(slope, torch.float32)), _ptr(_cont(q, torch.int32)),
            _ptr(_cont(grad_t_out, torch.float32)), _ptr(gW), _ptr(gt), _ptr(ws), ws.numel(),
            _stream(dev))
    if synfire is None:
        _check("dstd_lif_conv_backward", dstd_lif_conv_backward(p, cs, *args))
    else:
        _check("dstd_lif_conv_backward_synfire",
               dstd_lif_conv_backward_synfire(p, synfire, cs, *args))
    return gW, gt


def synfire_penalty(sp: dstd_synfire_params, t_out, W):
    """Values (T, Q) of the synfire terms as a device tensor [2]. t_out is
    [B, N_out] (dense) or [B, C_out, H_out, W_out] (conv); W is the layer's
    weight tensor (rows = its first dimension)."""
    torch = _torch()
    t_out = _cont(t_out, torch.float32)
    W = _cont(W)
    B = t_out.shape[0]
    rows = t_out.shape[1]
    spatial = 1
    for d in t_out.shape[2:]:
        spatial *= d
    row_len = W.numel() // max(W.shape[0], 1)
    dev = t_out.device
    value = torch.empty(2, dtype=torch.float32, device=dev)
    need = dstd_synfire_penalty_workspace_size(B, rows, spatial)
    ws = workspace(need, dev)
    _check("dstd_synfire_penalty",
           dstd_synfire_penalty(sp, B, rows, spatial, row_len, _ptr(t_out), _ptr(W), _wdtype(W),
                                _ptr(value), _ptr(ws), ws.numel(), _stream(dev)))
    return value


def softmax_ce_grad(t_out, labels, tau_soft: float = 1.0, t_cap: Optional[float] = None):
    """Returns (dL/dt [B, N], loss [B + 1]): loss[0] = L, loss[1 + b] = sample b's term."""
    torch = _torch()
    t_out = _cont(t_out, torch.float32)
    labels = _cont(labels, torch.int32)
    B, N = t_out.shape
    if t_cap is None:
        raise ValueError("t_cap is required (time used for outputs that did not fire)")
    grad = torch.empty_like(t_out)
    loss = torch.empty((B + 1,), dtype=torch.float32, device=t_out.device)
    _check("dstd_softmax_ce_grad",
           dstd_softmax_ce_grad(B, N, _ptr(t_out), _ptr(labels), float(tau_soft), float(t_cap),
                                _ptr(grad), _ptr(loss), _stream(t_out.device)))
    return grad, loss


def mse_grad(t_out, target):
    """Returns (dL/dt [B, N], loss [B + 1]): loss[0] = L, loss[1 + b] = sample b's term."""
    torch = _torch()
    t_out = _cont(t_out, torch.float32)
    target = _cont(target, torch.float32)
    B, N = t_out.shape
    grad = torch.empty_like(t_out)
    loss = torch.empty((B + 1,), dtype=torch.float32, device=t_out.device)
    _check("dstd_mse_grad", dstd_mse_grad(B, N, _ptr(t_out), _ptr(target), _ptr(grad), _ptr(loss),
                                          _stream(t_out.device)))
    return grad, loss


class TensorList:
    """The tensors of a training step and their table on the device (``c``: the
    C struct). It keeps the tensors and the table alive; a tensor that is
    replaced by another, or moved to other memory (``.data``, ``set_``,
    ``resize_``), needs a new list, and a graph that calls were captured into
    needs the list for as long as it is replayed.

    The table is written on the stream that is current when the list is built
    (``stream``; ``built``: the event behind it). Calls on another stream wait
    for it. A list built inside a capture (``captured``) has its table once the
    graph is replayed, and is for calls inside captures alone, whose graphs are
    replayed behind that one; streams that a capture forks are ordered by
    whoever forks them."""

    def __init__(self, c, mem, tensors, device, stream, built=None, captured=False):
        self.c, self.mem, self.tensors, self.device, self.stream = c, mem, tensors, device, stream
        self.built, self.captured = built, captured
        self.ws_bytes = dstd_tensor_list_workspace_size(c)


def _tensor(x, what):
    if not isinstance(x, _torch().Tensor):
        raise TypeError(f"{what} must be a tensor, got {type(x).__name__}")


def _list_array(torch, x, like, dev, dtypes, what, k):
    """Address of one array of tensor k of a list, checked."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what} {k} must be a tensor, got {type(x).__name__}")
    if x.dtype not in dtypes:
        raise TypeError(f"{what} {k} must be one of {list(dtypes)}, got {x.dtype}")
    if dev < 0 or x.get_device() != dev:
        raise ValueError(f"{what} {k} must live on the GPU of the list's other tensors")
    if x is not like and x.shape != like.shape:
        raise ValueError(f"{what} {k} has shape {tuple(x.shape)}, its gradient {tuple(like.shape)}")
    if not x.is_contiguous():
        raise ValueError(f"{what} {k} must be contiguous")
    return x.data_ptr()


def _per_tensor(x, n, what):
    x = [None] * n if x is None else list(x)
    if len(x) != n:
        raise ValueError(f"{len(x)} {what} for {n} gradients")
    return x


def make_tensor_list(grads, weights=None, m=None, v=None, master=None, out=None, lr_scale=None,
                     decay_scale=None) -> TensorList:
    """List of tensors for grad_norm, grad_clip and adamw_step. `grads` f32 or
    bf16 (the tensors that every backward writes: `grad_W` of the backward
    helpers); `weights` f32 or bf16 with their moments `m`, `v` (f32), and for bf16
    weights optionally their f32 copies `master`; `out` the tensors grad_clip
    writes (default: the gradients themselves); `lr_scale`, `decay_scale`
    factors per tensor (default 1). All contiguous, on one GPU; entries of
    master and out may be None."""
    torch = _torch()
    code = {torch.float32: DSTD_F32, torch.bfloat16: DSTD_BF16}
    f32 = (torch.float32,)
    grads = list(grads)
    n = len(grads)
    cols = [_per_tensor(x, n, what) for x, what in
            ((weights, "weights"), (m, "first moments"), (v, "second moments"),
             (master, "master weights"), (out, "outputs"))]
    scales = [[1.0] * n if x is None else _per_tensor(x, n, what) for x, what in
              ((lr_scale, "learning-rate factors"), (decay_scale, "decay factors"))]
    if n == 0:
        raise ValueError("a list needs a tensor")
    dev = grads[0].get_device() if isinstance(grads[0], torch.Tensor) else -1
    arr = (dstd_tensor * n)()
    for k, (t, g, w, mk, vk, w32, o, ls, ds) in enumerate(zip(arr, grads, *cols, *scales)):
        t.g = _list_array(torch, g, g, dev, code, "gradient", k)
        t.g_dtype, t.n = code[g.dtype], g.numel()
        if w is not None:
            t.w = _list_array(torch, w, g, dev, code, "weight", k)
            t.w_dtype = code[w.dtype]
        if mk is not None:
            t.m = _list_array(torch, mk, g, dev, f32, "first moment", k)
        if vk is not None:
            t.v = _list_array(torch, vk, g, dev, f32, "second moment", k)
        if w32 is not None:
            t.w32 = _list_array(torch, w32, g, dev, f32, "master weight", k)
        if o is not None:
            t.out = _list_array(torch, o, g, dev, code, "output", k)
            t.out_dtype = code[o.dtype]
        t.lr_scale, t.decay_scale = ls, ds
    device = torch.device("cuda", dev)
    mem = workspace(dstd_tensor_list_size(n, arr), device)
    c = dstd_tensor_list()
    stream = _stream(device)
    with torch.cuda.device(device):
        _check("dstd_tensor_list_build",
               dstd_tensor_list_build(n, arr, _ptr(mem), mem.numel(), c, stream))
        captured = torch.cuda.is_current_stream_capturing()
        built = None if captured else torch.cuda.current_stream(device).record_event()
    return TensorList(c, mem, (grads, *cols), device, stream, built, captured)


def _scalar(x, dtype, dev, what):
    if getattr(x, "dtype", None) != dtype or x.numel() != 1 or x.device != dev:
        _tensor(x, what)
        raise ValueError(f"{what} must hold one {dtype} on {dev}")
    return x.data_ptr()


def _optim_args(tl: TensorList, norm, norm_given, ws, want_norm):
    """(norm tensor or None, its pointer, workspace) of a call."""
    if norm is None:
        if norm_given:
            raise ValueError("norm_given needs the norm")
        if want_norm:
            torch = _torch()
            norm = torch.empty(1, dtype=torch.float32, device=tl.device)
    if ws is None or getattr(ws, "numel", int)() < tl.ws_bytes:
        if ws is not None:
            _tensor(ws, "ws")
        ws = workspace(tl.ws_bytes, tl.device)
    elif ws.device != tl.device:
        raise ValueError(f"ws must be on {tl.device}")
    elif not ws.is_contiguous():  # an expanded tensor has less memory than elements
        raise ValueError("ws must be contiguous")
    if norm is None:
        return None, None, ws
    return norm, _scalar(norm, _torch().float32, tl.device, "norm"), ws


def _behind_build(torch, tl: TensorList, dev):
    """Orders the current stream behind the launches that write the list's table,
    and the table's memory behind the current stream. A capture cannot wait for
    work outside it: its graph is replayed behind the build by whoever replays
    it (torch.cuda.graph waits for all earlier work before it captures)."""
    with torch.cuda.device(dev):
        capturing = torch.cuda.is_current_stream_capturing()
    if tl.captured and not capturing:
        raise RuntimeError("a list built inside a capture is for calls inside captures: "
                           "its table is written when the graph is replayed")
    stream = torch.cuda.current_stream(dev)
    if tl.built is not None and not capturing:
        if tl.built.query():
            tl.built = None
        else:
            stream.wait_event(tl.built)
    tl.mem.record_stream(stream)  # not reused before this stream has read it


def _launch(tl: TensorList, name, fn, *args):
    """One call on the list's device (launches go to the current one) and on
    that device's current stream."""
    torch = _torch()
    dev = tl.device.index
    stream = torch._C._cuda_getCurrentRawStream(dev)  # current_stream() builds an object: 2 us
    if stream != tl.stream or tl.captured:
        _behind_build(torch, tl, dev)
    if torch.cuda.current_device() == dev:
        _check(name, fn(*args, stream))
    else:
        with torch.cuda.device(dev):
            _check(name, fn(*args, stream))


def grad_norm(tl: TensorList, norm=None, ws=None):
    """L2 norm of all gradients of the list together, as a device tensor [1]
    (written to `norm` if given)."""
    norm, ptr, ws = _optim_args(tl, norm, False, ws, True)
    _launch(tl, "dstd_grad_norm", dstd_grad_norm, tl.c, ptr, _ptr(ws), ws.numel())
    return norm


def grad_clip(tl: TensorList, max_norm: float, norm=None, norm_given: bool = False, ws=None):
    """Clips the list's gradients to a norm of at most max_norm, in place or
    into the list's outputs; returns the norm before clipping, a device tensor
    [1]. With norm_given, `norm` is the norm to clip by."""
    norm, ptr, ws = _optim_args(tl, norm, norm_given, ws, True)
    _launch(tl, "dstd_grad_clip", dstd_grad_clip, tl.c, float(max_norm), ptr,
            1 if norm_given else 0, _ptr(ws), ws.numel())
    return norm


def make_adamw(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=1e-2,
               max_norm=math.inf) -> dstd_adamw_params:
    return dstd_adamw_params(float(lr), float(beta1), float(beta2), float(eps),
                             float(weight_decay), float(max_norm))


def adamw_step(tl: TensorList, hp: dstd_adamw_params, step, lr=None, norm=None,
               norm_given: bool = False, ws=None):
    """One AdamW step of the list's tensors, their gradients clipped to
    hp.max_norm on the way. `step` [1] int64: steps done, on the device, counted
    up (one for each list); `lr` [1] f32 on the device replaces hp.lr. Returns the norm before
    clipping (None where none is formed: no `norm` given and hp.max_norm infinite);
    a step whose norm is not finite changes nothing. (Finite gradients whose norm
    leaves fp32 are clipped and the step is made, though the norm reads inf.)"""
    norm, ptr, ws = _optim_args(tl, norm, norm_given, ws, math.isfinite(hp.max_norm))
    torch = _torch()
    _launch(tl, "dstd_adamw_step", dstd_adamw_step, tl.c, hp,
            None if lr is None else _scalar(lr, torch.float32, tl.device, "lr"),
            _scalar(step, torch.int64, tl.device, "step"), ptr, 1 if norm_given else 0, _ptr(ws),
            ws.numel())
    return norm
