"""ctypes binding of libprq.so (include/prq.h) -- argument marshalling only.

Every step of the hot path runs in the library: ``prq_prepare`` in its native
host code, ``prq_quant_act`` / ``prq_gemm`` / ``prq_grouped_gemm`` in its HIP
kernels.  torch supplies device memory (``data_ptr()``) and the stream
(``torch.cuda.current_stream().cuda_stream``); torch is imported before the
library is loaded so both use one HIP runtime instance.  There is no fallback:
a missing library raises ``ImportError`` at import time.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct

import numpy as np
import torch  # noqa: F401  (loads the HIP runtime the library binds to)

from . import build as _build

PRQ_OK, PRQ_EINVAL, PRQ_EALIGN, PRQ_EDEVICE, PRQ_EUNSUPPORTED, PRQ_EWORKSPACE = 0, -1, -2, -3, -4, -5
SCALE_MODES = {"smooth": 0, "act_only": 1, "none": 2}
GEMM_AUTO, GEMM_TILE, GEMM_STREAM, GEMM_STREAM_K = 0, 1, 2, 3
HEADER = os.path.join(_build.INCLUDE, "prq.h")

if not os.path.exists(_build.LIB):
    raise ImportError(f"{_build.LIB} is not built; run `python -m paper_2609_22106_amd.build`")
_lib = ctypes.CDLL(_build.LIB)

_p = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_sz = ctypes.c_size_t


def _decl(name, restype, argtypes):
    fn = getattr(_lib, name)
    fn.restype = restype
    fn.argtypes = argtypes
    return fn


_strerror = _decl("prq_strerror", ctypes.c_char_p, [ctypes.c_int])
_abi_version = _decl("prq_abi_version", ctypes.c_int, [])
_prepare = _decl("prq_prepare", ctypes.c_int,
                 [_p, _i32, _i32, _p, _i32, ctypes.c_double, _i32, _i32, _p, _p, _p, _p, _p, _p, _p])
_prepare_ex = _decl("prq_prepare_ex", ctypes.c_int,
                    [_p, _i32, _i32, _p, _i32, ctypes.c_double, _i32, _i32, _i32, _p, _p, _p, _p, _p,
                     _p, _p])
PREPARE_E8M0_SEARCH = 1
_expand = _decl("prq_expand_producer", ctypes.c_int, [_p, _p, _i32, _i32, _p, _p, _i32, _p, _p])
_evaluate = _decl("prq_evaluate_nrmse", ctypes.c_int,
                  [_p, _i32, _i32, _p, _i32, _p, _i32, ctypes.c_double, _i32, _i32, _i32, _p, _p])
_search = _decl("prq_search_alpha", ctypes.c_int,
                [_p, _i32, _i32, _p, _i32, _p, _i32, _i32, _i32, _i32, _p, _p, _p])
_quant_act = _decl("prq_quant_act", ctypes.c_int,
                   [_p, _i64, _i32, _i32, _i32, _p, _p, _p, _i32, _p, _p, _p])
_packed_bytes = _decl("prq_packed_weight_bytes", ctypes.c_int,
                      [_i32, _i32, _i32, ctypes.POINTER(_sz), ctypes.POINTER(_sz)])
_pack = _decl("prq_pack_weight", ctypes.c_int, [_p, _p, _i32, _i32, _i32, _p, _p, _p])
_gemm_ws = _decl("prq_gemm_workspace_bytes", _sz, [_i32, _i32, _i32])
_gemm_ws_ex = _decl("prq_gemm_workspace_bytes_ex", _sz, [_i32, _i32, _i32, _i32, _i32])
_gemm = _decl("prq_gemm", ctypes.c_int, [_p, _p, _i32, _p, _p, _i32, _i32, _p, _p, _sz, _p])
_gemm_ex = _decl("prq_gemm_ex", ctypes.c_int,
                 [_p, _p, _i32, _p, _p, _i32, _i32, _p, _p, _sz, _i32, _i32, _p])
_gemm_noalloc = _decl("prq_gemm_noalloc", ctypes.c_int, [_p, _p, _i32, _p, _p, _i32, _i32, _p, _p])
_gemm_noalloc_max = _decl("prq_gemm_noalloc_max_workspace_bytes", _sz, [])
_packed_act_bytes = _decl("prq_packed_act_bytes", ctypes.c_int,
                          [_i32, _i32, ctypes.POINTER(_sz), ctypes.POINTER(_sz)])
_quant_act_packed = _decl("prq_quant_act_packed", ctypes.c_int,
                          [_p, _i64, _i32, _i32, _i32, _p, _p, _p, _i32, _p, _p, _p])
_swiglu_quant = _decl("prq_swiglu_quant", ctypes.c_int, [_p, _p, _i64, _i32, _i32, _p, _p, _p])
_swiglu_quant_packed = _decl("prq_swiglu_quant_packed", ctypes.c_int,
                             [_p, _p, _i64, _i32, _i32, _p, _p, _p])
_gemm_packed_ws = _decl("prq_gemm_packed_workspace_bytes", _sz, [_i32, _i32, _i32])
_gemm_packed = _decl("prq_gemm_packed", ctypes.c_int,
                     [_p, _p, _i32, _p, _p, _i32, _i32, _p, _p, _sz, _p])
_ggemm_packed = _decl("prq_grouped_gemm_packed", ctypes.c_int,
                      [_p, _p, _p, _i32, _i32, _p, _p, _i32, _i32, _p, _p])
_ggemm_ws = _decl("prq_grouped_gemm_workspace_bytes", _sz, [_i32, _i32, _i32, _i32])
_ggemm = _decl("prq_grouped_gemm", ctypes.c_int,
               [_p, _p, _p, _i32, _i32, _p, _p, _i32, _i32, _p, _p, _sz, _p])
_ggemm_ex = _decl("prq_grouped_gemm_ex", ctypes.c_int,
                  [_p, _p, _p, _i32, _i32, _p, _p, _i32, _i32, _p, _p, _sz, _i32, _p])

PRQ_F32, PRQ_BF16 = 0, 1
_f32 = ctypes.c_float
_qk_norm_rope = _decl("prq_qk_norm_rope", ctypes.c_int,
                      [_p, _i64, _p, _i64, _p, _i64, _i32, _i32, _i32, _i32, _i32, _p, _p, _i32, _f32, _p, _p, _i32,
                       _i32, _i32, _p, _p, _p, _i64, _i32, _i32, _p, _p])
_tree_ws = _decl("prq_tree_attention_workspace_bytes", _sz, [_i32, _i32, _i32, _i32, _i32, _i32])
_tree = _decl("prq_tree_attention", ctypes.c_int,
              [_p, _i64, _i32, _i32, _i32, _i32, _p, _p, _i64, _i32, _i32, _p, _i64, _i32, _p, _p, _i32, _i32, _f32,
               _p, _i64, _i32, _p, _p, _p, _sz, _p])
_lora_ws = _decl("prq_lora_workspace_bytes", _sz, [_i32, _i32, _i32, _i32, _i32])
_lora = _decl("prq_lora", ctypes.c_int,
              [_p, _i64, _i32, _i32, _p, _p, _p, _p, _i32, _i32, _i32, _p, _p, _i32, _i32, _p, _i64, _p, _i64, _p,
               _sz, _p])
_lora_ex = _decl("prq_lora_ex", ctypes.c_int,
                 [_p, _i64, _i32, _i32, _p, _p, _p, _p, _p, _i32, _i32, _i32, _p, _p, _i32, _i32, _p, _i64, _p, _i64,
                  _p, _sz, _p])

ROUTE_SCORINGS = {"softmax": 0, "sigmoid": 1}


def _record(name, argtypes):
    """(pack, call) of prq_<name>_record: call(pack(*arguments)), with 0 for no pointer."""
    kinds = {_p: "Q", _sz: "Q", _i32: "q", _i64: "q", _f32: "d"}
    return (struct.Struct("=" + "".join(kinds[t] for t in argtypes)).pack,
            _decl(name + "_record", ctypes.c_int, [ctypes.c_char_p]))


_block_norm_types = [_p, _i64, _i32, _p, _i64, _i32, _i32, _i32, _p, _p, _i32, _f32, _p, _i64, _i32, _i32, _p, _f32,
                     _f32, _f32, _p, _i64, _p, _i64, _p]
_block_norm = _decl("prq_block_norm", ctypes.c_int, _block_norm_types)
_block_norm_pack, _block_norm_call = _record("prq_block_norm", _block_norm_types)
_route_ws = _decl("prq_moe_route_workspace_bytes", _sz, [_i32, _i32, _i32])
_route_types = [_p, _i64, _i32, _i32, _p, _i64, _i32, _i32, _i32, _p, _i32, _f32, _p, _p, _p, _i64, _p, _sz, _p]
_route = _decl("prq_moe_route", ctypes.c_int, _route_types)
_route_pack, _route_call = _record("prq_moe_route", _route_types)
_moe_ws = _decl("prq_moe_layer_workspace_bytes", _sz, [_i32, _i32, _i32, _i32, _i32, _i32, _i32])
_moe_types = [_p, _i64, _i32, _p, _p, _i32, _p, _p, _p, _p, _i32, _i32, _i32, _i32, _i32, _p, _i64, _p, _sz, _p]
_moe = _decl("prq_moe_layer", ctypes.c_int, _moe_types)
_moe_pack, _moe_call = _record("prq_moe_layer", _moe_types)


class PRQError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {prq_strerror(status)} (status {status})")


def _check(status, where):
    if status != PRQ_OK:
        raise PRQError(status, where)


def prq_strerror(status):
    return _strerror(int(status)).decode()


def prq_abi_version():
    return int(_abi_version())


def exported_symbols():
    """Names of the functions include/prq.h declares."""
    text = open(HEADER).read()
    return sorted(set(re.findall(r"\b(prq_\w+)\s*\(", text)))


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


# The current stream's handle without a torch.cuda.Stream object around it (3.5 of
# the 11 us that a call took on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_of_call(stream):
    """_stream for calls that have been given GPU tensors."""
    if stream is None and _raw_stream is not None and _cur_device is not None:
        return _raw_stream(_cur_device())
    return _stream(stream)


def _stream_at(stream):
    """_stream_of_call as a number."""
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_cur_device()) if _raw_stream is not None and _cur_device is not None else _stream(None).value or 0


def _alloc(make, shape, dtype, device, stream, kept=True):
    """make(shape) for a call on `stream`, which may not be the current one: made
    under that stream, so that the call is ordered after a fill and after the last
    use of memory that another tensor gave back.  kept: a tensor that the caller
    gets and uses on the current stream too (it holds its memory until that is done)."""
    device = torch.device(device)
    if stream is None or device.type != "cuda":
        return make(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        t = make(shape, dtype=dtype, device=device)
    current = torch.cuda.current_stream(device)
    if kept and current != stream:
        t.record_stream(current)
    return t


# --------------------------------------------------------------- prepare ---
def prq_prepare(W_bf16, Xcal_bf16, alpha, k_tail, scale_mode="smooth", with_col_err=False,
                scale_search=False):
    """Offline calibration/export (host).  W_bf16 [N, K] and Xcal_bf16 [T, K]
    are uint16 numpy arrays of bf16 bit patterns.  Returns numpy arrays.
    scale_search: the weight-side E8M0 block-scale search (prq_prepare_ex)."""
    W = np.ascontiguousarray(W_bf16, dtype=np.uint16)
    X = np.ascontiguousarray(Xcal_bf16, dtype=np.uint16)
    N, K = W.shape
    T = X.shape[0]
    if X.shape[1] != K:
        raise ValueError("calibration activations must have K columns")
    K_aug = K + int(k_tail)
    out = {
        "scale": np.empty(K, np.float32), "inv_scale": np.empty(K, np.float32),
        "perm": np.empty(K, np.int32), "inv_scale_pos": np.empty(K, np.float32),
        "Wq": np.empty((N, max(K_aug, 0) // 2), np.uint8),
        "Wsc": np.empty((N, max(K_aug, 0) // 32), np.uint8),
    }
    col_err = np.empty(K, np.float64) if with_col_err else None
    st = _prepare_ex(_ptr(W), N, K, _ptr(X), T, float(alpha), int(k_tail), SCALE_MODES[scale_mode],
                     PREPARE_E8M0_SEARCH if scale_search else 0,
                     _ptr(out["scale"]), _ptr(out["inv_scale"]), _ptr(out["perm"]),
                     _ptr(out["inv_scale_pos"]), _ptr(out["Wq"]), _ptr(out["Wsc"]), _ptr(col_err))
    _check(st, "prq_prepare")
    if with_col_err:
        out["col_err"] = col_err
    return out


def prq_expand_producer(W_up_bf16, W_gate_bf16, inv_scale, perm, k_tail):
    """Offline copy (host): (W_up_aug, W_gate_aug or None), each [C + k, H]
    bf16 bit patterns (uint16)."""
    up = _bf16_host(W_up_bf16, "W_up")
    gate = None if W_gate_bf16 is None else _bf16_host(W_gate_bf16, "W_gate")
    C, H = up.shape
    if gate is not None and gate.shape != up.shape:
        raise ValueError("W_gate must have W_up's shape")
    inv = np.ascontiguousarray(inv_scale, dtype=np.float32)
    p = np.ascontiguousarray(perm, dtype=np.int32)
    if inv.shape != (C,) or p.shape != (C,):
        raise ValueError("inv_scale and perm must have C entries")
    up_aug = np.empty((C + int(k_tail), H), np.uint16)
    gate_aug = None if gate is None else np.empty((C + int(k_tail), H), np.uint16)
    _check(_expand(_ptr(up), _ptr(gate), C, H, _ptr(inv), _ptr(p), int(k_tail), _ptr(up_aug),
                   _ptr(gate_aug)), "prq_expand_producer")
    return up_aug, gate_aug


# ------------------------------------------------------------ evaluation ---
def _bf16_host(a, name):
    a = np.ascontiguousarray(a)
    if a.dtype not in (np.uint16, np.int16) or a.ndim != 2:
        raise ValueError(f"{name} must be a 2-D array of bf16 bit patterns (uint16)")
    return a


def prq_evaluate_nrmse(W_bf16, Xcal_bf16, X_bf16, alpha, k_tail, scale_mode="smooth",
                       scale_search=False, stream=None):
    """y-NRMSE of one configuration on the rows X (offline; host arrays)."""
    W, Xc, X = _bf16_host(W_bf16, "W"), _bf16_host(Xcal_bf16, "Xcal"), _bf16_host(X_bf16, "X")
    N, K = W.shape
    if Xc.shape[1] != K or X.shape[1] != K:
        raise ValueError("activations must have K columns")
    out = ctypes.c_double()
    st = _evaluate(_ptr(W), N, K, _ptr(Xc), Xc.shape[0], _ptr(X), X.shape[0], float(alpha),
                   int(k_tail), SCALE_MODES[scale_mode], PREPARE_E8M0_SEARCH if scale_search else 0,
                   ctypes.byref(out), _stream(stream))
    _check(st, "prq_evaluate_nrmse")
    return float(out.value)


def prq_search_alpha(W_bf16, Xcal_bf16, alphas, k_tail, scale_mode="smooth", scale_search=False,
                     stream=None):
    """Algorithm 1's alpha search (offline): (best alpha, y-NRMSE per alpha)."""
    W, Xc = _bf16_host(W_bf16, "W"), _bf16_host(Xcal_bf16, "Xcal")
    N, K = W.shape
    if Xc.shape[1] != K:
        raise ValueError("calibration activations must have K columns")
    a = np.ascontiguousarray(alphas, dtype=np.float64)
    err = np.empty(a.size, np.float64)
    best = ctypes.c_int32()
    st = _search(_ptr(W), N, K, _ptr(Xc), Xc.shape[0], _ptr(a), a.size, int(k_tail),
                 SCALE_MODES[scale_mode], PREPARE_E8M0_SEARCH if scale_search else 0, _ptr(err),
                 ctypes.byref(best), _stream(stream))
    _check(st, "prq_search_alpha")
    return float(a[best.value]), err


# ------------------------------------------------------------- device ops ---
# The library receives bare pointers and cannot see buffer extents, so the
# binding checks every tensor against the sizes it passes (shape, dtype,
# contiguity) and that it lives on a GPU, before anything is launched.
def _need(t, name, dtype, shape=None, min_numel=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if min_numel is not None and t.numel() < min_numel:
        raise ValueError(f"{name} has {t.numel()} elements, needs at least {min_numel}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _on_gpu(**tensors):
    for name, t in tensors.items():
        if t is not None and not t.is_cuda:
            raise ValueError(f"{name} must be a GPU tensor")


_BF16_LIKE = (torch.int16, torch.uint16, torch.bfloat16)
_U8, _F32, _I32 = torch.uint8, torch.float32, torch.int32


# The same checks in one expression per tensor, for the calls of an inference
# step: whatever does not pass goes through the checks above, which say why.
def _is(t, dtype, shape):
    return (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.is_cuda
            and t.is_contiguous())


def _holds(t, dtype, numel):
    return (type(t) is torch.Tensor and t.dtype is dtype and t.numel() >= numel and t.is_cuda
            and t.is_contiguous())


def _packed_sizes(blocks, K_aug):
    """Code and scale bytes of `blocks` 16-row blocks (prq_packed_act_bytes,
    prq_packed_weight_bytes), or (None, None) where those refuse K_aug."""
    if K_aug <= 0 or K_aug % 32 or K_aug > 65536:
        return None, None
    steps = (K_aug + 127) // 128
    return blocks * steps * 1024, blocks * ((steps + 3) // 4) * 256


def _weight_fits(W):
    if not (1 <= W.E <= 4096 and W.N > 0 and W.N % 16 == 0):
        return False
    cb, sb = _packed_sizes(W.E * (W.N // 16), W.K_aug)
    return cb is not None and _holds(W.Wp, _U8, cb) and _holds(W.Wps, _U8, sb)


def _packed_act_fits(A):
    cb, sb = _packed_sizes((A.M + 15) // 16, A.K_aug) if A.M >= 0 else (None, None)
    return cb is not None and _holds(A.Ap, _U8, cb) and _holds(A.Aps, _U8, sb)


def _scales_fit(inv_scale_pos, perm, group_offsets, G, K):
    return ((inv_scale_pos is None or _holds(inv_scale_pos, _F32, G * K))
            and (perm is None or _holds(perm, _I32, G * K))
            and (G <= 1 or (group_offsets is not None and _holds(group_offsets, _I32, G + 1))))


def _workspace_arg(workspace):
    """(address, bytes) of a workspace argument."""
    if workspace is None:
        return None, 0
    if not _holds(workspace, _U8, 0):
        _need(workspace, "workspace", torch.uint8)
        _on_gpu(workspace=workspace)
    return workspace.data_ptr(), workspace.numel()


def _check_scales(inv_scale_pos, perm, group_offsets, G, K):
    if inv_scale_pos is not None:
        _need(inv_scale_pos, "inv_scale_pos", torch.float32, min_numel=G * K)
    if perm is not None:
        _need(perm, "perm", torch.int32, min_numel=G * K)
    if G > 1:
        if group_offsets is None:
            raise ValueError("G > 1 needs group_offsets")
        _need(group_offsets, "group_offsets", torch.int32, min_numel=G + 1)


def prq_quant_act(X, K, k_tail, inv_scale_pos=None, perm=None, group_offsets=None, G=1,
                  Aq=None, Asc=None, stream=None):
    """Quantize bf16 activations X [M, ld] (device) -> (Aq [M, K_aug/2], Asc [M, K_aug/32]).
    inv_scale_pos[p] = 1/s_{perm[p]} (prq_prepare's ``inv_scale_pos``)."""
    if not isinstance(X, torch.Tensor) or X.dim() != 2 or X.dtype not in _BF16_LIKE:
        raise ValueError("X must be a 2-D tensor of bf16 values (or their int16 bit patterns)")
    M = X.shape[0]
    K_aug = K + k_tail
    if X.shape[1] < K or (M > 1 and X.stride(0) < K) or X.stride(1) != 1:
        raise ValueError(f"X rows must hold K={K} contiguous values (shape {tuple(X.shape)}, "
                         f"strides {X.stride()})")
    if Aq is None:
        Aq = _alloc(torch.empty, (M, K_aug // 2), torch.uint8, X.device, stream)
    if Asc is None:
        Asc = _alloc(torch.empty, (M, K_aug // 32), torch.uint8, X.device, stream)
    if not (X.is_cuda and _is(Aq, _U8, (M, K_aug // 2)) and _is(Asc, _U8, (M, K_aug // 32))
            and _scales_fit(inv_scale_pos, perm, group_offsets, G, K)):
        _need(Aq, "Aq", torch.uint8, (M, K_aug // 2))
        _need(Asc, "Asc", torch.uint8, (M, K_aug // 32))
        _check_scales(inv_scale_pos, perm, group_offsets, G, K)
        _on_gpu(X=X, Aq=Aq, Asc=Asc, inv_scale_pos=inv_scale_pos, perm=perm,
                group_offsets=group_offsets if G > 1 else None)
    ld = X.stride(0) if M > 1 else K
    st = _quant_act(X.data_ptr(), ld, M, K, k_tail, _ptr(inv_scale_pos), _ptr(perm), _ptr(group_offsets), G,
                    Aq.data_ptr(), Asc.data_ptr(), _stream_of_call(stream))
    _check(st, "prq_quant_act")
    return Aq, Asc


class PackedWeight:
    """Device buffers of a weight in the GEMM's packed layout (include/prq.h)."""

    def __init__(self, Wp, Wps, E, N, K_aug):
        self.Wp, self.Wps, self.E, self.N, self.K_aug = Wp, Wps, E, N, K_aug

    def check_sizes(self):
        cb, sb = prq_packed_weight_bytes(self.E, self.N, self.K_aug)
        _need(self.Wp, "W.Wp", torch.uint8, min_numel=cb)
        _need(self.Wps, "W.Wps", torch.uint8, min_numel=sb)


def _check_gemm_operands(Aq, Asc, W, Y, M):
    if (_is(Aq, _U8, (M, W.K_aug // 2)) and _is(Asc, _U8, (M, W.K_aug // 32)) and _is(Y, _F32, (M, W.N))
            and _weight_fits(W)):
        return
    _need(Aq, "Aq", torch.uint8, (M, W.K_aug // 2))
    _need(Asc, "Asc", torch.uint8, (M, W.K_aug // 32))
    _need(Y, "Y", torch.float32, (M, W.N))
    W.check_sizes()
    _on_gpu(Aq=Aq, Asc=Asc, Y=Y, Wp=W.Wp, Wps=W.Wps)


def prq_packed_weight_bytes(E, N, K_aug):
    cb, sb = _sz(0), _sz(0)
    _check(_packed_bytes(E, N, K_aug, ctypes.byref(cb), ctypes.byref(sb)), "prq_packed_weight_bytes")
    return int(cb.value), int(sb.value)


def prq_pack_weight(Wq, Wsc, stream=None):
    """Canonical device Wq [N, K_aug/2] / Wsc [N, K_aug/32] (or [E, N, ...]) ->
    PackedWeight in the layout the GEMM kernels read."""
    if not isinstance(Wq, torch.Tensor) or Wq.dim() not in (2, 3):
        raise ValueError("Wq must be a [N, K_aug/2] or [E, N, K_aug/2] tensor")
    E = Wq.shape[0] if Wq.dim() == 3 else 1
    N = Wq.shape[-2]
    K_aug = Wq.shape[-1] * 2
    _need(Wq, "Wq", torch.uint8)
    _need(Wsc, "Wsc", torch.uint8, tuple(Wq.shape[:-1]) + (K_aug // 32,))
    _on_gpu(Wq=Wq, Wsc=Wsc)
    cb, sb = prq_packed_weight_bytes(E, N, K_aug)
    Wp = _alloc(torch.empty, cb, torch.uint8, Wq.device, stream)
    Wps = _alloc(torch.empty, sb, torch.uint8, Wq.device, stream)
    _check(_pack(_ptr(Wq), _ptr(Wsc), E, N, K_aug, _ptr(Wp), _ptr(Wps), _stream(stream)),
           "prq_pack_weight")
    return PackedWeight(Wp, Wps, E, N, K_aug)


def prq_gemm_workspace_bytes(M, N, K_aug, variant=GEMM_AUTO, splits=0):
    return int(_gemm_ws_ex(M, N, K_aug, variant, splits))


def prq_gemm(Aq, Asc, W, Y=None, workspace=None, variant=GEMM_AUTO, splits=0, stream=None):
    """Y [M, N] float32 = deq(A_aug) deq(W_aug)^T over K_aug (device); W is a
    PackedWeight (E = 1)."""
    M = Aq.shape[0]
    N, K_aug = W.N, W.K_aug
    if W.E != 1:
        raise ValueError("prq_gemm takes a single weight (E = 1); use prq_grouped_gemm")
    if Y is None:
        Y = _alloc(torch.empty, (M, N), torch.float32, W.Wp.device, stream)
    _check_gemm_operands(Aq, Asc, W, Y, M)
    if workspace is None:
        need = prq_gemm_workspace_bytes(M, N, K_aug, variant, splits)
        if need:
            workspace = _alloc(torch.zeros, need, torch.uint8, W.Wp.device, stream, kept=False)
    ws, ws_bytes = _workspace_arg(workspace)
    st = _gemm_ex(Aq.data_ptr(), Asc.data_ptr(), M, W.Wp.data_ptr(), W.Wps.data_ptr(), N, K_aug,
                  Y.data_ptr(), ws, ws_bytes, variant, splits, _stream_of_call(stream))
    _check(st, "prq_gemm")
    return Y


def prq_gemm_noalloc_max_workspace_bytes():
    return int(_gemm_noalloc_max())


def prq_gemm_noalloc(Aq, Asc, W, Y, stream=None):
    """prq_gemm (AUTO) with the library's own device scratch as its workspace:
    nothing is allocated, Y [M, N] float32 must be given."""
    M = Aq.shape[0]
    if W.E != 1:
        raise ValueError("prq_gemm_noalloc takes a single weight (E = 1)")
    _check_gemm_operands(Aq, Asc, W, Y, M)
    st = _gemm_noalloc(Aq.data_ptr(), Asc.data_ptr(), M, W.Wp.data_ptr(), W.Wps.data_ptr(), W.N, W.K_aug,
                       Y.data_ptr(), _stream_of_call(stream))
    _check(st, "prq_gemm_noalloc")
    return Y


class PackedAct:
    """Device buffers of an activation in the packed layout (include/prq.h)."""

    def __init__(self, Ap, Aps, M, K_aug):
        self.Ap, self.Aps, self.M, self.K_aug = Ap, Aps, M, K_aug

    def check_sizes(self):
        cb, sb = prq_packed_act_bytes(self.M, self.K_aug)
        _need(self.Ap, "A.Ap", torch.uint8, min_numel=cb)
        _need(self.Aps, "A.Aps", torch.uint8, min_numel=sb)


def prq_packed_act_bytes(M, K_aug):
    cb, sb = _sz(0), _sz(0)
    _check(_packed_act_bytes(M, K_aug, ctypes.byref(cb), ctypes.byref(sb)), "prq_packed_act_bytes")
    return int(cb.value), int(sb.value)


def prq_quant_act_packed(X, K, k_tail, inv_scale_pos=None, perm=None, out=None, stream=None,
                         group_offsets=None, G=1):
    """prq_quant_act into the packed activation layout -> PackedAct.
    out: a PackedAct of the same M and K_aug to write into (else allocated).
    G > 1: rows sorted by group, group_offsets [G + 1] device int32, and
    inv_scale_pos / perm hold G rows of K (one per expert)."""
    if not isinstance(X, torch.Tensor) or X.dim() != 2 or X.dtype not in _BF16_LIKE:
        raise ValueError("X must be a 2-D tensor of bf16 values (or their int16 bit patterns)")
    M = X.shape[0]
    K_aug = K + k_tail
    if X.shape[1] < K or (M > 1 and X.stride(0) < K) or X.stride(1) != 1:
        raise ValueError(f"X rows must hold K={K} contiguous values (shape {tuple(X.shape)}, "
                         f"strides {X.stride()})")
    if out is None:
        cb, sb = prq_packed_act_bytes(M, K_aug)
        out = PackedAct(_alloc(torch.empty, cb, torch.uint8, X.device, stream),
                        _alloc(torch.empty, sb, torch.uint8, X.device, stream), M, K_aug)
    if out.M != M or out.K_aug != K_aug:
        raise ValueError(f"out holds {out.M} rows of K_aug {out.K_aug}, expected {M} x {K_aug}")
    if not (X.is_cuda and _packed_act_fits(out) and _scales_fit(inv_scale_pos, perm, group_offsets, G, K)):
        out.check_sizes()
        _check_scales(inv_scale_pos, perm, group_offsets, G, K)
        _on_gpu(X=X, Ap=out.Ap, Aps=out.Aps, inv_scale_pos=inv_scale_pos, perm=perm,
                group_offsets=group_offsets if G > 1 else None)
    ld = X.stride(0) if M > 1 else K
    st = _quant_act_packed(X.data_ptr(), ld, M, K, k_tail, _ptr(inv_scale_pos), _ptr(perm),
                           _ptr(group_offsets) if G > 1 else None, G, out.Ap.data_ptr(), out.Aps.data_ptr(),
                           _stream_of_call(stream))
    _check(st, "prq_quant_act_packed")
    return out


def prq_swiglu_quant(gate, up, K_aug, packed=False, out=None, stream=None):
    """Q(SiLU(gate) * up) of the expanded producers' bf16 outputs [M, >= K_aug]
    (offline copy, producer side): row-major (Aq, Asc) or, with packed=True, a
    PackedAct.  out: (Aq, Asc) or a PackedAct to write into (else allocated)."""
    for name, t in (("gate", gate), ("up", up)):
        if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.dtype not in _BF16_LIKE:
            raise ValueError(f"{name} must be a 2-D tensor of bf16 values (or their int16 bit patterns)")
        if t.shape[1] < K_aug or t.stride(1) != 1:
            raise ValueError(f"{name} rows must hold K_aug={K_aug} contiguous values "
                             f"(shape {tuple(t.shape)}, strides {t.stride()})")
    if gate.shape != up.shape or gate.stride() != up.stride():
        raise ValueError(f"gate {tuple(gate.shape)} / {gate.stride()} and up {tuple(up.shape)} / "
                         f"{up.stride()} must have the same shape and strides")
    M = gate.shape[0]
    ld = gate.stride(0) if M > 1 else K_aug
    if packed:
        if out is None:
            cb, sb = prq_packed_act_bytes(M, K_aug)
            out = PackedAct(_alloc(torch.empty, cb, torch.uint8, gate.device, stream),
                            _alloc(torch.empty, sb, torch.uint8, gate.device, stream), M, K_aug)
        if out.M != M or out.K_aug != K_aug:
            raise ValueError(f"out holds {out.M} rows of K_aug {out.K_aug}, expected {M} x {K_aug}")
        if not _packed_act_fits(out):
            out.check_sizes()
        A, As = out.Ap, out.Aps
    else:
        if out is None:
            out = (_alloc(torch.empty, (M, K_aug // 2), torch.uint8, gate.device, stream),
                   _alloc(torch.empty, (M, K_aug // 32), torch.uint8, gate.device, stream))
        A, As = out
        if not (_is(A, _U8, (M, K_aug // 2)) and _is(As, _U8, (M, K_aug // 32))):
            _need(A, "Aq", torch.uint8, (M, K_aug // 2))
            _need(As, "Asc", torch.uint8, (M, K_aug // 32))
    _on_gpu(gate=gate, up=up, A=A, As=As)
    fn = _swiglu_quant_packed if packed else _swiglu_quant
    st = fn(gate.data_ptr(), up.data_ptr(), ld, M, K_aug, A.data_ptr(), As.data_ptr(), _stream_of_call(stream))
    _check(st, "prq_swiglu_quant_packed" if packed else "prq_swiglu_quant")
    return out


def prq_gemm_packed_workspace_bytes(M, N, K_aug):
    return int(_gemm_packed_ws(M, N, K_aug))


def prq_gemm_packed(A, W, Y=None, workspace=None, stream=None):
    """Y [M, N] float32 = Eq. 3 over K_aug for a PackedAct A and a PackedWeight W (E = 1).
    workspace: uint8 device tensor of prq_gemm_packed_workspace_bytes (split along
    K when the planner wants it; without it the call runs unsplit)."""
    if W.E != 1:
        raise ValueError("prq_gemm_packed takes a single weight (E = 1)")
    if A.K_aug != W.K_aug:
        raise ValueError(f"K_aug differs: activation {A.K_aug}, weight {W.K_aug}")
    M, N = A.M, W.N
    if Y is None:
        Y = _alloc(torch.empty, (M, N), torch.float32, W.Wp.device, stream)
    if not (_is(Y, _F32, (M, N)) and _packed_act_fits(A) and _weight_fits(W)):
        _need(Y, "Y", torch.float32, (M, N))
        A.check_sizes()
        W.check_sizes()
        _on_gpu(Ap=A.Ap, Aps=A.Aps, Y=Y, Wp=W.Wp, Wps=W.Wps)
    ws, ws_bytes = _workspace_arg(workspace)
    st = _gemm_packed(A.Ap.data_ptr(), A.Aps.data_ptr(), M, W.Wp.data_ptr(), W.Wps.data_ptr(), N, W.K_aug,
                      Y.data_ptr(), ws, ws_bytes, _stream_of_call(stream))
    _check(st, "prq_gemm_packed")
    return Y


def prq_grouped_gemm_packed(A, group_offsets, W, Y=None, stream=None):
    """prq_grouped_gemm on a PackedAct A (rows sorted by expert, from
    prq_quant_act_packed with the same group_offsets); Y [M_total, N] float32."""
    if A.K_aug != W.K_aug:
        raise ValueError(f"K_aug differs: activation {A.K_aug}, weight {W.K_aug}")
    M, E, N = A.M, W.E, W.N
    if Y is None:
        Y = _alloc(torch.empty, (M, N), torch.float32, W.Wp.device, stream)
    if not (_is(Y, _F32, (M, N)) and _is(group_offsets, _I32, (E + 1,)) and _packed_act_fits(A)
            and _weight_fits(W)):
        _need(Y, "Y", torch.float32, (M, N))
        _need(group_offsets, "group_offsets", torch.int32, (E + 1,))
        A.check_sizes()
        W.check_sizes()
        _on_gpu(Ap=A.Ap, Aps=A.Aps, Y=Y, Wp=W.Wp, Wps=W.Wps, group_offsets=group_offsets)
    st = _ggemm_packed(A.Ap.data_ptr(), A.Aps.data_ptr(), group_offsets.data_ptr(), E, M, W.Wp.data_ptr(),
                       W.Wps.data_ptr(), N, W.K_aug, Y.data_ptr(), _stream_of_call(stream))
    _check(st, "prq_grouped_gemm_packed")
    return Y


def prq_grouped_gemm_workspace_bytes(M_total, E, N, K_aug):
    return int(_ggemm_ws(M_total, E, N, K_aug))


def prq_grouped_gemm(Aq, Asc, group_offsets, W, Y=None, workspace=None, variant=GEMM_AUTO,
                     stream=None):
    """Rows sorted by expert; W a PackedWeight of E experts; Y [M_total, N] float32."""
    M = Aq.shape[0]
    E, N, K_aug = W.E, W.N, W.K_aug
    if Y is None:
        Y = _alloc(torch.empty, (M, N), torch.float32, W.Wp.device, stream)
    if not _is(group_offsets, _I32, (E + 1,)):
        _need(group_offsets, "group_offsets", torch.int32, (E + 1,))
    _check_gemm_operands(Aq, Asc, W, Y, M)
    _on_gpu(group_offsets=group_offsets)
    ws, ws_bytes = _workspace_arg(workspace)
    st = _ggemm_ex(Aq.data_ptr(), Asc.data_ptr(), group_offsets.data_ptr(), E, M, W.Wp.data_ptr(),
                   W.Wps.data_ptr(), N, K_aug, Y.data_ptr(), ws, ws_bytes, variant, _stream_of_call(stream))
    _check(st, "prq_grouped_gemm")
    return Y


# --------------------------------------------------------- attention block ---
_BF16, _I64, _BOOL = torch.bfloat16, torch.int64, torch.bool
_ROPE_IN = (_F32, _BF16)
_I32_MAX = (1 << 31) - 1


class PagedKV:
    """A paged key/value cache: K and V [pages, kv heads, page size, D] bf16, each page
    contiguous (views into a larger pool may leave room between pages)."""

    __slots__ = ("K", "V", "pages", "heads", "page_size", "D", "stride")

    def __init__(self, K, V):
        self.K, self.V = K, V
        if not (isinstance(K, torch.Tensor) and isinstance(V, torch.Tensor) and K.dtype is V.dtype is _BF16
                and K.dim() == 4 and K.is_cuda and V.is_cuda and K.shape == V.shape):
            raise ValueError("K and V must be bfloat16 GPU tensors [pages, kv heads, page size, D] of one shape")
        self.pages, self.heads, self.page_size, self.D = K.shape
        page = self.heads * self.page_size * self.D
        self.stride = page
        if not (K.is_contiguous() and V.is_contiguous()):
            strides = K.stride()
            if strides[1:] != (self.page_size * self.D, self.D, 1) or V.stride() != strides:
                raise ValueError(f"each page of K and V must be contiguous, at one stride (strides {strides}, "
                                 f"{V.stride()})")
            self.stride = max(strides[0], page) if self.pages == 1 else strides[0]


def prq_paged_kv(pages, heads, page_size, D, device="cuda"):
    """A cache of `pages` empty pages (zeros)."""
    return PagedKV(*(_alloc(torch.zeros, (pages, heads, page_size, D), _BF16, device, None) for _ in range(2)))


def prq_rope_table(positions, rotary_dim, theta=10000.0, scaling="none", factor=1.0, original_positions=None,
                   beta_fast=32.0, beta_slow=1.0, device="cuda"):
    """Cosine and sine of every position and rotated pair, float32 [positions, rotary_dim / 2, 2],
    from angles in float64: position * f_i, f_i = theta^(-2i / rotary_dim), i < rotary_dim / 2.

    scaling, for contexts `factor` >= 1 times the one that a model was trained on:
      "linear": f_i / factor;
      "ntk":    theta * factor^(rotary_dim / (rotary_dim - 2)) in theta's place (the slowest pair
                then turns as with "linear", the fastest as without);
      "yarn":   f_i (g_i / factor + 1 - g_i), g_i a ramp over i from 0 to 1 between the pairs that
                turn beta_fast and beta_slow times in original_positions (their indices rounded
                outwards), and cosine and sine times 0.1 ln(factor) + 1."""
    r = int(rotary_dim)
    if r <= 0 or r % 8 or positions < 0:
        raise ValueError(f"rotary_dim {rotary_dim} must be a positive multiple of 8, positions {positions} >= 0")
    if scaling not in ("none", "linear", "ntk", "yarn"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if not theta > 1 or not factor >= 1:
        raise ValueError(f"theta {theta} must be above 1 and factor {factor} at least 1")
    i = np.arange(r // 2, dtype=np.float64)
    base = theta * factor ** (r / (r - 2)) if scaling == "ntk" else theta
    f = base ** (-2.0 * i / r)
    gain = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "yarn":
        if not original_positions or original_positions < 1 or not beta_fast > beta_slow > 0:
            raise ValueError("yarn needs original_positions and beta_fast > beta_slow > 0")
        # index whose pair turns `turns` times over the original context
        index = [r * np.log(original_positions / (turns * 2 * np.pi)) / (2 * np.log(theta))
                 for turns in (beta_fast, beta_slow)]
        lo, hi = max(np.floor(index[0]), 0.0), min(np.ceil(index[1]), r - 1.0)
        ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        f = f * (ramp / factor + (1.0 - ramp))
        gain = 0.1 * np.log(factor) + 1.0
    angle = np.arange(int(positions), dtype=np.float64)[:, None] * f
    table = np.stack([np.cos(angle), np.sin(angle)], axis=-1) * gain
    return torch.from_numpy(table.astype(np.float32)).to(device)


def _rows(t, name, dtypes, M, wide):
    """A GPU tensor [M, wide] whose rows are contiguous -> its row stride."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.is_cuda and t.shape == (M, wide):
        if t.is_contiguous():
            return wide
        if t.stride(1) == 1 or wide == 1:
            return t.stride(0) if M > 1 else wide
    raise ValueError(f"{name} must be a GPU tensor of {' or '.join(map(str, dtypes))}, {M} rows of {wide} "
                     f"contiguous elements"
                     + (f" (is {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device})"
                        if isinstance(t, torch.Tensor) else ""))


def _vector(t, name, dtype, n):
    if not _is(t, dtype, (n,)):
        _need(t, name, dtype, (n,))
        _on_gpu(**{name: t})


def _head_weight(w, name, D):
    """(address, type) of a norm's weight [D]."""
    if _is(w, _BF16, (D,)):
        return w.data_ptr(), PRQ_BF16
    if not _is(w, _F32, (D,)):
        _need(w, name, (_F32, _BF16), (D,))
        _on_gpu(**{name: w})
    return w.data_ptr(), PRQ_BF16 if w.dtype is _BF16 else PRQ_F32


def _output(t, name, shape, dtype, like, stream):
    """An output of a call: `t`, checked, or a new one beside the tensor `like`."""
    if t is None:
        return like.new_empty(shape, dtype=dtype) if stream is None else _alloc(torch.empty, shape, dtype, like.device,
                                                                                stream)
    if not _is(t, dtype, shape):
        _need(t, name, dtype, shape)
        _on_gpu(**{name: t})
    return t


def prq_qk_norm_rope(q, k, v, positions, table, cache, slots, q_weight=None, k_weight=None, eps=1e-6,
                     interleaved=False, out=None, stream=None):
    """Queries, keys and values [M, heads * D] (float32 or bf16) -> queries [M, Hq, D] bf16, normed
    per head (where a weight is given) and rotated by `positions` int32 [M]; keys, the same, and
    values go to `slots` int64 [M] of the cache (-1: nowhere).  table: prq_rope_table's, or None
    for no rotation."""
    D, Hk = cache.D, cache.heads
    if not isinstance(q, torch.Tensor) or q.dim() != 2:
        raise ValueError(f"q must be [M, heads * {D}]")
    M, wide = q.shape
    if wide % D or not wide:
        raise ValueError(f"q must be [M, heads * {D}]")
    Hq, kind, wide_k = wide // D, (q.dtype,), Hk * D
    ld_q = _rows(q, "q", _ROPE_IN, M, wide)
    ld_k, ld_v = _rows(k, "k", kind, M, wide_k), _rows(v, "v", kind, M, wide_k)
    rot = rows = 0
    table_at = positions_at = None
    if table is not None:
        if not (isinstance(table, torch.Tensor) and table.dtype is _F32 and table.is_cuda and table.is_contiguous()
                and table.dim() == 3 and table.shape[2] == 2):
            raise ValueError("table must be a contiguous float32 GPU tensor [positions, rotary_dim / 2, 2]")
        rows, half, _ = table.shape
        rot = 2 * half
        if rot:
            _vector(positions, "positions", _I32, M)
            table_at, positions_at = table.data_ptr(), positions.data_ptr()
    _vector(slots, "slots", _I64, M)
    wq = wk = None
    w_kind = 0
    if k_weight is not None:
        wk, w_kind = _head_weight(k_weight, "k_weight", D)
    if q_weight is not None:
        wq, kind = _head_weight(q_weight, "q_weight", D)
        if wk is not None and kind != w_kind:
            raise ValueError("q_weight and k_weight must have one type")
        w_kind = kind
    out = _output(out, "out", (M, Hq, D), _BF16, q, stream)
    st = _qk_norm_rope(q.data_ptr(), ld_q, k.data_ptr(), ld_k, v.data_ptr(), ld_v, int(q.dtype is _BF16), M, Hq, Hk, D,
                       wq, wk, w_kind, eps, positions_at, table_at, rows, rot,
                       int(interleaved), out.data_ptr(), cache.K.data_ptr(), cache.V.data_ptr(), cache.stride,
                       cache.pages, cache.page_size, slots.data_ptr(), _stream_of_call(stream))
    _check(st, "prq_qk_norm_rope")
    return out


def prq_tree_attention_workspace_bytes(M, B, Hq, Hk, D, max_kv_len):
    return int(_tree_ws(M, B, Hq, Hk, D, min(max_kv_len, _I32_MAX)))


def prq_tree_attention(q, cache, page_table, cached_lens, q_offsets, scale, tree_mask=None, max_kv_len=None,
                       out=None, lse=None, workspace=None, stream=None):
    """q [M, Hq, D] bf16 (rows of B requests, q_offsets int32 [B + 1]) over the cache -> (out [M, Hq, D]
    bf16, lse [M, Hq] float32).  Request b's own tokens follow its cached_lens[b] (int32 [B]) cached
    ones on its pages (page_table int32 [B, pages]); tree_mask bool [M, w] says which of its own tokens
    a row sees (None: itself and those before it).  max_kv_len: the most tokens a request has (default:
    what the page table holds).  workspace: uint8, prq_tree_attention_workspace_bytes, zeroed before its
    first use and left ready by every call (else allocated, zeroed by another launch)."""
    if not (isinstance(q, torch.Tensor) and q.dtype is _BF16 and q.is_cuda and q.dim() == 3 and q.shape[2] == cache.D
            and (q.is_contiguous() or (q.stride(2) == 1 and (q.shape[1] <= 1 or q.stride(1) == cache.D)))):
        raise ValueError(f"q must be a bfloat16 GPU tensor [M, heads, {cache.D}] with contiguous rows")
    M, Hq, D = q.shape
    ld_q = q.stride(0) if M > 1 else Hq * D
    if not (isinstance(page_table, torch.Tensor) and page_table.dim() == 2):
        raise ValueError("page_table must be a GPU tensor [requests, pages]")
    B, wide = page_table.shape
    ld_pages = _rows(page_table, "page_table", (_I32,), B, wide)
    _vector(cached_lens, "cached_lens", _I32, B)
    _vector(q_offsets, "q_offsets", _I32, B + 1)
    mask, ld_mask, mask_wide = None, 0, 0
    if tree_mask is not None:
        mask_wide = tree_mask.shape[1] if tree_mask.dim() == 2 else -1
        ld_mask = _rows(tree_mask, "tree_mask", (_BOOL, _U8), M, mask_wide)
        # without a column nothing is seen, which a null pointer would not say
        mask = tree_mask.data_ptr() if mask_wide else q_offsets.data_ptr()
    if max_kv_len is None:
        max_kv_len = wide * cache.page_size
    max_kv_len = min(max_kv_len, _I32_MAX)        # (ctypes would take its low 32 bits)
    out = _output(out, "out", (M, Hq, D), _BF16, q, stream)
    lse = _output(lse, "lse", (M, Hq), _F32, q, stream)
    if workspace is None:
        need = int(_tree_ws(M, B, Hq, cache.heads, D, max_kv_len))
        if need:
            workspace = _alloc(torch.zeros, need, _U8, q.device, stream, kept=False)
    ws, ws_bytes = _workspace_arg(workspace)
    st = _tree(q.data_ptr(), ld_q, M, Hq, cache.heads, D, cache.K.data_ptr(), cache.V.data_ptr(), cache.stride,
               cache.pages, cache.page_size, page_table.data_ptr(), ld_pages, wide, cached_lens.data_ptr(),
               q_offsets.data_ptr(), B, max_kv_len, scale, mask, ld_mask, mask_wide, out.data_ptr(), lse.data_ptr(),
               ws, ws_bytes, _stream_of_call(stream))
    _check(st, "prq_tree_attention")
    return out, lse


class LoraAdapters:
    """Device buffers of a set of adapters: A [sum of ranks, K] bf16, B bf16 flat (adapter a's [N, rank]
    from element N * rank_offsets[a]), rank_offsets int32 [adapters + 1] in multiples of 8, scales float32
    [adapters], the largest rank, and where ranks are padded to those multiples the ranks themselves,
    int32 [adapters] (None: what lies between the offsets)."""

    __slots__ = ("A", "B", "rank_offsets", "scales", "max_rank", "ranks", "rank_rows", "count")

    def __init__(self, A, B, rank_offsets, scales, max_rank, ranks=None):
        self.A, self.B, self.rank_offsets, self.scales, self.max_rank = A, B, rank_offsets, scales, max_rank
        self.ranks = ranks
        self.rank_rows, self.count = A.shape[0], scales.shape[0]


def prq_lora_adapters(pairs, scales, device="cuda"):
    """LoraAdapters of [(A [r, K], B [N, r]), ...] and one scale each; ranks padded with zeros to multiples
    of 8, values rounded to bf16."""
    if not pairs or len(pairs) != len(scales):
        raise ValueError("as many scales as adapters are needed, and one adapter at least")
    K, N = pairs[0][0].shape[1], pairs[0][1].shape[0]
    own, ranks, As, Bs = [], [], [], []
    for A, B in pairs:
        r = A.shape[0]
        if A.shape != (r, K) or B.shape != (N, r):
            raise ValueError(f"adapter shapes {tuple(A.shape)}, {tuple(B.shape)} do not fit [r, {K}], [{N}, r]")
        pad = -r % 8
        A, B = A.to(device, _BF16), B.to(device, _BF16)
        As.append(torch.nn.functional.pad(A, (0, 0, 0, pad)))
        Bs.append(torch.nn.functional.pad(B, (0, pad)).reshape(-1))
        own.append(r)
        ranks.append(r + pad)
    return LoraAdapters(torch.cat(As).contiguous(), torch.cat(Bs).contiguous(),
                        torch.tensor(np.concatenate([[0], np.cumsum(ranks)]), dtype=_I32, device=device),
                        torch.tensor([float(s) for s in scales], dtype=_F32, device=device), max(ranks),
                        torch.tensor(own, dtype=_I32, device=device) if own != ranks else None)


def prq_lora_workspace_bytes(M, segments, N, K, max_rank):
    return int(_lora_ws(M, segments, N, K, max_rank))


def prq_lora(x, adapters, segment_offsets, segment_adapter, Y, out=None, workspace=None, stream=None):
    """out [M, N] float32 = Y + scale * B_a (A_a x) with each segment's adapter (segment_offsets int32
    [S + 1] over x's rows [M, K] bf16, segment_adapter int32 [S], -1: none).  out=None adds into Y.
    workspace: uint8, prq_lora_workspace_bytes (else allocated)."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or not isinstance(Y, torch.Tensor) or Y.dim() != 2:
        raise ValueError("x and Y must be 2-D tensors")
    (M, K), N = x.shape, Y.shape[1]
    ld_x, ld_y = _rows(x, "x", (_BF16,), M, K), _rows(Y, "Y", (_F32,), M, N)
    if out is None:
        out = Y
    ld_out = _rows(out, "out", (_F32,), M, N)
    a = adapters
    n, R = a.count, a.rank_rows
    if a.ranks is not None:
        _vector(a.ranks, "adapters.ranks", _I32, n)
    if not (_is(a.A, _BF16, (R, K)) and _holds(a.B, _BF16, N * R) and _is(a.rank_offsets, _I32, (n + 1,))
            and _is(a.scales, _F32, (n,))):
        _need(a.A, "adapters.A", _BF16, (R, K))
        _need(a.B, "adapters.B", _BF16, min_numel=N * R)
        _need(a.rank_offsets, "adapters.rank_offsets", _I32, (n + 1,))
        _need(a.scales, "adapters.scales", _F32, (n,))
        _on_gpu(A=a.A, B=a.B, rank_offsets=a.rank_offsets, scales=a.scales)
    if not (isinstance(segment_adapter, torch.Tensor) and segment_adapter.dim() == 1):
        raise ValueError("segment_adapter must be an int32 GPU tensor [segments]")
    segments = segment_adapter.shape[0]
    _vector(segment_adapter, "segment_adapter", _I32, segments)
    _vector(segment_offsets, "segment_offsets", _I32, segments + 1)
    if workspace is None:
        ws, ws_bytes = None, _lora_ws(M, segments, N, K, a.max_rank)
        if ws_bytes:
            workspace = (x.new_empty(ws_bytes, dtype=_U8) if stream is None
                         else _alloc(torch.empty, ws_bytes, _U8, x.device, stream, kept=False))
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _workspace_arg(workspace)
    st = _lora_ex(x.data_ptr(), ld_x, M, K, a.A.data_ptr(), a.B.data_ptr(), a.rank_offsets.data_ptr(),
                  None if a.ranks is None else a.ranks.data_ptr(), a.scales.data_ptr(), n, R, a.max_rank,
                  segment_offsets.data_ptr(), segment_adapter.data_ptr(), segments, N, Y.data_ptr(), ld_y,
                  out.data_ptr(), ld_out, ws, ws_bytes, _stream_of_call(stream))
    _check(st, "prq_lora")
    return out


# ---------------------------------------------------- mixture-of-experts half ---
def _device_of(t, name):
    """The device of a call's leading tensor, which must be the current one: the launch goes there."""
    d = t.get_device()
    if d < 0:
        raise ValueError(f"{name} must be a GPU tensor")
    if d != (torch.cuda.current_device() if _cur_device is None else _cur_device()):
        raise ValueError(f"{name} is on {t.device}, which is not the current device")
    return d


# The checks of these calls: one expression a tensor, on one device d; whatever does not pass goes
# through the functions behind, which say why.
def _here(t, dtype, shape, d):
    return (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == d
            and t.is_contiguous())


def _on_device(t, name, d):
    if t.get_device() != d:
        raise ValueError(f"{name} is on {t.device}, which is not the current device")


def _matrix(t, name, dtypes, M, wide, d):
    """_rows on the current device."""
    ld = _rows(t, name, dtypes, M, wide)
    _on_device(t, name, d)
    return ld


def _exact(t, name, dtype, shape, d):
    """A contiguous tensor of a shape on the current device."""
    if not _here(t, dtype, shape, d):
        _need(t, name, dtype, shape)
        _on_gpu(**{name: t})
        _on_device(t, name, d)


def _norm_weight(w, name, H, d):
    """(address, type) of a norm's weight [H] on the current device."""
    if not _here(w, _BF16, (H,), d):
        _exact(w, name, (_F32, _BF16), (H,), d)
    return w.data_ptr(), PRQ_BF16 if w.dtype is _BF16 else PRQ_F32


def prq_block_norm(y, residual, pre_weight=None, post_weight=None, gate=None, gate_index=None, eps=1e-6,
                   weight_offset=0.0, residual_scale=1.0, block_scale=1.0, out=None, residual_out=None, stream=None):
    """A block's output y and the residual, [M, H] float32 or bf16 -> (h, r') with
    u = y, or y / rms(y) * (weight_offset + post_weight); r' = residual_scale * residual +
    block_scale * gate * u; h [M, H] bf16 = r' / rms(r') * (weight_offset + pre_weight).

    y None: no block.  residual None: none, and r' (then y's type) is stored only with residual_out.
    Else residual_out=None writes r' over residual.  gate: [rows, H] float32 or bf16, one row for
    all, one for each, or gate_index int32 [M] names each row's (outside: none).  pre_weight None:
    h is None."""
    lead = residual if y is None else y
    if not isinstance(lead, torch.Tensor) or lead.dim() != 2:
        raise ValueError("y or residual must be [M, H]")
    if y is None and (post_weight is not None or gate is not None):
        raise ValueError("post_weight and gate need y")
    M, H = shape = lead.shape
    d = _device_of(lead, "residual" if y is None else "y")
    y_at = r_at = ro_at = h_at = post = pre = gate_at = index_at = 0          # (no pointer)
    ld_y = ld_r = ld_ro = ld_h = ld_gate = w_kind = gate_rows = gate_kind = 0
    y_kind = r_kind = lead.dtype
    if y is not None:
        ld_y = H if _here(y, _F32, shape, d) else _matrix(y, "y", _ROPE_IN, M, H, d)
        y_at = y.data_ptr()
    if residual is not None:
        ld_r = H if _here(residual, _BF16, shape, d) else _matrix(residual, "residual", _ROPE_IN, M, H, d)
        r_at, r_kind = residual.data_ptr(), residual.dtype
        if residual_out is None and (y is not None or residual_scale != 1.0):
            residual_out = residual
    stores = residual_out is not None
    if residual_out is residual:
        ro_at, ld_ro = r_at, ld_r
        if y is None and residual_scale == 1.0:      # (nothing to change)
            ro_at, stores = 0, False
    elif residual_out is not None:
        ld_ro = H if _here(residual_out, r_kind, shape, d) else _matrix(residual_out, "residual_out", (r_kind,), M, H, d)
        ro_at = residual_out.data_ptr()
    if pre_weight is not None:
        pre, w_kind = _norm_weight(pre_weight, "pre_weight", H, d)
    if post_weight is not None:
        post, kind = _norm_weight(post_weight, "post_weight", H, d)
        if pre_weight is not None and kind != w_kind:
            raise ValueError("post_weight and pre_weight must have one type")
        w_kind = kind
    if gate is not None:
        if not isinstance(gate, torch.Tensor) or gate.dim() != 2:
            raise ValueError(f"gate must be [rows, {H}]")
        gate_rows = gate.shape[0]
        ld_gate, gate_kind = _matrix(gate, "gate", _ROPE_IN, gate_rows, H, d), int(gate.dtype is _BF16)
        gate_at = gate.data_ptr()
        if gate_index is not None:
            _exact(gate_index, "gate_index", _I32, (M,), d)
            index_at = gate_index.data_ptr()
    elif gate_index is not None:
        raise ValueError("gate_index needs a gate")
    if pre_weight is not None:
        if out is None:
            out = _output(None, "out", (M, H), _BF16, lead, stream)
        ld_h = H if _here(out, _BF16, shape, d) else _matrix(out, "out", (_BF16,), M, H, d)
        h_at = out.data_ptr()
    elif out is not None:
        raise ValueError("out needs pre_weight")
    if stores or pre_weight is not None:
        st = _block_norm_call(_block_norm_pack(
            y_at, ld_y, 1 if y_kind is _BF16 else 0, r_at, ld_r, 1 if r_kind is _BF16 else 0, M, H, post, pre, w_kind,
            weight_offset, gate_at, ld_gate, gate_kind, gate_rows, index_at, eps, residual_scale, block_scale, ro_at, ld_ro,
            h_at, ld_h, _stream_at(stream)))
        if st:
            _check(st, "prq_block_norm")
    return out, residual if residual_out is None else residual_out


def prq_moe_route_workspace_bytes(M, E, H):
    return int(_route_ws(M, E, H))


def _state_workspace(workspace, need, like, stream, d):
    """A workspace with a state head (need() bytes, zeroed, where none is given), or None."""
    if workspace is None:
        n = need()
        return _alloc(torch.zeros, n, _U8, like.device, stream, kept=False) if n else None
    if not _holds(workspace, _U8, 0):
        _need(workspace, "workspace", _U8)
        _on_gpu(workspace=workspace)
    _on_device(workspace, "workspace", d)
    return workspace


def _extent(workspace):
    return (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())


def prq_moe_route(x, W, k, scoring="softmax", bias=None, renormalize=True, scale=1.0, ids=None, weights=None,
                  logits=None, workspace=None, stream=None):
    """x [M, H] bf16, router weight W [E, H] bf16 -> (ids int32 [M, k], weights float32 [M, k]): the k
    experts with the largest softmax or sigmoid of x W^T (+ bias float32 [E], with the sigmoid),
    descending, the lower index first among equals, and their scores (renormalize: divided by their
    sum; a softmax of the k alone, so a NaN that is not chosen does not count) times scale.  logits: float32 [M, E] to write x W^T into.  workspace: uint8,
    prq_moe_route_workspace_bytes, zeroed before its first use and left ready by every call (else
    allocated, zeroed by another launch)."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or not isinstance(W, torch.Tensor) or W.dim() != 2:
        raise ValueError("x must be [M, H] and W [E, H]")
    (M, H), E = x.shape, W.shape[0]
    if scoring not in ROUTE_SCORINGS:
        raise ValueError(f"unknown scoring {scoring!r}")
    if not 1 <= k <= E:
        raise ValueError(f"k {k} must lie between 1 and the {E} experts")
    d = _device_of(x, "x")
    ld_x = H if _here(x, _BF16, (M, H), d) else _matrix(x, "x", (_BF16,), M, H, d)
    ld_w = H if _here(W, _BF16, (E, H), d) else _matrix(W, "W", (_BF16,), E, H, d)
    if bias is not None:
        _exact(bias, "bias", _F32, (E,), d)
    if ids is None:
        ids = _output(None, "ids", (M, k), _I32, x, stream)
    if weights is None:
        weights = _output(None, "weights", (M, k), _F32, x, stream)
    _exact(ids, "ids", _I32, (M, k), d)
    _exact(weights, "weights", _F32, (M, k), d)
    ld_l = _matrix(logits, "logits", (_F32,), M, E, d) if logits is not None else 0
    workspace = _state_workspace(workspace, lambda: _route_ws(M, E, H), x, stream, d)
    st = _route_call(_route_pack(
        x.data_ptr(), ld_x, M, H, W.data_ptr(), ld_w, E, k, ROUTE_SCORINGS[scoring], 0 if bias is None else bias.data_ptr(),
        1 if renormalize else 0, scale, ids.data_ptr(), weights.data_ptr(), 0 if logits is None else logits.data_ptr(), ld_l,
        *_extent(workspace), _stream_at(stream)))
    if st:
        _check(st, "prq_moe_route")
    return ids, weights


def prq_moe_layer_workspace_bytes(M, k, E, H, I, k_tail, N):
    return int(_moe_ws(M, k, E, H, I, k_tail, N))


def _weight_here(W, name, d):
    """(codes, scales) addresses of a PackedWeight on the current device."""
    Wp, Wps = W.Wp, W.Wps
    steps = (W.K_aug + 127) // 128
    blocks = W.E * (W.N // 16)
    if not (W.N % 16 == 0 and W.K_aug % 32 == 0 and _here(Wp, _U8, (blocks * steps * 1024,), d)
            and _here(Wps, _U8, (blocks * ((steps + 3) // 4) * 256,), d)):
        W.check_sizes()
        _on_gpu(**{name + ".Wp": Wp, name + ".Wps": Wps})
        _on_device(Wp, name + ".Wp", d)
        _on_device(Wps, name + ".Wps", d)
    return Wp.data_ptr(), Wps.data_ptr()


def prq_moe_layer(x, ids, weights, gate_up, down, k_tail=0, out=None, workspace=None, stream=None):
    """All experts of up to 64 tokens: x [M, H] bf16, ids int32 and weights float32 [M, k] (prq_moe_route's;
    an id outside [0, E) adds nothing) -> out [M, N] bf16 = sum_j weights[:, j] * down_e [h; last k_tail of
    h], h = SiLU(gate_e x) * (up_e x).  gate_up: PackedWeight of E weights [2 I, H], gate rows first;
    down: of E weights [N, I + k_tail].  workspace: as prq_moe_route's, prq_moe_layer_workspace_bytes."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("x must be [M, H] and ids [M, k]")
    (M, H), k = x.shape, ids.shape[1]
    E, N, I = gate_up.E, down.N, down.K_aug - k_tail
    if gate_up.K_aug != H or gate_up.N != 2 * I or down.E != E:
        raise ValueError(f"gate_up ({gate_up.E} x [{gate_up.N}, {gate_up.K_aug}]) and down ({down.E} x [{down.N}, "
                         f"{down.K_aug}]) do not fit [2 I, {H}] and [N, I + {k_tail}]")
    d = _device_of(x, "x")
    ld_x = H if _here(x, _BF16, (M, H), d) else _matrix(x, "x", (_BF16,), M, H, d)
    _exact(ids, "ids", _I32, (M, k), d)
    _exact(weights, "weights", _F32, (M, k), d)
    up_at, up_scales_at = _weight_here(gate_up, "gate_up", d)
    down_at, down_scales_at = _weight_here(down, "down", d)
    if out is None:
        out = _output(None, "out", (M, N), _BF16, x, stream)
    ld_out = N if _here(out, _BF16, (M, N), d) else _matrix(out, "out", (_BF16,), M, N, d)
    workspace = _state_workspace(workspace, lambda: _moe_ws(M, k, E, H, I, k_tail, N), x, stream, d)
    st = _moe_call(_moe_pack(
        x.data_ptr(), ld_x, M, ids.data_ptr(), weights.data_ptr(), k, up_at, up_scales_at, down_at, down_scales_at, E, H, I,
        k_tail, N, out.data_ptr(), ld_out, *_extent(workspace), _stream_at(stream)))
    if st:
        _check(st, "prq_moe_layer")
    return out
