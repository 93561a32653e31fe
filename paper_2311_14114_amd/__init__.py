"""Python binding of libsoniq (gfx950): SONIQ's per-channel mixed-precision
quantized matrix multiply (arXiv 2311.14114, Sec. 3 codec and Alg. 1 Phase II
integer MAC).

The functions carry the C-ABI names of ``include/soniq.h`` and only marshal
arguments: torch tensors provide device pointers and the current HIP stream;
every step runs in the library's HIP kernels.  There is no CPU fallback: if
``libsoniq.so`` is missing, importing the binding's entry points raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsoniq.so")

SONIQ_OK = 0
SONIQ_ERR_INVALID_ARGUMENT = 1
SONIQ_ERR_UNSUPPORTED = 2
SONIQ_ERR_OUT_OF_MEMORY = 3
SONIQ_ERR_HIP = 4
SONIQ_WQ_SYMMETRIC = 0
SONIQ_WQ_TWOS_FRACTION = 1
SONIQ_WPACK_SIGN_NIBBLES = 0x100
SONIQ_WPACK_F8F6F4 = 0x200
SONIQ_WPACK_DENSE = 0x400
SONIQ_MAX_K = 65536
SONIQ_F32 = 0
SONIQ_BF16 = 1
SONIQ_F16 = 2

# Every symbol include/soniq.h declares.
EXPORTED = [
    "soniq_pack_weights", "soniq_pack_weights_ex", "soniq_pack_weights_grouped",
    "soniq_pack_weights_conv3x3", "soniq_act_create", "soniq_act_create_conv3x3",
    "soniq_quantize_act", "soniq_quantize_act_conv3x3", "soniq_mp_gemm", "soniq_quantize_mp_gemm",
    "soniq_quantize_mp_gemm_scratch",
    "soniq_mp_gemm_quantize_next", "soniq_mp_gemm_quantize_next_max",
    "soniq_weights_info",
    "soniq_plan_input_channels", "soniq_weights_unpack_debug",
    "soniq_act_unpack_debug", "soniq_act_wait_timeouts", "soniq_debug_stream_read",
    "soniq_weights_destroy",
    "soniq_act_destroy",
    "soniq_last_error",
    "soniq_quantize_rows", "soniq_i8_gemm", "soniq_quantize_i8_gemm",
    "soniq_quantize_i8_gemm_workspace",
    "soniq_kv_write", "soniq_kv_read", "soniq_kv_attention", "soniq_kv_attention_workspace",
]


class SoniqError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"soniq status {status}: {msg}")
        self.status = status


class WeightsInfo(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int64), ("K", ctypes.c_int64), ("S", ctypes.c_int32),
        ("a_signed", ctypes.c_int32), ("wq_mode", ctypes.c_int32),
        ("a_bits", ctypes.c_uint8 * 2), ("w_bits", ctypes.c_uint8 * 2),
        ("a_count", ctypes.c_int64 * 2), ("a_count_padded", ctypes.c_int64 * 2),
        ("w_count", ctypes.c_int64 * 2), ("packed_w_bytes", ctypes.c_int64),
        ("packed_w_bytes_algorithmic", ctypes.c_int64),
        ("act_group_bits", ctypes.c_int32), ("act_scales", ctypes.c_int32),
        ("f8f6f4", ctypes.c_int32), ("dense_w_bytes", ctypes.c_int64),
    ]


class KVCacheStruct(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
        ("v", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("bits", ctypes.c_int32),
    ]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libsoniq.so (fails loudly when it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                              "or python -m paper_2311_14114_amd.build")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, i32, st = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_int
        L.soniq_pack_weights.restype = st
        L.soniq_pack_weights.argtypes = [vp, i64, i64, i64, vp, vp, i32, vp, ctypes.POINTER(vp)]
        L.soniq_pack_weights_ex.restype = st
        L.soniq_pack_weights_ex.argtypes = [vp, i64, i64, i64, vp, vp, i32, i32, vp, ctypes.POINTER(vp)]
        L.soniq_pack_weights_grouped.restype = st
        L.soniq_pack_weights_grouped.argtypes = [vp, i64, i64, i64, vp, vp, i32, i32, i32, vp,
                                                 ctypes.POINTER(vp)]
        L.soniq_pack_weights_conv3x3.restype = st
        L.soniq_pack_weights_conv3x3.argtypes = [vp, i64, i64, vp, vp, i32, i32, vp,
                                                 ctypes.POINTER(vp)]
        L.soniq_act_create_conv3x3.restype = st
        L.soniq_act_create_conv3x3.argtypes = [vp, i64, i64, i64, ctypes.POINTER(vp)]
        L.soniq_act_create.restype = st
        L.soniq_act_create.argtypes = [vp, i64, ctypes.POINTER(vp)]
        L.soniq_quantize_act.restype = st
        L.soniq_quantize_act.argtypes = [vp, vp, i64, i64, vp]
        L.soniq_quantize_act_conv3x3.restype = st
        L.soniq_quantize_act_conv3x3.argtypes = [vp, vp, i64, i64, i64, i64, vp]
        L.soniq_mp_gemm.restype = st
        L.soniq_mp_gemm.argtypes = [vp, vp, vp, i64, vp, vp]
        L.soniq_mp_gemm_quantize_next.restype = st
        L.soniq_mp_gemm_quantize_next.argtypes = [vp, vp, vp, vp, vp, i64, vp, vp]
        L.soniq_mp_gemm_quantize_next_max.restype = st
        L.soniq_mp_gemm_quantize_next_max.argtypes = [vp, vp, vp, vp, i64, vp, vp]
        L.soniq_quantize_mp_gemm.restype = st
        L.soniq_quantize_mp_gemm.argtypes = [vp, vp, vp, i64, i64, vp, i64, vp, vp]
        L.soniq_quantize_mp_gemm_scratch.restype = st
        L.soniq_quantize_mp_gemm_scratch.argtypes = [vp, vp, i64, i64, vp, i64, vp, vp]
        L.soniq_weights_info.restype = st
        L.soniq_weights_info.argtypes = [vp, ctypes.POINTER(WeightsInfo)]
        L.soniq_plan_input_channels.restype = st
        L.soniq_plan_input_channels.argtypes = [vp, i64, vp, vp, vp, vp]
        L.soniq_weights_unpack_debug.restype = st
        L.soniq_weights_unpack_debug.argtypes = [vp, vp, vp]
        L.soniq_act_unpack_debug.restype = st
        L.soniq_act_unpack_debug.argtypes = [vp, vp, vp]
        L.soniq_act_wait_timeouts.restype = st
        L.soniq_act_wait_timeouts.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64)]
        L.soniq_debug_stream_read.restype = st
        L.soniq_debug_stream_read.argtypes = [vp, i64, vp, vp]
        f32 = ctypes.c_float
        L.soniq_quantize_rows.restype = st
        L.soniq_quantize_rows.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, vp]
        L.soniq_i8_gemm.restype = st
        L.soniq_i8_gemm.argtypes = [vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp]
        L.soniq_quantize_i8_gemm.restype = st
        L.soniq_quantize_i8_gemm.argtypes = [vp, i32, i64, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64,
                                             vp, i64, vp]
        L.soniq_quantize_i8_gemm_workspace.restype = st
        L.soniq_quantize_i8_gemm_workspace.argtypes = [i64, i64, ctypes.POINTER(i64)]
        rows = [vp, vp, i64, i64, vp, i64, i64, i32, i64, vp, i64, i64, i64, vp, vp, vp]
        L.soniq_kv_write.restype = st
        L.soniq_kv_write.argtypes = rows
        L.soniq_kv_read.restype = st
        L.soniq_kv_read.argtypes = rows
        L.soniq_kv_attention.restype = st
        L.soniq_kv_attention.argtypes = [vp, vp, i64, i64, i32, i64, i32, vp, i64, i64, i64, vp, vp, vp,
                                         i32, f32, i64, i64, vp, i64, i64, vp, vp, i64, vp]
        L.soniq_kv_attention_workspace.restype = st
        L.soniq_kv_attention_workspace.argtypes = [vp, i64, i32, i64, i64, i64, ctypes.POINTER(i64)]
        L.soniq_weights_destroy.restype = None
        L.soniq_weights_destroy.argtypes = [vp]
        L.soniq_act_destroy.restype = None
        L.soniq_act_destroy.argtypes = [vp]
        L.soniq_last_error.restype = ctypes.c_char_p
        L.soniq_last_error.argtypes = []
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != SONIQ_OK:
        raise SoniqError(status, lib().soniq_last_error().decode())


def _u8(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=np.uint8)


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(int(stream))
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(t, dtype_name: str):
    import torch
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError(f"expected a device tensor ({dtype_name})")
    return ctypes.c_void_p(t.data_ptr())


class Weights:
    """Owner of a packed weights handle (soniq_weights)."""

    def __init__(self, handle: ctypes.c_void_p, N: int, K: int):
        self.handle = handle
        self.N, self.K = N, K
        self.info = soniq_weights_info(self)
        # accumulators per output: precision groups, or sub-group blocks
        self.S = self.info.act_scales

    def close(self):
        if self.handle:
            lib().soniq_weights_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Activations:
    """Owner of a packed activation handle (soniq_act)."""

    def __init__(self, handle: ctypes.c_void_p, weights: Weights, max_M: int):
        self.handle = handle
        self.weights = weights      # keeps the weights alive
        self.max_M = max_M
        self.M = 0

    def close(self):
        if self.handle:
            lib().soniq_act_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def soniq_pack_weights(W, w_bits, a_bits, a_signed: bool, wq_mode: int = SONIQ_WQ_SYMMETRIC,
                       stream=None, act_group_bits: int = 0, sign_nibbles: bool = False,
                       f8f6f4: bool = False, dense: bool = False) -> Weights:
    """Quantize, re-order and bit-pack W (device float32 [N, K], row-major).
    act_group_bits > 0 gives the activations sub-group scales (blocks of
    that many bits of storage inside each precision group); sign_nibbles
    stores 1-bit channels in 4-bit containers (SONIQ_WPACK_SIGN_NIBBLES);
    f8f6f4 also keeps the narrow operands in fp4/fp6 MFMA operand formats
    (SONIQ_WPACK_F8F6F4); dense also keeps every code in exactly its width
    for the GEMV forms (SONIQ_WPACK_DENSE)."""
    import torch
    if W.dtype != torch.float32 or W.dim() != 2 or W.stride(1) != 1:
        raise TypeError("W must be a 2-D float32 device tensor with unit column stride")
    N, K = W.shape
    wb, ab = _u8(w_bits), _u8(a_bits)
    if wb.shape != (N,) or ab.shape != (K,):
        raise ValueError("w_bits must have N entries and a_bits K entries")
    h = ctypes.c_void_p()
    _check(lib().soniq_pack_weights_grouped(_dev(W, "float32"), N, K, W.stride(0),
                                            wb.ctypes.data_as(ctypes.c_void_p),
                                            ab.ctypes.data_as(ctypes.c_void_p),
                                            1 if a_signed else 0,
                                            int(wq_mode) | (SONIQ_WPACK_SIGN_NIBBLES if sign_nibbles else 0)
                                            | (SONIQ_WPACK_F8F6F4 if f8f6f4 else 0)
                                            | (SONIQ_WPACK_DENSE if dense else 0),
                                            int(act_group_bits), _stream(stream),
                                            ctypes.byref(h)))
    return Weights(h, N, K)


def soniq_pack_weights_conv3x3(Wf, w_bits, c_bits, a_signed: bool,
                               wq_mode: int = SONIQ_WQ_SYMMETRIC, stream=None,
                               sign_nibbles: bool = False) -> Weights:
    """Pack a 3x3 filter (device float32 [N, C, 3, 3], contiguous) for the
    implicit-GEMM convolution; c_bits holds one width per input channel.
    The handle behaves as weights of K = 9*C columns (k = c*9 + kh*3 + kw)."""
    import torch
    if Wf.dtype != torch.float32 or Wf.dim() != 4 or tuple(Wf.shape[2:]) != (3, 3) \
            or not Wf.is_contiguous():
        raise TypeError("the filter must be a contiguous float32 [N, C, 3, 3] device tensor")
    N, C = Wf.shape[0], Wf.shape[1]
    wb, cb = _u8(w_bits), _u8(c_bits)
    if wb.shape != (N,) or cb.shape != (C,):
        raise ValueError("w_bits must have N entries and c_bits C entries")
    h = ctypes.c_void_p()
    _check(lib().soniq_pack_weights_conv3x3(_dev(Wf, "float32"), N, C,
                                            wb.ctypes.data_as(ctypes.c_void_p),
                                            cb.ctypes.data_as(ctypes.c_void_p),
                                            1 if a_signed else 0,
                                            int(wq_mode) | (SONIQ_WPACK_SIGN_NIBBLES if sign_nibbles else 0),
                                            _stream(stream), ctypes.byref(h)))
    return Weights(h, N, 9 * C)


def soniq_act_create_conv3x3(weights: Weights, B: int, H: int, W: int) -> Activations:
    h = ctypes.c_void_p()
    _check(lib().soniq_act_create_conv3x3(weights.handle, int(B), int(H), int(W), ctypes.byref(h)))
    return Activations(h, weights, int(B) * int(H) * int(W))


def soniq_act_create(weights: Weights, max_M: int) -> Activations:
    h = ctypes.c_void_p()
    _check(lib().soniq_act_create(weights.handle, int(max_M), ctypes.byref(h)))
    return Activations(h, weights, int(max_M))


def soniq_quantize_act(act: Activations, A, stream=None) -> None:
    """Quantize and pack A (device float32 [M, K], row-major) into `act`."""
    import torch
    if A.dtype != torch.float32 or A.dim() != 2 or A.stride(1) != 1:
        raise TypeError("A must be a 2-D float32 device tensor with unit column stride")
    if A.shape[1] != act.weights.K:
        raise ValueError("A has the wrong number of input channels")
    _check(lib().soniq_quantize_act(act.handle, _dev(A, "float32"), A.shape[0], A.stride(0),
                                    _stream(stream)))
    act.M = A.shape[0]


def soniq_quantize_act_conv3x3(act: Activations, X, stream=None) -> None:
    """Quantize and pack the activations of a stride-1, pad-1 3x3 convolution
    straight from its input X (device float32 [B, C, H, W], contiguous); the
    handle's weights are the [N, C, 3, 3] filter viewed as [N, 9C]."""
    import torch
    if X.dtype != torch.float32 or X.dim() != 4 or not X.is_contiguous():
        raise TypeError("X must be a contiguous 4-D float32 device tensor")
    B, C, H, W = X.shape
    _check(lib().soniq_quantize_act_conv3x3(act.handle, _dev(X, "float32"), B, C, H, W,
                                            _stream(stream)))
    act.M = B * H * W


def soniq_mp_gemm(act: Activations, weights: Weights, out=None, acc=None, stream=None):
    """Y[M, N] (bf16) from the last quantized activations; optional int32
    accumulator dump acc[S, M, N].  Returns Y."""
    import torch
    M, N = act.M, weights.N
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    if out.dtype != torch.bfloat16 or out.dim() != 2 or out.stride(1) != 1 or out.shape[0] < M:
        raise TypeError("out must be a bf16 [M, >=N] device tensor with unit column stride")
    accp = None
    if acc is not None:
        if acc.dtype != torch.int32 or not acc.is_contiguous() or tuple(acc.shape) != (weights.S, M, N):
            raise TypeError("acc must be a contiguous int32 [S, M, N] device tensor")
        accp = _dev(acc, "int32")
    _check(lib().soniq_mp_gemm(act.handle, weights.handle, _dev(out, "bf16"), out.stride(0),
                               accp, _stream(stream)))
    return out



def soniq_quantize_mp_gemm(act: Activations, weights: Weights, A, out=None, acc=None, stream=None):
    """soniq_quantize_act(act, A) then soniq_mp_gemm(act, weights) in one call
    (a single launch for a batch of one row).  Returns Y."""
    import torch
    if A.dtype != torch.float32 or A.dim() != 2 or A.stride(1) != 1:
        raise TypeError("A must be a 2-D float32 device tensor with unit column stride")
    if A.shape[1] != act.weights.K:
        raise ValueError("A has the wrong number of input channels")
    M, N = A.shape[0], weights.N
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    if out.dtype != torch.bfloat16 or out.dim() != 2 or out.stride(1) != 1 or out.shape[0] < M:
        raise TypeError("out must be a bf16 [M, >=N] device tensor with unit column stride")
    accp = None
    if acc is not None:
        if acc.dtype != torch.int32 or not acc.is_contiguous() or tuple(acc.shape) != (weights.S, M, N):
            raise TypeError("acc must be a contiguous int32 [S, M, N] device tensor")
        accp = _dev(acc, "int32")
    _check(lib().soniq_quantize_mp_gemm(act.handle, weights.handle, _dev(A, "float32"), M, A.stride(0),
                                        _dev(out, "bf16"), out.stride(0), accp, _stream(stream)))
    act.M = M
    return out


def soniq_quantize_mp_gemm_scratch(weights: Weights, A, out=None, acc=None, stream=None):
    """soniq_quantize_mp_gemm without an activation handle: the library's
    per-device scratch holds the packed activations, and the call allocates
    nothing (pass `out` to keep the binding from allocating Y).  Returns Y."""
    import torch
    if A.dtype != torch.float32 or A.dim() != 2 or A.stride(1) != 1:
        raise TypeError("A must be a 2-D float32 device tensor with unit column stride")
    if A.shape[1] != weights.K:
        raise ValueError("A has the wrong number of input channels")
    M, N = A.shape[0], weights.N
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    if out.dtype != torch.bfloat16 or out.dim() != 2 or out.stride(1) != 1 or out.shape[0] < M:
        raise TypeError("out must be a bf16 [M, >=N] device tensor with unit column stride")
    accp = None
    if acc is not None:
        if acc.dtype != torch.int32 or not acc.is_contiguous() or tuple(acc.shape) != (weights.S, M, N):
            raise TypeError("acc must be a contiguous int32 [S, M, N] device tensor")
        accp = _dev(acc, "int32")
    _check(lib().soniq_quantize_mp_gemm_scratch(weights.handle, _dev(A, "float32"), M, A.stride(0),
                                                _dev(out, "bf16"), out.stride(0), accp,
                                                _stream(stream)))
    return out


def soniq_mp_gemm_quantize_next(act: Activations, weights: Weights, next_act: Activations,
                                s_next, out=None, acc=None, stream=None):
    """soniq_mp_gemm(act, weights) whose epilogue also quantizes the outputs
    into next_act with the static scales s_next (one per next-layer
    activation group, or per block for sub-group weights).  out=None skips
    Y; returns out."""
    import torch
    M, N = act.M, weights.N
    sn = np.ascontiguousarray(np.asarray(s_next, np.float32).ravel())
    if sn.shape[0] < next_act.weights.S:
        raise ValueError("one static scale per next-layer activation group (or block)")
    outp, ldy = None, N
    if out is not None:
        if out.dtype != torch.bfloat16 or out.dim() != 2 or out.stride(1) != 1 or out.shape[0] < M:
            raise TypeError("out must be a bf16 [M, >=N] device tensor with unit column stride")
        outp, ldy = _dev(out, "bf16"), out.stride(0)
    accp = None
    if acc is not None:
        if acc.dtype != torch.int32 or not acc.is_contiguous() or tuple(acc.shape) != (weights.S, M, N):
            raise TypeError("acc must be a contiguous int32 [S, M, N] device tensor")
        accp = _dev(acc, "int32")
    _check(lib().soniq_mp_gemm_quantize_next(act.handle, weights.handle, next_act.handle,
                                             sn.ctypes.data_as(ctypes.c_void_p), outp, ldy, accp,
                                             _stream(stream)))
    next_act.M = M
    return out


def soniq_mp_gemm_quantize_next_max(act: Activations, weights: Weights, next_act: Activations,
                                    out=None, acc=None, stream=None):
    """soniq_mp_gemm(act, weights) storing Y (out, allocated when None) whose
    epilogue also folds each next-layer group's largest |Y|; next_act then
    holds soniq_quantize_act of float(Y) with that batch maximum.  Returns
    out."""
    import torch
    M, N = act.M, weights.N
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    if out.dtype != torch.bfloat16 or out.dim() != 2 or out.stride(1) != 1 or out.shape[0] < M:
        raise TypeError("out must be a bf16 [M, >=N] device tensor with unit column stride")
    accp = None
    if acc is not None:
        if acc.dtype != torch.int32 or not acc.is_contiguous() or tuple(acc.shape) != (weights.S, M, N):
            raise TypeError("acc must be a contiguous int32 [S, M, N] device tensor")
        accp = _dev(acc, "int32")
    _check(lib().soniq_mp_gemm_quantize_next_max(act.handle, weights.handle, next_act.handle,
                                                 _dev(out, "bf16"), out.stride(0), accp,
                                                 _stream(stream)))
    next_act.M = M
    return out


def soniq_weights_info(weights: Weights) -> WeightsInfo:
    info = WeightsInfo()
    _check(lib().soniq_weights_info(weights.handle, ctypes.byref(info)))
    return info


def soniq_plan_input_channels(a_bits):
    """Host-only input-channel plan: (pos[K], seg_len[2], seg_pad[2], S)."""
    ab = _u8(a_bits)
    K = ab.shape[0]
    pos = np.empty(K, np.int64)
    seg_len = np.zeros(2, np.int64)
    seg_pad = np.zeros(2, np.int64)
    S = ctypes.c_int32()
    _check(lib().soniq_plan_input_channels(ab.ctypes.data_as(ctypes.c_void_p), K,
                                           pos.ctypes.data_as(ctypes.c_void_p),
                                           seg_len.ctypes.data_as(ctypes.c_void_p),
                                           seg_pad.ctypes.data_as(ctypes.c_void_p),
                                           ctypes.byref(S)))
    return pos, seg_len, seg_pad, S.value


def soniq_weights_unpack_debug(weights: Weights):
    """Codes int32 [N, K] (original order) and scales float32 [N]."""
    codes = np.empty((weights.N, weights.K), np.int32)
    s_w = np.empty(weights.N, np.float32)
    _check(lib().soniq_weights_unpack_debug(weights.handle, codes.ctypes.data_as(ctypes.c_void_p),
                                            s_w.ctypes.data_as(ctypes.c_void_p)))
    return codes, s_w


def soniq_act_unpack_debug(act: Activations):
    """Codes int32 [M, K] (original order) and scales float32 [S] (one per
    precision group, or per sub-group block)."""
    codes = np.empty((act.M, act.weights.K), np.int32)
    s_a = np.zeros(max(2, act.weights.S), np.float32)
    _check(lib().soniq_act_unpack_debug(act.handle, codes.ctypes.data_as(ctypes.c_void_p),
                                        s_a.ctypes.data_as(ctypes.c_void_p)))
    return codes, s_a[: act.weights.S].copy()


def soniq_debug_stream_read(src, nbytes: int, sink, offset: int = 0, stream=None) -> None:
    """One plain read of nbytes of the device tensor src from byte offset
    `offset` (a measurement aid: the ceiling a bandwidth-bound kernel is
    held against); sink, an int32 device tensor of at least
    ceil(nbytes / 8192) elements, receives one XOR per workgroup."""
    import torch
    if not (isinstance(src, torch.Tensor) and src.is_cuda and src.is_contiguous()):
        raise TypeError("src must be a contiguous device tensor")
    if offset < 0 or offset + nbytes > src.numel() * src.element_size():
        raise ValueError("the read lies outside src")
    if sink.dtype != torch.int32 or not sink.is_cuda or sink.numel() < (nbytes + 8191) // 8192:
        raise TypeError("sink must be an int32 device tensor of ceil(nbytes / 8192) elements")
    _check(lib().soniq_debug_stream_read(ctypes.c_void_p(src.data_ptr() + offset), nbytes,
                                         _dev(sink, "int32"), _stream(stream)))


def soniq_act_wait_timeouts(act: Activations) -> int:
    """Workgroups of the single-pass quantizer whose grid wait timed out
    since the handle was made (results unchanged; the call was slow)."""
    n = ctypes.c_uint64(0)
    _check(lib().soniq_act_wait_timeouts(act.handle, ctypes.byref(n)))
    return int(n.value)


# ---- 8-bit linear layers, and the quantized key/value cache -----------------
# These calls take a few microseconds of GPU time at decode sizes, so their
# checks are written to cost little: one query of the device and the stream a
# call, sizes of workspaces remembered by their arguments.
torch = None     # imported with the first call
_TYPES = None


def _load():
    global torch, _TYPES
    import torch
    _TYPES = {torch.float32: SONIQ_F32, torch.bfloat16: SONIQ_BF16, torch.float16: SONIQ_F16,
              torch.int8: None, torch.int32: None, torch.uint8: None, torch.int64: None}
    lib()


def _device(t, what: str) -> int:
    """Index of the current device, where t has to be: the library works on the
    current device alone."""
    if torch is None:
        _load()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a device tensor")
    d = torch._C._cuda_getDevice()
    if t.get_device() != d:
        raise ValueError(f"{what} is on {t.device}, the current device is cuda:{d}")
    return d


def _raw_stream(stream, device: int):
    if stream is not None:
        return int(stream)
    return torch._C._cuda_getCurrentRawStream(device)


def _empty(like, shape, dtype, stream):
    """Memory on like's device that a call on `stream` writes: taken on that
    stream, so that it is neither in use elsewhere before nor given away too
    early after."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    s = torch.cuda.ExternalStream(int(stream), like.device) if int(stream) else torch.cuda.default_stream(like.device)
    with torch.cuda.stream(s):
        return like.new_empty(shape, dtype=dtype)


def _is(t, what: str, d: int, dtype, dim: int):
    """Refuses what is not a tensor of that type and number of dimensions on
    device d.  The checks below come here once something is amiss."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a device tensor")
    if t.get_device() != d:
        raise ValueError(f"{what} is on {t.device}, the current device is cuda:{d}")
    if t.dtype is not dtype:
        raise TypeError(f"{what} must be {dtype}")
    if t.dim() != dim:
        raise TypeError(f"{what} must have {dim} dimensions")


def _vector(t, what: str, d: int, dtype, n: int) -> int:
    """Address of a contiguous tensor of n elements."""
    try:
        if t.dtype is dtype and t.get_device() == d and t.shape == (n,) and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _is(t, what, d, dtype, 1)
    raise ValueError(f"{what} must be a contiguous tensor of {n} elements")


def _rows(t, what: str, d: int, dtype):
    """(M, K, leading dimension, address) of an [M, K] tensor with unit column
    stride (a stride says nothing where there is one row, or one column)."""
    try:
        if t.dtype is dtype and t.get_device() == d:
            M, K = t.shape
            ld, unit = t.stride()
            if unit == 1 and ld >= K:
                return M, K, ld, t.data_ptr()
    except (AttributeError, ValueError):
        pass
    _is(t, what, d, dtype, 2)
    M, K = t.shape
    ld, unit = t.stride()
    if unit != 1 and K > 1:
        raise TypeError(f"{what} must have unit column stride")
    if ld < K and M > 1:
        raise TypeError(f"{what} has rows that overlap")
    return M, K, max(ld, K), t.data_ptr()


def _type_of(t, what: str) -> int:
    code = _TYPES.get(getattr(t, "dtype", t))
    if code is None:
        raise TypeError(f"{what} must be float32, bfloat16 or float16")
    return code


def soniq_quantize_rows(A, out=None, scales=None, stream=None):
    """Symmetric 8-bit codes of the rows of A (device float32, bfloat16 or
    float16 [M, K]) with one scale each: tokens, or the output channels of a
    weight matrix.  Returns (codes int8 [M, K], scales float32 [M])."""
    d = _device(A, "A")
    ta = _type_of(A, "A")
    M, K, lda, a = _rows(A, "A", d, A.dtype)
    if out is None:
        ldq = -(-K // 16) * 16
        out = _empty(A, (M, ldq), torch.int8, stream)[:, :K]
        q = out.data_ptr()
    else:
        Mq, Kq, ldq, q = _rows(out, "out", d, torch.int8)
        if Mq != M or Kq != K:
            raise ValueError("out must have A's shape")
    if scales is None:
        scales = _empty(A, (M,), torch.float32, stream)
    s = _vector(scales, "scales", d, torch.float32, M)
    _check(_lib.soniq_quantize_rows(a, ta, M, K, lda, q, ldq, s, _raw_stream(stream, d)))
    return out, scales


def _i8_weights(W, s_w, bias, d, K):
    """N, then the C arguments W, ldw, s_w, bias."""
    N, Kw, ldw, w = _rows(W, "W", d, torch.int8)
    if Kw != K:
        raise ValueError("W has the wrong number of input channels")
    return N, w, ldw, _vector(s_w, "s_w", d, torch.float32, N), \
        None if bias is None else _vector(bias, "bias", d, torch.float32, N)


def _i8_out(A, M, N, out, dtype, d, stream):
    """out, then the C arguments Y, y_type, ldy."""
    if out is None:
        dtype = torch.bfloat16 if dtype is None else dtype
        code = _type_of(dtype, "dtype")
        out = _empty(A, (M, N), dtype, stream)
        return out, out.data_ptr(), code, N
    code = _type_of(out, "out")
    My, Ny, ldy, y = _rows(out, "out", d, out.dtype if dtype is None else dtype)
    if My != M or Ny != N:
        raise ValueError("out must be [M, N]")
    return out, y, code, ldy


def soniq_i8_gemm(A, s_a, W, s_w, bias=None, out=None, dtype=None, stream=None):
    """Y = (A W^T) * s_a[:, None] * s_w + bias of int8 codes A [M, K] and
    W [N, K] with float32 scales per row; Y [M, N] of `dtype` (bfloat16 unless
    given).  Returns Y."""
    d = _device(A, "A")
    M, K, lda, a = _rows(A, "A", d, torch.int8)
    sa = _vector(s_a, "s_a", d, torch.float32, M)
    N, w, ldw, sw, b = _i8_weights(W, s_w, bias, d, K)
    out, y, ty, ldy = _i8_out(A, M, N, out, dtype, d, stream)
    _check(_lib.soniq_i8_gemm(a, lda, sa, w, ldw, sw, b, M, N, K, y, ty, ldy, _raw_stream(stream, d)))
    return out


@functools.lru_cache(maxsize=4096)
def soniq_quantize_i8_gemm_workspace(M: int, K: int) -> int:
    n = ctypes.c_int64()
    _check(lib().soniq_quantize_i8_gemm_workspace(M, K, ctypes.byref(n)))
    return n.value


def _work(work, need: int, d: int, like, stream):
    """The workspace, its address and size: the caller's, or one of `need`
    bytes that lives until the call returns."""
    if work is None:
        if need == 0:
            return None, None, 0
        work = _empty(like, (need,), torch.uint8, stream)
        return work, work.data_ptr(), need
    _is(work, "work", d, torch.uint8, 1)
    if not work.is_contiguous():
        raise ValueError("work must be contiguous")
    return work, work.data_ptr(), work.numel()


def soniq_quantize_i8_gemm(A, W, s_w, bias=None, out=None, dtype=None, work=None, stream=None):
    """soniq_quantize_rows(A), then soniq_i8_gemm with W and s_w, in one call.
    work: a uint8 device tensor of soniq_quantize_i8_gemm_workspace(M, K)
    bytes (allocated when None).  Returns Y."""
    d = _device(A, "A")
    ta = _type_of(A, "A")
    M, K, lda, a = _rows(A, "A", d, A.dtype)
    N, w, ldw, sw, b = _i8_weights(W, s_w, bias, d, K)
    out, y, ty, ldy = _i8_out(A, M, N, out, dtype, d, stream)
    work, wp, wn = _work(work, soniq_quantize_i8_gemm_workspace(M, K), d, A, stream)
    _check(_lib.soniq_quantize_i8_gemm(a, ta, lda, w, ldw, sw, b, M, N, K, y, ty, ldy, wp, wn,
                                        _raw_stream(stream, d)))
    return out


class KVCache:
    """A key/value cache of 8- or 4-bit codes in pages (soniq_kv_cache_t).

    k, v: int8 or uint8 codes [pages, heads, page_size, head_dim * bits / 8];
    k_scale, v_scale: float32 [pages, heads, page_size]; all contiguous, on
    one device.  The object keeps the tensors; they stay the caller's to read,
    copy and move.  KVCache.empty makes them."""

    def __init__(self, k, k_scale, v, v_scale, bits: int = 8):
        d = _device(k, "k")
        for t, what in ((k, "k"), (v, "v")):
            _is(t, what, d, t.dtype, 4)
            if t.dtype not in (torch.int8, torch.uint8) or not t.is_contiguous():
                raise TypeError(f"{what} must be a contiguous int8 or uint8 tensor")
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _is(t, what, d, torch.float32, 3)
            if not t.is_contiguous():
                raise TypeError(f"{what} must be contiguous")
        if bits not in (4, 8):
            raise ValueError("bits must be 4 or 8")
        if v.shape != k.shape or k_scale.shape != k.shape[:3] or v_scale.shape != k.shape[:3]:
            raise ValueError("k, v and the scales have different extents")
        self.k, self.k_scale, self.v, self.v_scale, self.bits = k, k_scale, v, v_scale, bits
        self.pages, self.heads, self.page_size, width = k.shape
        if self.pages * self.heads * self.page_size >= 1 << 31:
            raise ValueError("a cache has fewer than 2^31 rows")
        self.head_dim = width * 8 // bits
        self.device, self.device_index = k.device, d
        self._c = KVCacheStruct(k.data_ptr(), k_scale.data_ptr(), v.data_ptr(), v_scale.data_ptr(),
                                self.pages, self.page_size, self.heads, self.head_dim, bits)
        self._ref = ctypes.addressof(self._c)

    @classmethod
    def empty(cls, pages: int, page_size: int, heads: int, head_dim: int, bits: int = 8):
        """A cache of zeros on the current device."""
        if torch is None:
            _load()
        if bits not in (4, 8) or head_dim * bits % 8:
            raise ValueError("bits must be 4 or 8, and a row a whole number of bytes")
        device = torch.device("cuda", torch.cuda.current_device())
        codes = lambda: torch.zeros((pages, heads, page_size, head_dim * bits // 8), dtype=torch.int8, device=device)  # noqa: E731
        scales = lambda: torch.zeros((pages, heads, page_size), dtype=torch.float32, device=device)  # noqa: E731
        return cls(codes(), scales(), codes(), scales(), bits)


def _kv_batch(cache, page_table, cu, lengths, what):
    """Device, and (B, width, leading dimension, addresses) of a ragged batch."""
    d = cache.device_index
    if torch._C._cuda_getDevice() != d:
        raise ValueError(f"the cache is on {cache.device}, the current device is another one")
    B, width, ld, table = _rows(page_table, "page_table", d, torch.int32)
    return (d, B, width, ld, table, _vector(cu, "cu", d, torch.int32, B + 1),
            _vector(lengths, what, d, torch.int32, B))


def _kv_rows(t, what: str, d: int, heads: int, head_dim: int):
    """Tokens, type code, strides and address of a [T, heads, head_dim] tensor."""
    code = _type_of(t, what)
    try:
        T, h, n = t.shape
    except (AttributeError, ValueError):
        T = h = n = -1
    if t.get_device() != d or T < 0:
        _is(t, what, d, t.dtype, 3)
    if h != heads or n != head_dim:
        raise ValueError(f"{what} must be [T, {heads}, {head_dim}]")
    ts, hs, unit = t.stride()
    if unit != 1:
        raise TypeError(f"{what} must have unit stride in its last dimension")
    return T, code, ts, hs, t.data_ptr()


def _kv_out(t, what: str, ts: int, hs: int):
    """An output's rows must not overlap."""
    T, heads, n = t.shape
    (a, na), (b, nb) = sorted(((ts, T), (hs, heads)))
    if T * heads and ((na > 1 and a < n) or (nb > 1 and b < (a * (na - 1) if na > 1 else 0) + n)):
        raise TypeError(f"{what} has rows that overlap")


def soniq_kv_write(cache: KVCache, K, V, page_table, cu, start, stream=None) -> None:
    """Quantizes new keys and values [T, heads, head_dim] into the cache: row
    cu[b] + i goes to position start[b] + i of sequence b, whose pages
    page_table[b] names.  page_table int32 [B, width], cu int32 [B + 1],
    start int32 [B], all on the device."""
    d, B, width, ld, table, cu, start = _kv_batch(cache, page_table, cu, start, "start")
    T, tk, kts, khs, k = _kv_rows(K, "K", d, cache.heads, cache.head_dim)
    Tv, tv, vts, vhs, v = _kv_rows(V, "V", d, cache.heads, cache.head_dim)
    if tk != tv or T != Tv:
        raise ValueError("K and V must have one type and one number of tokens")
    _check(_lib.soniq_kv_write(cache._ref, k, kts, khs, v, vts, vhs, tk, T, table, ld, width, B, cu, start,
                                _raw_stream(stream, d)))


def soniq_kv_read(cache: KVCache, page_table, cu, start, tokens: int, dtype=None, out=None, stream=None):
    """The values of cached positions: position start[b] + i of sequence b in
    row cu[b] + i of K and V [tokens, heads, head_dim] (of `dtype`, bfloat16
    unless given, or into the pair `out`).  Returns (K, V); rows from cu[B] on
    are left as they are (out=None: uninitialised)."""
    d, B, width, ld, table, cu, start = _kv_batch(cache, page_table, cu, start, "start")
    heads, D = cache.heads, cache.head_dim
    if out is None:
        dtype = torch.bfloat16 if dtype is None else dtype
        tk = _type_of(dtype, "dtype")
        K, V = _empty(cache.k, (2, tokens, heads, D), dtype, stream).unbind(0)
        kts = vts = heads * D
        khs = vhs = D
        k, v = K.data_ptr(), V.data_ptr()
    else:
        K, V = out
        Tk, tk, kts, khs, k = _kv_rows(K, "K", d, heads, D)
        Tv, tv, vts, vhs, v = _kv_rows(V, "V", d, heads, D)
        if tk != tv or Tk != tokens or Tv != tokens or (dtype is not None and K.dtype is not dtype):
            raise ValueError("K and V must have one type (dtype) and `tokens` rows")
        _kv_out(K, "K", kts, khs)
        _kv_out(V, "V", vts, vhs)
    _check(_lib.soniq_kv_read(cache._ref, k, kts, khs, v, vts, vhs, tk, tokens, table, ld, width, B, cu, start,
                               _raw_stream(stream, d)))
    return K, V


@functools.lru_cache(maxsize=4096)
def _kv_work(pages, page_size, heads, head_dim, bits, tokens, q_heads, B, max_q, max_kv) -> int:
    # the pointers say nothing about the size, but have to look like a cache's
    c = KVCacheStruct(16, 16, 16, 16, pages, page_size, heads, head_dim, bits)
    n = ctypes.c_int64()
    _check(lib().soniq_kv_attention_workspace(ctypes.addressof(c), tokens, q_heads, B, max_q, max_kv,
                                              ctypes.byref(n)))
    return n.value


def soniq_kv_attention_workspace(cache: KVCache, tokens: int, q_heads: int, B: int, max_q: int,
                                 max_kv: int) -> int:
    return _kv_work(cache.pages, cache.page_size, cache.heads, cache.head_dim, cache.bits, tokens, q_heads, B,
                    max_q, max_kv)


def soniq_kv_attention(cache: KVCache, q, page_table, cu, kv_len, scale=None, mask=None, max_q=None,
                       max_kv=None, out=None, lse=None, work=None, stream=None):
    """Attention of new tokens q [T, q_heads, head_dim] (bfloat16 or float16)
    over the cache that already holds their keys and values.  Sequence b has
    kv_len[b] positions, the last cu[b+1] - cu[b] of them its new tokens'.
    mask (int64 [T, words]): bit j % 64 of word j / 64 of a row says whether
    that token sees new token j of its sequence; None: each sees the new ones
    up to itself.  scale: 1 / sqrt(head_dim) unless given.  max_q: the most
    new tokens of a sequence, at most 256 (T unless given; has to be given for
    batches of more than 256 tokens, however few of each sequence); max_kv:
    the longest kv_len, a hint.  lse: a float32 [T, q_heads] tensor to fill.
    work: a uint8 device tensor of soniq_kv_attention_workspace(...) bytes
    (allocated when None).  Returns out (like q)."""
    d, B, width, ld, table, cu, kv_len = _kv_batch(cache, page_table, cu, kv_len, "kv_len")
    D = cache.head_dim
    heads = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
    T, code, qts, qhs, qp = _kv_rows(q, "q", d, heads, D)
    if out is None:
        out = _empty(q, (T, heads, D), q.dtype, stream)
        ots, ohs = heads * D, D
    else:
        To, to, ots, ohs, _ = _kv_rows(out, "out", d, heads, D)
        if to != code or To != T:
            raise ValueError("out must have q's shape and type")
        _kv_out(out, "out", ots, ohs)
    words, bits = 0, None
    if mask is not None:
        _is(mask, "mask", d, torch.int64, 2)
        if mask.shape[0] != T or not mask.is_contiguous():
            raise ValueError("mask must be a contiguous [T, words] tensor")
        if mask.shape[1] == 0:                        # its address is null: the library would see no mask
            raise ValueError("mask must have at least one word")
        if T:
            words, bits = mask.shape[1], mask.data_ptr()
    if lse is not None:
        _is(lse, "lse", d, torch.float32, 2)
        if lse.shape[0] != T or lse.shape[1] != heads or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous [T, q_heads] tensor")
    if max_q is None:
        if T > 256:                                   # the sequences' numbers are on the device
            raise ValueError(f"q has {T} tokens: give max_q, the most of one sequence (at most 256)")
        max_q = max(T, 1)
    if max_kv is None:
        max_kv = width * cache.page_size
    need = _kv_work(cache.pages, cache.page_size, cache.heads, D, cache.bits, T, heads, B, max_q, max_kv)
    work, wp, wn = _work(work, need, d, q, stream)
    _check(_lib.soniq_kv_attention(cache._ref, qp, qts, qhs, code, T, heads, table, ld, width, B, cu, kv_len, bits,
                                    words, D ** -0.5 if scale is None else scale, max_q, max_kv, out.data_ptr(), ots,
                                    ohs, None if lse is None else lse.data_ptr(), wp, wn, _raw_stream(stream, d)))
    return out
