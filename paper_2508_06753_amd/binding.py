"""Thin ctypes binding over the C ABI declared in include/w2mm.h.

Argument marshalling only: every step of the path runs in the HIP kernels of
libw2mm.so.  torch is used for device memory and streams.  There is no CPU
fallback: if the shared library is missing or fails to load, importing this
module raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libw2mm.so")

CODEC_INT2, CODEC_TERNARY = 0, 1
DT_F32, DT_BF16 = 0, 1
VARIANT_AUTO, VARIANT_DOT4, VARIANT_SMALLM, VARIANT_TILED, VARIANT_MIDM, VARIANT_SCALED16 = 0, 1, 2, 3, 4, 5
VARIANT_GEMV = 6

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED_SHAPE, ERR_MISALIGNED = -1, -2, -3
ERR_BUFFER_TOO_SMALL, ERR_HIP, ERR_BAD_CODE = -4, -5, -6

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2508_06753_amd.build` "
        "(there is no CPU fallback)")

_lib = ctypes.CDLL(LIB_PATH)

_i64, _int, _sz, _vp = ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p
_dbl = ctypes.c_double
_SIGS = {
    "w2_packed_size": [_i64, _i64, _int, ctypes.POINTER(_sz)],
    "w2_prepack": [_vp, _vp, _i64, _i64, _int, _int, _vp, _sz, _vp, _vp],
    "w2_quantize_rows": [_vp, _int, _i64, _i64, _i64, _int, _vp, _vp, _vp, _vp],
    "w2_matmul_a8": [_vp, _i64, _i64, _int, _vp, _vp, _i64, _vp, _i64, _vp, _sz, _vp],
    "w2_matmul_a8_ex": [_vp, _i64, _i64, _int, _vp, _vp, _i64, _vp, _i64, _vp, _sz, _vp, _vp],
    "w2_matmul_a8_fused": [_vp, _i64, _i64, _int, _vp, _int, _i64, _i64, _vp, _i64, _vp, _sz, _vp],
    "w2_init": [],
    "w2_matmul_a8_fused_noalloc": [_vp, _i64, _i64, _int, _vp, _int, _i64, _i64, _vp, _i64, _vp],
    "w2_matmul_a16": [_vp, _i64, _i64, _int, _vp, _i64, _i64, _vp, _i64, _vp, _sz, _vp],
    "w2_matmul_a16_ex": [_vp, _i64, _i64, _int, _vp, _i64, _i64, _vp, _i64, _vp, _sz, _vp, _vp],
    "w2_workspace_size": [_i64, _i64, _i64, _int, _int, ctypes.POINTER(_sz)],
    "w2_debug_group_acc_a8": [_vp, _i64, _i64, _int, _vp, _i64, _vp, _vp, _vp],
    "w2_debug_unpack": [_vp, _i64, _i64, _int, _int, _vp, _vp, _vp],
    "w2_debug_stream_read": [_vp, _sz, _vp, _vp, _vp],
    "w2_debug_int8_gemv": [_vp, _i64, _i64, _vp, _vp, _vp],
    "w2_matmul_a8_epi": [_vp, _i64, _i64, _int, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _sz, _vp, _vp],
    "w2_matmul_a16_epi": [_vp, _i64, _i64, _int, _vp, _i64, _i64, _vp, _i64, _vp, _vp, _sz, _vp, _vp],
    "w2_matmul_a8_fused_epi": [_vp, _i64, _i64, _int, _vp, _int, _i64, _i64, _vp, _i64, _vp, _vp, _sz, _vp, _vp],
    "w2_lora_workspace_size": [_vp, _i64, _i64, _i64, ctypes.POINTER(_sz)],
    "w2_lora_add": [_vp, _i64, _i64, _vp, _int, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _int, _vp, _sz, _vp],
    "w2_rope_phases": [_dbl, _int, _int, _dbl, _dbl, _dbl, _dbl, _vp],
    "w2_qk_norm_rope": [_vp, _i64, _i64, _int, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _i64, _vp, _vp, _vp],
    "w2_tree_attention_workspace_size": [_i64, _i64, _int, _int, _int, _i64, _i64, _i64, ctypes.POINTER(_sz)],
    "w2_tree_attention": [_vp, _i64, _i64, _int, _vp, _vp, _i64, _i64, _vp, _vp, _i64, _i64, _i64, _i64, _vp, _int,
                          ctypes.c_float, _vp, _i64, _vp, _vp, _sz, _vp],
}
for _name, _args in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _int
_lib.w2_status_string.argtypes = [_int]
_lib.w2_status_string.restype = ctypes.c_char_p
_lib.w2_last_error.argtypes = []
_lib.w2_last_error.restype = ctypes.c_char_p

EXPORTED = sorted(list(_SIGS) + ["w2_status_string", "w2_last_error"])


class W2Error(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        detail = _lib.w2_last_error().decode()
        super().__init__(f"{fn}: {_lib.w2_status_string(status).decode()} ({status}): {detail}")


def raw():
    """The ctypes library object (tests call entry points with raw pointers)."""
    return _lib


def _check(fn, status):
    if status != OK:
        raise W2Error(fn, status)


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle, looked up on every call.  torch.cuda.current_stream() builds a Stream object for it:
# 2.8 us of a 9.7 us call (one row, 2048 x 2048) where these two take 0.2; without them, the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)
if _raw_stream is not None and _raw_device is not None:
    def _stream():
        return _raw_stream(_raw_device())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def _dev(t, dtype, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t


def packed_size(K, N, G):
    out = _sz(0)
    _check("w2_packed_size", _lib.w2_packed_size(K, N, G, ctypes.byref(out)))
    return out.value


def workspace_size(M, K, N, G, a16=False):
    out = _sz(0)
    _check("w2_workspace_size", _lib.w2_workspace_size(M, K, N, G, int(a16), ctypes.byref(out)))
    return out.value


def prepack(codes, scales, G, codec=CODEC_INT2, bad_codes=None):
    """codes uint8 [K,N], scales bf16 bits (int16/uint16 storage) [K/G,N], both on device.
    Returns the packed blob (uint8 tensor)."""
    _dev(codes, torch.uint8, "codes")
    K, N = codes.shape
    if scales.dtype not in (torch.int16, torch.uint16, torch.bfloat16) or not scales.is_cuda:
        raise ValueError("scales must be a 16-bit device tensor")
    if tuple(scales.shape) != (K // G, N):
        raise ValueError("scales must be [K/G, N]")
    codes, scales = codes.contiguous(), scales.contiguous()
    nbytes = packed_size(K, N, G)
    packed = torch.empty(nbytes, dtype=torch.uint8, device=codes.device)
    _check("w2_prepack", _lib.w2_prepack(_ptr(codes), _ptr(scales), K, N, G, codec, _ptr(packed),
                                         nbytes, _ptr(bad_codes), _stream()))
    return packed


def quantize_rows(X, G=128, want_gsum=False):
    """X fp32 or bf16 [M,K] on device (row stride may exceed K).  Returns (xq, sx, gsum|None)."""
    if X.dtype == torch.float32:
        dt = DT_F32
    elif X.dtype == torch.bfloat16:
        dt = DT_BF16
    else:
        raise ValueError("X must be float32 or bfloat16")
    if not X.is_cuda or X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be a 2-D device tensor with unit inner stride")
    M, K = X.shape
    xq = torch.empty((M, K), dtype=torch.int8, device=X.device)
    sx = torch.empty((M,), dtype=torch.float32, device=X.device)
    gsum = torch.empty((M, K // G), dtype=torch.int32, device=X.device) if want_gsum else None
    ldx = X.stride(0) if M > 1 else K
    _check("w2_quantize_rows", _lib.w2_quantize_rows(_ptr(X), dt, M, K, ldx, G, _ptr(xq), _ptr(sx),
                                                     _ptr(gsum), _stream()))
    return xq, sx, gsum


class Tuning(ctypes.Structure):
    """w2_tuning_t: overrides for tests and sweeps; every field 0 = the library's own rule."""
    _fields_ = [(n, ctypes.c_int) for n in (
        "variant", "dot4_max_m", "midm_min_m", "midm_max_m", "small_waves", "small_cbw", "small_kc", "gemv_window",
        "gemv_max_m", "midm_cbw", "tiled_bm", "tiled_bn", "tiled_kw", "tiled_wd", "tiled_group_m", "splitk", "splitk_min_tiles", "stream_unroll", "stream_blocks",
        "gemv_cbw", "gemv_ks", "fused_rows")]


def _tune(variant=VARIANT_AUTO, tune=None):
    """NULL when nothing is overridden, else a Tuning (kept alive by the caller's frame)."""
    if tune is None and variant == VARIANT_AUTO:
        return None
    t = Tuning()
    if isinstance(tune, Tuning):
        ctypes.memmove(ctypes.byref(t), ctypes.byref(tune), ctypes.sizeof(t))
    elif tune:
        for k, v in tune.items():
            if not hasattr(t, k):
                raise ValueError(f"w2_tuning_t has no field {k}")
            setattr(t, k, int(v))
    if variant != VARIANT_AUTO:
        t.variant = int(variant)
    return t


def _tp(t):
    return None if t is None else ctypes.byref(t)


def _ws(workspace):
    if workspace is None:
        return None, 0
    _dev(workspace, torch.uint8, "workspace")
    return _ptr(workspace), workspace.numel()


def matmul_a8(packed, K, N, G, xq, sx, out=None, variant=VARIANT_AUTO, workspace=None, tune=None):
    """Y bf16 [M,N] = dequant-fused int8 matmul.  xq int8 [M,K], sx fp32 [M].  `workspace`: optional uint8
    device tensor; with workspace_size(M, K, N, G) bytes the tiled kernel may split K across workgroups."""
    _dev(xq, torch.int8, "xq")
    _dev(sx, torch.float32, "sx")
    M = xq.shape[0]
    if tuple(xq.shape) != (M, K) or not xq.is_contiguous() or tuple(sx.shape) != (M,):
        raise ValueError("xq must be contiguous [M,K], sx [M]")
    Y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=xq.device)
    ldy = Y.stride(0) if M > 1 else N
    wp, wb = _ws(workspace)
    t = _tune(variant, tune)
    _check("w2_matmul_a8", _lib.w2_matmul_a8_ex(_ptr(packed), K, N, G, _ptr(xq), _ptr(sx), M,
                                                _ptr(Y), ldy, wp, wb, _tp(t), _stream()))
    return Y


ACT_NONE, ACT_SILU, ACT_SILU_MUL = 0, 1, 2


class _Epilogue(ctypes.Structure):
    _fields_ = [("bias", ctypes.c_void_p), ("act", ctypes.c_int)]


def _epi(bias, act, N):
    if bias is not None:
        if bias.dtype not in (torch.int16, torch.bfloat16) or bias.numel() != N or not bias.is_cuda:
            raise ValueError("bias must be a device tensor of N bf16 values")
    return _Epilogue(bias.data_ptr() if bias is not None else None, int(act))


def matmul_a8_epi(packed, K, N, G, xq, sx, bias=None, act=ACT_NONE, out=None, variant=VARIANT_AUTO, workspace=None,
                  tune=None):
    """matmul_a8 with the fused epilogue: bias (bf16 [N]) and activation; ACT_SILU_MUL gives N/2 columns."""
    _dev(xq, torch.int8, "xq")
    _dev(sx, torch.float32, "sx")
    M = xq.shape[0]
    if tuple(xq.shape) != (M, K) or not xq.is_contiguous() or tuple(sx.shape) != (M,):
        raise ValueError("xq must be contiguous [M,K], sx [M]")
    n_out = N // 2 if act == ACT_SILU_MUL else N
    Y = out if out is not None else torch.empty((M, n_out), dtype=torch.bfloat16, device=xq.device)
    ldy = Y.stride(0) if M > 1 else n_out
    e = _epi(bias, act, N)
    wp, wb = _ws(workspace)
    t = _tune(variant, tune)
    _check("w2_matmul_a8_epi", _lib.w2_matmul_a8_epi(_ptr(packed), K, N, G, _ptr(xq), _ptr(sx), M, _ptr(Y), ldy,
                                                     ctypes.byref(e), wp, wb, _tp(t), _stream()))
    return Y


def matmul_a8_fused_epi(packed, K, N, G, X, bias=None, act=ACT_NONE, out=None, workspace=None, tune=None):
    """matmul_a8_fused with the fused epilogue."""
    if X.dtype == torch.float32:
        dt = DT_F32
    elif X.dtype == torch.bfloat16:
        dt = DT_BF16
    else:
        raise ValueError("X must be float32 or bfloat16")
    if not X.is_cuda or X.dim() != 2 or X.shape[1] != K or X.stride(1) != 1:
        raise ValueError("X must be a device tensor [M,K] with unit inner stride")
    M = X.shape[0]
    n_out = N // 2 if act == ACT_SILU_MUL else N
    Y = out if out is not None else torch.empty((M, n_out), dtype=torch.bfloat16, device=X.device)
    ldx = X.stride(0) if M > 1 else K
    ldy = Y.stride(0) if M > 1 else n_out
    e = _epi(bias, act, N)
    wp, wb = _ws(workspace)
    t = _tune(VARIANT_AUTO, tune)
    _check("w2_matmul_a8_fused_epi", _lib.w2_matmul_a8_fused_epi(_ptr(packed), K, N, G, _ptr(X), dt, ldx, M,
                                                                 _ptr(Y), ldy, ctypes.byref(e), wp, wb, _tp(t),
                                                                 _stream()))
    return Y


def matmul_a16_epi(packed, K, N, G, X, bias=None, act=ACT_NONE, out=None, variant=VARIANT_AUTO, workspace=None,
                   tune=None):
    """matmul_a16 with the fused epilogue."""
    _dev(X, torch.bfloat16, "X")
    M = X.shape[0]
    if X.dim() != 2 or X.shape[1] != K or X.stride(1) != 1:
        raise ValueError("X must be [M,K] with unit inner stride")
    n_out = N // 2 if act == ACT_SILU_MUL else N
    Y = out if out is not None else torch.empty((M, n_out), dtype=torch.bfloat16, device=X.device)
    ldx = X.stride(0) if M > 1 else K
    ldy = Y.stride(0) if M > 1 else n_out
    e = _epi(bias, act, N)
    wp, wb = _ws(workspace)
    t = _tune(variant, tune)
    _check("w2_matmul_a16_epi", _lib.w2_matmul_a16_epi(_ptr(packed), K, N, G, _ptr(X), ldx, M, _ptr(Y), ldy,
                                                       ctypes.byref(e), wp, wb, _tp(t), _stream()))
    return Y


def matmul_a8_fused(packed, K, N, G, X, out=None, workspace=None):
    """Y bf16 [M,N] from unquantised X (fp32 or bf16); `workspace`: a uint8 device tensor of
    workspace_size(M, K, N, G) bytes, needed for M > 4."""
    if X.dtype == torch.float32:
        dt = DT_F32
    elif X.dtype == torch.bfloat16:
        dt = DT_BF16
    else:
        raise ValueError("X must be float32 or bfloat16")
    if not X.is_cuda or X.dim() != 2 or X.shape[1] != K or X.stride(1) != 1:
        raise ValueError("X must be a device tensor [M,K] with unit inner stride")
    M = X.shape[0]
    Y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    ldx = X.stride(0) if M > 1 else K
    ldy = Y.stride(0) if M > 1 else N
    ws, ws_bytes = (None, 0) if workspace is None else (_ptr(workspace), workspace.numel() * workspace.element_size())
    _check("w2_matmul_a8_fused", _lib.w2_matmul_a8_fused(_ptr(packed), K, N, G, _ptr(X), dt, ldx, M,
                                                         _ptr(Y), ldy, ws, ws_bytes, _stream()))
    return Y


NOALLOC_SCRATCH_BYTES = 24 << 20


def init():
    """Resolves the built-in scratch buffer's address on the current device (optional; see the header)."""
    _check("w2_init", _lib.w2_init())


def matmul_a8_fused_noalloc(packed, K, N, G, X, out):
    """matmul_a8_fused out of the library's built-in scratch buffer: the call allocates nothing, so `out`
    (bf16 [M,N]) is required."""
    if X.dtype == torch.float32:
        dt = DT_F32
    elif X.dtype == torch.bfloat16:
        dt = DT_BF16
    else:
        raise ValueError("X must be float32 or bfloat16")
    if not X.is_cuda or X.dim() != 2 or X.shape[1] != K or X.stride(1) != 1:
        raise ValueError("X must be a device tensor [M,K] with unit inner stride")
    M = X.shape[0]
    _dev(out, torch.bfloat16, "out")
    ldx = X.stride(0) if M > 1 else K
    ldy = out.stride(0) if M > 1 else N
    _check("w2_matmul_a8_fused_noalloc", _lib.w2_matmul_a8_fused_noalloc(_ptr(packed), K, N, G, _ptr(X), dt, ldx, M,
                                                                         _ptr(out), ldy, _stream()))
    return out


def matmul_a16(packed, K, N, G, X, out=None, variant=VARIANT_AUTO, workspace=None, tune=None):
    """Y bf16 [M,N] from bf16 activations X [M,K] (unquantised).  `workspace`: as for matmul_a8
    (workspace_size(..., a16=True) bytes)."""
    _dev(X, torch.bfloat16, "X")
    M = X.shape[0]
    if X.dim() != 2 or X.shape[1] != K or X.stride(1) != 1:
        raise ValueError("X must be [M,K] with unit inner stride")
    Y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    ldx = X.stride(0) if M > 1 else K
    ldy = Y.stride(0) if M > 1 else N
    wp, wb = _ws(workspace)
    t = _tune(variant, tune)
    _check("w2_matmul_a16", _lib.w2_matmul_a16_ex(_ptr(packed), K, N, G, _ptr(X), ldx, M, _ptr(Y),
                                                  ldy, wp, wb, _tp(t), _stream()))
    return Y


# ---- the operators between the projections of an attention block

_BF16, _F32, _I32, _I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


def _vector(t, dtype, n, name, what):
    """A dense one-dimensional device tensor of n elements (checks in the order of their cost: these calls are short)."""
    if t.dtype is not dtype or t.numel() != n or t.dim() != 1 or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be a contiguous device tensor {what} of {dtype}")
    return t.data_ptr()


def _rows(t, dtype, M, N, name):
    """A device tensor [M, N] with unit inner stride -> (address, row stride)."""
    if t.dtype is not dtype or t.shape != (M, N) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor [{M}, {N}] of {dtype}")
    s = t.stride()
    if s[1] != 1 and N > 1:
        raise ValueError(f"{name} must have unit inner stride")
    return t.data_ptr(), s[0] if M > 1 else N


def _heads(t, M, n, D, name):
    """A bf16 device tensor [M, n, D], dense within a row -> (address, row stride)."""
    if t.dtype is not _BF16 or t.shape != (M, n, D) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor [{M}, {n}, {D}] of bfloat16")
    s = t.stride()
    if s[2] != 1 or (n > 1 and s[1] != D):
        raise ValueError(f"{name} must be dense within a row")
    return t.data_ptr(), s[0] if M > 1 else n * D


class _LoraStruct(ctypes.Structure):
    _fields_ = [("A", _vp), ("B", _vp), ("rank", _vp), ("scale", _vp), ("a_stride", _i64), ("b_stride", _i64),
                ("part_end", _i64 * 4), ("n_adapters", _int), ("max_rank", _int), ("n_parts", _int), ("gated", _int)]


class Lora:
    """Low-rank adapters of one projection [K -> N], laid out once (w2_lora_t).

    A bf16 [n_adapters, parts * max_rank, K], B bf16 [n_adapters, N, max_rank]; rank int32 / scale fp32 [n_adapters] on
    the device or None.  `parts`: the widths of the column ranges that have an A of their own (default: one);
    gated=True: gate and up columns alternate by 16 instead."""

    def __init__(self, A, B, rank=None, scale=None, parts=None, gated=False):
        _dev(A, torch.bfloat16, "A")
        _dev(B, torch.bfloat16, "B")
        if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[0] < 1:
            raise ValueError("A must be [n_adapters, parts * max_rank, K] and B [n_adapters, N, max_rank]")
        n, N, R = B.shape
        if gated and parts is not None:
            raise ValueError("gated adapters have their two parts by blocks of 16 columns: give no widths")
        widths = [N] if parts is None else [int(w) for w in parts]
        n_parts = 2 if gated else len(widths)
        if not 1 <= n_parts <= 4 or sum(widths) != N or min(widths) <= 0:
            raise ValueError("parts must be one to four positive widths that add up to N")
        if A.shape[1] != n_parts * R:
            raise ValueError("A must have parts * max_rank rows")
        if A.stride(2) != 1 or A.stride(1) != A.shape[2] or B.stride(2) != 1 or B.stride(1) != R:
            raise ValueError("A and B must be dense within an adapter")
        for t, dt, name in ((rank, torch.int32, "rank"), (scale, torch.float32, "scale")):
            if t is not None and (_dev(t, dt, name).shape != (n,) or not t.is_contiguous()):
                raise ValueError(f"{name} must be contiguous [n_adapters]")
        self.A, self.B, self.rank, self.scale = A, B, rank, scale
        self.K, self.N, self.max_rank, self.n_adapters, self.n_parts, self.gated = A.shape[2], N, R, n, n_parts, gated
        ends = [sum(widths[:i + 1]) for i in range(len(widths))] + [0] * (4 - len(widths))
        self._c = _LoraStruct(_ptr(A), _ptr(B), _ptr(rank), _ptr(scale), A.stride(0), B.stride(0), (_i64 * 4)(*ends), n, R,
                              n_parts, int(gated))
        self._ref = ctypes.byref(self._c)


def lora_workspace_size(lora, M):
    out = _sz(0)
    _check("w2_lora_workspace_size", _lib.w2_lora_workspace_size(lora._ref, M, lora.K, lora.N, ctypes.byref(out)))
    return out.value


def lora_add(lora, X, adapter, base, act=ACT_NONE, out=None, workspace=None):
    """Y bf16 = act(base + scale * (X A^T) B^T), each row of X (fp32 or bf16 [M,K]) with the adapter that `adapter` (int32
    [M], -1: none) names.  `base`: bf16 [M,N], the projection's result before its activation, or None for zero.
    `workspace`: a uint8 device tensor of lora_workspace_size(lora, M) bytes, or of a larger batch's; allocated here if None."""
    xdt = X.dtype
    if xdt is not _F32 and xdt is not _BF16:
        raise ValueError("X must be float32 or bfloat16")
    M, K, N = X.shape[0], lora.K, lora.N
    n_out = N // 2 if act == ACT_SILU_MUL else N
    xp, ldx = _rows(X, xdt, M, K, "X")
    ap = _vector(adapter, _I32, M, "adapter", "[M]")
    bp, ldb = (None, N) if base is None else _rows(base, _BF16, M, N, "base")
    if out is None:
        out = torch.empty((M, n_out), dtype=_BF16, device=X.device)
    yp, ldy = _rows(out, _BF16, M, n_out, "out")
    if workspace is None:
        workspace = torch.empty(lora_workspace_size(lora, M), dtype=torch.uint8, device=X.device)
    wp, wb = _ws(workspace)
    _check("w2_lora_add", _lib.w2_lora_add(lora._ref, K, N, xp, DT_F32 if xdt is _F32 else DT_BF16, ldx, M, ap, bp, ldb, yp, ldy,
                                           act, wp, wb, _stream()))
    return out


ROPE_NONE, ROPE_LINEAR, ROPE_NTK, ROPE_BANDS = 0, 1, 2, 3


class _RopeStruct(ctypes.Structure):
    _fields_ = [("phase", _vp), ("rotary_dim", _int), ("interleaved", _int), ("mscale", ctypes.c_float)]


def rope_phases(rotary_dim, base=10000.0, scaling=None):
    """The frequencies of the rotated pairs as 64-bit fractions of a turn per position: int64 [rotary_dim/2] on the host.

    scaling: None, ("linear", factor), ("ntk", factor) or ("bands", factor, original_len, low, high)."""
    kind, args = ROPE_NONE, ()
    if scaling is not None:
        kinds = {"linear": (ROPE_LINEAR, 1), "ntk": (ROPE_NTK, 1), "bands": (ROPE_BANDS, 4)}
        if scaling[0] not in kinds or len(scaling) - 1 != kinds[scaling[0]][1]:
            raise ValueError("scaling must be ('linear', factor), ('ntk', factor) or ('bands', factor, original_len, low, high)")
        kind, args = kinds[scaling[0]][0], scaling[1:]
    factor, original_len, low, high = (tuple(float(a) for a in args) + (1.0, 0.0, 0.0, 0.0)[len(args):])
    phase = torch.empty(max(1, rotary_dim // 2), dtype=torch.int64)
    _check("w2_rope_phases", _lib.w2_rope_phases(base, rotary_dim, kind, factor, original_len, low, high, _ptr(phase)))
    return phase


class Rope:
    """Rotary positions (w2_rope_t): the frequencies on the device and how a head's numbers pair up."""

    def __init__(self, rotary_dim, base=10000.0, interleaved=False, scaling=None, mscale=1.0, device="cuda"):
        self.rotary_dim, self.interleaved, self.mscale = rotary_dim, bool(interleaved), float(mscale)
        self.phase = rope_phases(rotary_dim, base, scaling).to(device)
        self._c = _RopeStruct(_ptr(self.phase), rotary_dim, int(self.interleaved), self.mscale)
        self._ref = ctypes.byref(self._c)


class _CacheStruct(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("n_pages", _i64), ("page_size", _i64),
                ("k_page_stride", _i64), ("k_slot_stride", _i64), ("k_head_stride", _i64),
                ("v_page_stride", _i64), ("v_slot_stride", _i64), ("v_head_stride", _i64),
                ("n_heads", _int), ("head_dim", _int)]


class KVCache:
    """A paged cache (w2_kv_cache_t): k and v bf16 [pages, page_size, heads, head_dim], any strides with a unit inner one
    (a cache stored [pages, heads, page_size, head_dim] is passed transposed)."""

    def __init__(self, k, v):
        _dev(k, torch.bfloat16, "k")
        _dev(v, torch.bfloat16, "v")
        if k.dim() != 4 or k.shape != v.shape or k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("k and v must be [pages, page_size, heads, head_dim] with unit inner stride")
        self.k, self.v = k, v
        self.n_pages, self.page_size, self.n_heads, self.head_dim = k.shape
        self._c = _CacheStruct(_ptr(k), _ptr(v), k.shape[0], k.shape[1], *k.stride()[:3], *v.stride()[:3], k.shape[2], k.shape[3])
        self._ref = ctypes.byref(self._c)


def qk_norm_rope(x, n_q, rope, positions, cache, slots=None, q_weight=None, k_weight=None, eps=1e-6, out=None):
    """Norm and rotation of the heads of x (bf16 [M, (n_q + 2 * cache.n_heads) * head_dim], a fused QKV projection's rows):
    returns the queries, bf16 [M, n_q, head_dim]; keys and values go to the cache's `slots` (int64 [M], page * page_size +
    place; -1: not written; None: row m to slot m).  rope None: no rotation; a weight None: not normed."""
    D, M = cache.head_dim, x.shape[0]
    xp, ldx = _rows(x, _BF16, M, (n_q + 2 * cache.n_heads) * D, "x")
    pp = None if positions is None else _vector(positions, _I32, M, "positions", "[M]")
    sp = None if slots is None else _vector(slots, _I64, M, "slots", "[M]")
    qw = None if q_weight is None else _vector(q_weight, _BF16, D, "q_weight", "[head_dim]")
    kw = None if k_weight is None else _vector(k_weight, _BF16, D, "k_weight", "[head_dim]")
    if out is None:
        out = torch.empty((M, n_q, D), dtype=_BF16, device=x.device)
    qp, ldq = _heads(out, M, n_q, D, "out")
    _check("w2_qk_norm_rope", _lib.w2_qk_norm_rope(xp, ldx, M, n_q, qw, kw, eps, None if rope is None else rope._ref, pp, qp, ldq,
                                                   cache._ref, sp, _stream()))
    return out


def tree_attention_workspace_size(n_requests, M, n_q, cache, max_rows, max_len, total_len=0):
    out = _sz(0)
    _check("w2_tree_attention_workspace_size", _lib.w2_tree_attention_workspace_size(
        n_requests, M, n_q, cache.n_heads, cache.head_dim, max_rows, max_len, total_len, ctypes.byref(out)))
    return out.value


def tree_attention(q, cache, page_table, row_start, kv_len, max_rows, max_len, mask=None, scale=None, total_len=0, out=None,
                   lse=None, workspace=None):
    """Attention of the rows q (bf16 [M, n_q, head_dim]) of every request over its keys in the cache: out like q.

    page_table int32 [requests, pages], row_start int32 [requests + 1], kv_len int32 [requests]; mask int64 [M, words], bit
    j: the row sees its request's drafted token j (None: causal); scale None: 1/sqrt(head_dim).  lse: fp32 [M, n_q], written
    if given.  Rows that no request owns are not written.  `workspace`: a uint8 device tensor of tree_attention_workspace_size
    bytes; None: the keys of a request are not shared out over workgroups."""
    M, n_q, D = q.shape
    if D != cache.head_dim:
        raise ValueError("q must be [M, n_q, head_dim] of the cache's head_dim")
    qp, ldq = _heads(q, M, n_q, D, "q")
    R = kv_len.shape[0]
    if page_table.dim() != 2:
        raise ValueError("page_table must be [requests, pages]")
    cols = page_table.shape[1]
    tp, ldt = _rows(page_table, _I32, R, cols, "page_table")
    rp = _vector(row_start, _I32, R + 1, "row_start", "[requests + 1]")
    lp = _vector(kv_len, _I32, R, "kv_len", "[requests]")
    words, mp = 0, None
    if mask is not None:
        if mask.dtype is not _I64 or mask.dim() != 2 or mask.shape[0] != M or not mask.is_contiguous() or not mask.is_cuda:
            raise ValueError("mask must be a contiguous device tensor [M, words] of int64")
        words, mp = mask.shape[1], mask.data_ptr()
    if out is None:
        out = torch.empty((M, n_q, D), dtype=_BF16, device=q.device)
    op, ldo = _heads(out, M, n_q, D, "out")
    ep = None
    if lse is not None:
        if lse.dtype is not _F32 or lse.shape != (M, n_q) or not lse.is_contiguous() or not lse.is_cuda:
            raise ValueError("lse must be a contiguous device tensor [M, n_q] of float32")
        ep = lse.data_ptr()
    wp, wb = _ws(workspace)
    _check("w2_tree_attention", _lib.w2_tree_attention(
        qp, ldq, M, n_q, cache._ref, tp, cols, ldt, rp, lp, R, max_rows, max_len, total_len, mp, words,
        D ** -0.5 if scale is None else scale, op, ldo, ep, wp, wb, _stream()))
    return out


def debug_group_acc_a8(packed, K, N, G, xq, variant=VARIANT_AUTO, tune=None):
    _dev(xq, torch.int8, "xq")
    M = xq.shape[0]
    acc = torch.empty((M, K // G, N), dtype=torch.int32, device=xq.device)
    t = _tune(variant, tune)
    _check("w2_debug_group_acc_a8", _lib.w2_debug_group_acc_a8(_ptr(packed), K, N, G, _ptr(xq), M,
                                                               _tp(t), _ptr(acc), _stream()))
    return acc


def debug_unpack(packed, K, N, G, codec=CODEC_INT2):
    codes = torch.empty((K, N), dtype=torch.uint8, device=packed.device)
    scales = torch.empty((K // G, N), dtype=torch.int16, device=packed.device)
    _check("w2_debug_unpack", _lib.w2_debug_unpack(_ptr(packed), K, N, G, codec, _ptr(codes),
                                                   _ptr(scales), _stream()))
    return codes, scales


def debug_int8_gemv(W8, xq, out=None):
    """Comparator: out int32 [N] = W8 int8 [N,K] @ xq int8 [K], exact."""
    _dev(W8, torch.int8, "W8")
    _dev(xq, torch.int8, "xq")
    N, K = W8.shape
    if not W8.is_contiguous() or xq.numel() != K:
        raise ValueError("W8 must be contiguous [N,K] and xq [K]")
    if out is None:
        out = torch.empty(N, dtype=torch.int32, device=W8.device)
    _check("w2_debug_int8_gemv", _lib.w2_debug_int8_gemv(_ptr(W8), K, N, _ptr(xq), _ptr(out), _stream()))
    return out


def debug_stream_read(buf, sink=None, tune=None):
    if sink is None:
        sink = torch.zeros(1, dtype=torch.int32, device=buf.device)
    t = _tune(VARIANT_AUTO, tune)
    _check("w2_debug_stream_read", _lib.w2_debug_stream_read(_ptr(buf), buf.numel() * buf.element_size(),
                                                             _ptr(sink), _tp(t), _stream()))
    return sink
