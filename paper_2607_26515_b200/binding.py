"""Thin ctypes binding of the C ABI in include/resq.h (argument marshalling only).

PyTorch supplies device memory (`tensor.data_ptr()`) and the stream; every step of the path
runs in the CUDA library.  There is no CPU fallback: if the library is missing or a call fails,
this module raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libresq.so")

S_NONE, S_DENSE, S_2_4, S_ROW50, S_CHAN50, S_BLOCK = 0, 1, 2, 3, 4, 5
OUT_BF16, OUT_F32 = 0, 1
PATTERN_NAMES = {S_NONE: "none", S_DENSE: "dense", S_2_4: "2:4", S_ROW50: "row50", S_CHAN50: "chan50",
                 S_BLOCK: "block32x64"}
STATUS_NAMES = {0: "OK", 1: "ERR_NULL", 2: "ERR_SHAPE", 3: "ERR_ALIGN", 4: "ERR_WORKSPACE", 5: "ERR_PATTERN",
                6: "ERR_CUDA", 7: "ERR_TIMEOUT"}

# every symbol include/resq.h declares: (name, restype, argtypes)
_i64, _vp, _ci, _sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
_cf = ctypes.c_float
SYMBOLS = {
    "hif4_codes_bytes": (_sz, [_i64, _i64]),
    "hif4_meta_bytes": (_sz, [_i64, _i64]),
    "mxfp4_codes_bytes": (_sz, [_i64, _i64]),
    "mxfp4_scale_bytes": (_sz, [_i64, _i64]),
    "resq_mask_bytes": (_sz, [_i64, _i64]),
    "resq_residual_mask_workspace_bytes": (_sz, [_i64, _i64, _ci]),
    "hif4_resq_workspace_bytes": (_sz, [_i64, _i64, _i64, _ci]),
    "mxfp4_resq_workspace_bytes": (_sz, [_i64, _i64, _i64, _ci]),
    "hif4_pack_weight": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "mxfp4_pack_weight": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "hif4_quantize_act": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "mxfp4_quantize_act": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "hif4_dequantize": (_ci, [_vp, _vp, _i64, _i64, _vp, _vp]),
    "mxfp4_dequantize": (_ci, [_vp, _vp, _i64, _i64, _vp, _vp]),
    "resq_residual_mask": (_ci, [_vp, _i64, _i64, _i64, _ci, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "mxfp4_residual_mask": (_ci, [_vp, _i64, _i64, _i64, _ci, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "resq_residual_mask_static": (_ci, [_vp, _i64, _i64, _i64, _ci, _vp, _vp, _vp, _vp, _vp, _vp]),
    "hif4_resq_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_resq_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_resq_group_workspace_bytes": (_sz, [_vp, _ci, _ci]),
    "mxfp4_resq_group_workspace_bytes": (_sz, [_vp, _ci, _ci]),
    "hif4_resq_linear_group": (_ci, [_vp, _ci, _ci, _ci, _vp, _sz, _vp]),
    "mxfp4_resq_linear_group": (_ci, [_vp, _ci, _ci, _ci, _vp, _sz, _vp]),
    "resq_transposed_workspace_bytes": (_sz, [_i64, _i64]),
    "hif4_pack_weight_transposed": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _sz, _vp]),
    "mxfp4_pack_weight_transposed": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _sz, _vp]),
    "hif4_dgrad_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "mxfp4_dgrad_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "hif4_dgrad_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_dgrad_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_wgrad_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "mxfp4_wgrad_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "hif4_wgrad_linear": (_ci, [_vp, _vp, _i64, _i64, _i64, _i64, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_wgrad_linear": (_ci, [_vp, _vp, _i64, _i64, _i64, _i64, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "resq_w4a16_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "resq_w4a8_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "hif4_w4a8_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_w4a8_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_w4a16_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_w4a16_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_swiglu_resq_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_swiglu_resq_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_rmsnorm_resq_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, ctypes.c_float, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_rmsnorm_resq_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, ctypes.c_float, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_rht_pack_weight": (_ci, [_vp, _i64, _i64, _i64, ctypes.c_ulonglong, _vp, _vp, _vp]),
    "mxfp4_rht_pack_weight": (_ci, [_vp, _i64, _i64, _i64, ctypes.c_ulonglong, _vp, _vp, _vp]),
    "hif4_rht_resq_linear": (_ci, [_vp, _i64, _i64, _i64, ctypes.c_ulonglong, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_rht_resq_linear": (_ci, [_vp, _i64, _i64, _i64, ctypes.c_ulonglong, _vp, _vp, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_w16a4_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _i64, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "mxfp4_w16a4_linear": (_ci, [_vp, _i64, _i64, _i64, _vp, _i64, _i64, _ci, _vp, _ci, _i64, _vp, _sz, _vp]),
    "hif4_w4a16_gemv": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp]),
    "mxfp4_w4a16_gemv": (_ci, [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _ci, _i64, _vp]),
    "resq_block_join": (_ci, [_vp, _ci, _vp, _i64, _i64, _i64, _i64, _vp, _i64, _ci, _vp, _vp, _cf, _cf, _vp, _i64, _vp, _i64, _vp]),
    "resq_block_join_backward_workspace_bytes": (_sz, [_i64, _i64]),
    "resq_block_join_backward": (_ci, [_vp, _vp, _vp, _ci, _vp, _i64, _i64, _i64, _i64, _i64, _i64, _vp, _i64, _ci, _vp, _vp, _cf, _cf,
                                       _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _sz, _vp]),
    "resq_token_logprobs": (_ci, [_vp, _ci, _i64, _i64, _i64, _vp, _cf, _ci, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "resq_token_logprobs_backward": (_ci, [_vp, _ci, _i64, _i64, _i64, _vp, _cf, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp]),
    "resq_rope_append": (_ci, [_vp, _ci, _i64, _i64, _i64, _i64, _i64, _vp, _vp, _i64, _ci, _vp, _vp, _vp, _vp, _i64, _vp]),
    "resq_paged_attention_workspace_bytes": (_sz, [_i64, _i64, _i64, _i64, _i64, _i64]),
    "resq_paged_attention": (_ci, [_vp, _i64, _i64, _i64, _i64, _i64, _vp, _vp, _i64, _cf, _vp, _i64, _vp, _vp, _sz, _vp]),
    "resq_verify_drafts_workspace_bytes": (_sz, [_i64]),
    "resq_verify_drafts": (_ci, [_vp, _ci, _i64, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _cf, _vp, _vp, _vp, _vp,
                                 _sz, _vp]),
    "resq_check": (_ci, [_vp, _vp]),
    "resq_last_error": (ctypes.c_char_p, []),
    "resq_kernel_launches": (_i64, []),
    "resq_debug_expire_next_wait": (_ci, [_ci]),
    "resq_profile_enable": (_ci, [_ci]),
    "resq_profile_read": (_ci, [_vp, _vp]),
}

_lib: Optional[ctypes.CDLL] = None


class ResqError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"resq: {STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_26515_b200.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SYMBOLS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def last_error() -> str:
    return lib().resq_last_error().decode()


def _check(status: int) -> None:
    if status != 0:
        raise ResqError(status, last_error())


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _side(fmt: str, rows: int, K: int, device) -> torch.Tensor:
    if fmt == "hif4":
        return torch.empty((rows, K // 64), dtype=torch.int32, device=device)
    return torch.empty((rows, K // 32), dtype=torch.uint8, device=device)


def _fn(fmt: str, hif4_name: str, mx_name: str):
    if fmt not in ("hif4", "mxfp4"):
        raise ValueError(f"unknown format {fmt!r}")
    return getattr(lib(), hif4_name if fmt == "hif4" else mx_name)


def _require_bf16_matrix(x: torch.Tensor, name: str) -> None:
    if x.dtype != torch.bfloat16 or x.dim() != 2 or not x.is_cuda or x.stride(1) != 1:
        raise ValueError(f"{name} must be a 2-D CUDA bf16 tensor with unit inner stride")


# ------------------------------------------------------------------ size queries

def residual_mask_workspace_bytes(M: int, K: int, pattern: int) -> int:
    return int(lib().resq_residual_mask_workspace_bytes(M, K, pattern))


def resq_workspace_bytes(M: int, N: int, K: int, pattern: int, fmt: str = "hif4") -> int:
    return int(_fn(fmt, "hif4_resq_workspace_bytes", "mxfp4_resq_workspace_bytes")(M, N, K, pattern))


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ------------------------------------------------------------------ calls

def keep_quarters(pattern: int, q: int) -> int:
    """RESQ_KEEP_QUARTERS: the pattern with q/4 of the entries kept instead of one half (q = 1, 2, 3)."""
    return pattern | (q << 8)


def per_strip(pattern: int) -> int:
    """RESQ_BLOCK_PER_STRIP: the 32x64 block pattern with the selection taken inside every strip of 32 token rows."""
    return pattern | (1 << 12)


def pack_weight(W: torch.Tensor, fmt: str = "hif4", stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """*_pack_weight: W bf16 [N,K] -> (codes u8 [N,K/2], meta i32 [N,K/64] | scale u8 [N,K/32])."""
    _require_bf16_matrix(W, "W")
    N, K = W.shape
    codes = torch.empty((N, K // 2), dtype=torch.uint8, device=W.device)
    side = _side(fmt, N, K, W.device)
    _check(_fn(fmt, "hif4_pack_weight", "mxfp4_pack_weight")(W.data_ptr(), N, K, W.stride(0), codes.data_ptr(),
                                                              side.data_ptr(), _stream(stream)))
    return codes, side


def rht_pack_weight(W: torch.Tensor, signs: int, fmt: str = "hif4", stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """*_rht_pack_weight: rotate every block of 64 channels by the randomized Hadamard transform, then pack."""
    _require_bf16_matrix(W, "W")
    N, K = W.shape
    codes = torch.empty((N, K // 2), dtype=torch.uint8, device=W.device)
    side = _side(fmt, N, K, W.device)
    _check(_fn(fmt, "hif4_rht_pack_weight", "mxfp4_rht_pack_weight")(W.data_ptr(), N, K, W.stride(0), signs & (2 ** 64 - 1),
                                                                      codes.data_ptr(), side.data_ptr(), _stream(stream)))
    return codes, side


def rht_resq_linear(X: torch.Tensor, signs: int, w_codes: torch.Tensor, w_side: torch.Tensor, pattern: int = S_NONE,
                    fmt: str = "hif4", out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_rht_resq_linear: Eq. (5) on the rotated activations against weights packed by rht_pack_weight."""
    _require_bf16_matrix(X, "X")
    M, K = X.shape
    N = w_codes.shape[0]
    if Y is None:
        ld = (N + 7) // 8 * 8
        Y = torch.empty((M, ld), dtype=out_dtype, device=X.device)[:, :N]
    if Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    if workspace is None:
        workspace = alloc_workspace(resq_workspace_bytes(M, N, K, pattern, fmt), X.device)
    _check(_fn(fmt, "hif4_rht_resq_linear", "mxfp4_rht_resq_linear")(
        X.data_ptr(), M, K, X.stride(0), signs & (2 ** 64 - 1), w_codes.data_ptr(), w_side.data_ptr(), N, pattern,
        Y.data_ptr(), OUT_BF16 if Y.dtype == torch.bfloat16 else OUT_F32, Y.stride(0), workspace.data_ptr(),
        workspace.numel(), _stream(stream)))
    return Y


def quantize_act(X: torch.Tensor, fmt: str = "hif4", stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """*_quantize_act: X bf16 [M,K] -> (codes, meta | scale)."""
    _require_bf16_matrix(X, "X")
    M, K = X.shape
    codes = torch.empty((M, K // 2), dtype=torch.uint8, device=X.device)
    side = _side(fmt, M, K, X.device)
    _check(_fn(fmt, "hif4_quantize_act", "mxfp4_quantize_act")(X.data_ptr(), M, K, X.stride(0), codes.data_ptr(),
                                                                side.data_ptr(), _stream(stream)))
    return codes, side


def dequantize(codes: torch.Tensor, side: torch.Tensor, fmt: str = "hif4", stream=None) -> torch.Tensor:
    rows, K = codes.shape[0], codes.shape[1] * 2
    out = torch.empty((rows, K), dtype=torch.float32, device=codes.device)
    _check(_fn(fmt, "hif4_dequantize", "mxfp4_dequantize")(codes.data_ptr(), side.data_ptr(), rows, K, out.data_ptr(),
                                                            _stream(stream)))
    return out


def residual_mask(X: torch.Tensor, pattern: int, fmt: str = "hif4", workspace: Optional[torch.Tensor] = None,
                  stream=None):
    """resq_residual_mask / mxfp4_residual_mask -> dict(x_codes, x_side, r_codes, r_side, mask)."""
    _require_bf16_matrix(X, "X")
    M, K = X.shape
    dev = X.device
    out = {"x_codes": torch.empty((M, K // 2), dtype=torch.uint8, device=dev), "x_side": _side(fmt, M, K, dev),
           "r_codes": None, "r_side": None, "mask": None}
    if pattern != S_NONE:
        out["r_codes"] = torch.empty((M, K // 2), dtype=torch.uint8, device=dev)
        out["r_side"] = _side(fmt, M, K, dev)
        out["mask"] = torch.empty((M, K // 8), dtype=torch.uint8, device=dev)
    if workspace is None:
        workspace = alloc_workspace(residual_mask_workspace_bytes(M, K, pattern), dev)
    _check(_fn(fmt, "resq_residual_mask", "mxfp4_residual_mask")(
        X.data_ptr(), M, K, X.stride(0), pattern, _ptr(out["x_codes"]), _ptr(out["x_side"]), _ptr(out["r_codes"]),
        _ptr(out["r_side"]), _ptr(out["mask"]), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return out


STATIC_SCRATCH_MAX_SCORES = 32768


def residual_mask_static(X: torch.Tensor, pattern: int, stream=None):
    """resq_residual_mask_static: the HiF4 residual / mask pass without a caller workspace, for callers that
    cannot allocate device memory; its selection scratch is a fixed array inside the library (at most
    STATIC_SCRATCH_MAX_SCORES channel or block scores).  Calls that overlap on the GPU race on that array."""
    _require_bf16_matrix(X, "X")
    M, K = X.shape
    dev = X.device
    out = {"x_codes": torch.empty((M, K // 2), dtype=torch.uint8, device=dev), "x_side": _side("hif4", M, K, dev),
           "r_codes": None, "r_side": None, "mask": None}
    if pattern != S_NONE:
        out["r_codes"] = torch.empty((M, K // 2), dtype=torch.uint8, device=dev)
        out["r_side"] = _side("hif4", M, K, dev)
        out["mask"] = torch.empty((M, K // 8), dtype=torch.uint8, device=dev)
    _check(lib().resq_residual_mask_static(
        X.data_ptr(), M, K, X.stride(0), pattern, _ptr(out["x_codes"]), _ptr(out["x_side"]), _ptr(out["r_codes"]),
        _ptr(out["r_side"]), _ptr(out["mask"]), _stream(stream)))
    return out


def resq_linear(X: torch.Tensor, w_codes: torch.Tensor, w_side: torch.Tensor, pattern: int, fmt: str = "hif4",
                out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_resq_linear: Y = Q(X) Q(W)^T + S(Q(X - deq Q(X))) Q(W)^T  (Eq. (5))."""
    _require_bf16_matrix(X, "X")
    M, K = X.shape
    N = w_codes.shape[0]
    if Y is None:
        ld = (N + 7) // 8 * 8  # rows of Y start on 16-byte boundaries
        Y = torch.empty((M, ld), dtype=out_dtype, device=X.device)[:, :N]
    if Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    if workspace is None:
        workspace = alloc_workspace(resq_workspace_bytes(M, N, K, pattern, fmt), X.device)
    _check(_fn(fmt, "hif4_resq_linear", "mxfp4_resq_linear")(
        X.data_ptr(), M, K, X.stride(0), w_codes.data_ptr(), w_side.data_ptr(), N, pattern, Y.data_ptr(),
        OUT_BF16 if Y.dtype == torch.bfloat16 else OUT_F32, Y.stride(0), workspace.data_ptr(), workspace.numel(),
        _stream(stream)))
    return Y


class _Problem(ctypes.Structure):
    """struct resq_problem of include/resq.h."""
    _fields_ = [("X_bf16", _vp), ("M", _i64), ("K", _i64), ("ldx", _i64), ("w_codes", _vp), ("w_side", _vp), ("N", _i64),
                ("Y", _vp), ("ldy", _i64)]


MAX_GROUP = 8


def _problem_array(problems, out_dtype):
    """problems: sequence of (X, w_codes, w_side) or (X, w_codes, w_side, Y) -> (ctypes array, list of Y)."""
    arr = (_Problem * len(problems))()
    ys = []
    for i, pr in enumerate(problems):
        X, wc, ws = pr[0], pr[1], pr[2]
        _require_bf16_matrix(X, "X")
        M, K = X.shape
        N = wc.shape[0]
        Y = pr[3] if len(pr) > 3 and pr[3] is not None else torch.empty((M, (N + 7) // 8 * 8), dtype=out_dtype, device=X.device)[:, :N]
        if Y.dtype != out_dtype:
            raise ValueError("every Y of a group has the group's output type")
        ys.append(Y)
        arr[i] = _Problem(X.data_ptr(), M, K, X.stride(0), wc.data_ptr(), ws.data_ptr(), N, Y.data_ptr(), Y.stride(0))
    return arr, ys


def resq_group_workspace_bytes(problems, pattern: int, fmt: str = "hif4", out_dtype: torch.dtype = torch.bfloat16) -> int:
    arr, _ = _problem_array(problems, out_dtype)
    return int(_fn(fmt, "hif4_resq_group_workspace_bytes", "mxfp4_resq_group_workspace_bytes")(
        ctypes.cast(arr, _vp), len(problems), pattern))


def resq_linear_group(problems, pattern: int, fmt: str = "hif4", out_dtype: torch.dtype = torch.bfloat16,
                      workspace: Optional[torch.Tensor] = None, stream=None):
    """*_resq_linear_group: up to MAX_GROUP independent projections of Eq. (5) in one quantizer launch and one GEMM
    launch.  problems: sequence of (X, w_codes, w_side[, Y]); returns the list of outputs."""
    if out_dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    arr, ys = _problem_array(problems, out_dtype)
    fn_b = _fn(fmt, "hif4_resq_group_workspace_bytes", "mxfp4_resq_group_workspace_bytes")
    if workspace is None:
        workspace = alloc_workspace(int(fn_b(ctypes.cast(arr, _vp), len(problems), pattern)), problems[0][0].device)
    _check(_fn(fmt, "hif4_resq_linear_group", "mxfp4_resq_linear_group")(
        ctypes.cast(arr, _vp), len(problems), pattern, OUT_BF16 if out_dtype == torch.bfloat16 else OUT_F32,
        workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return ys


def _out(rows: int, cols: int, dtype: torch.dtype, device) -> torch.Tensor:
    """An output matrix whose rows start on 16-byte boundaries."""
    return torch.empty((rows, (cols + 7) // 8 * 8), dtype=dtype, device=device)[:, :cols]


def pack_weight_transposed(W: torch.Tensor, fmt: str = "hif4", stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """*_pack_weight_transposed: W bf16 [N,K] -> Q(W^T) as (codes [K,N/2], meta [K,N/64] | scale [K,N/32]), for dgrad."""
    _require_bf16_matrix(W, "W")
    N, K = W.shape
    codes = torch.empty((K, N // 2), dtype=torch.uint8, device=W.device)
    side = _side(fmt, K, N, W.device)
    work = alloc_workspace(int(lib().resq_transposed_workspace_bytes(N, K)), W.device)
    _check(_fn(fmt, "hif4_pack_weight_transposed", "mxfp4_pack_weight_transposed")(
        W.data_ptr(), N, K, W.stride(0), codes.data_ptr(), side.data_ptr(), work.data_ptr(), work.numel(), _stream(stream)))
    return codes, side


def dgrad_linear(dY: torch.Tensor, wt_codes: torch.Tensor, wt_side: torch.Tensor, fmt: str = "hif4",
                 out_dtype: torch.dtype = torch.bfloat16, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_dgrad_linear: dX^ [M,K] = Q(dY) Q(W^T)^T with the transposed pack of the weight."""
    _require_bf16_matrix(dY, "dY")
    M, N = dY.shape
    K = wt_codes.shape[0]
    dX = _out(M, K, out_dtype, dY.device)
    if workspace is None:
        workspace = alloc_workspace(int(_fn(fmt, "hif4_dgrad_workspace_bytes", "mxfp4_dgrad_workspace_bytes")(M, N, K)), dY.device)
    _check(_fn(fmt, "hif4_dgrad_linear", "mxfp4_dgrad_linear")(
        dY.data_ptr(), M, N, dY.stride(0), wt_codes.data_ptr(), wt_side.data_ptr(), K, dX.data_ptr(),
        OUT_BF16 if out_dtype == torch.bfloat16 else OUT_F32, dX.stride(0), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return dX


def wgrad_linear(dY: torch.Tensor, X: torch.Tensor, fmt: str = "hif4", out_dtype: torch.dtype = torch.bfloat16,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_wgrad_linear: dW^ [N,K] = Q(dY^T) Q(X^T)^T."""
    _require_bf16_matrix(dY, "dY")
    _require_bf16_matrix(X, "X")
    M, N = dY.shape
    K = X.shape[1]
    if X.shape[0] != M:
        raise ValueError("dY and X must have the same number of token rows")
    dW = _out(N, K, out_dtype, dY.device)
    if workspace is None:
        workspace = alloc_workspace(int(_fn(fmt, "hif4_wgrad_workspace_bytes", "mxfp4_wgrad_workspace_bytes")(M, N, K)), dY.device)
    _check(_fn(fmt, "hif4_wgrad_linear", "mxfp4_wgrad_linear")(
        dY.data_ptr(), X.data_ptr(), M, N, K, dY.stride(0), X.stride(0), dW.data_ptr(),
        OUT_BF16 if out_dtype == torch.bfloat16 else OUT_F32, dW.stride(0), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return dW


def w4a16_linear(X: torch.Tensor, w_codes: torch.Tensor, w_side: torch.Tensor, fmt: str = "hif4",
                 out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_w4a16_linear: Y = X deq(Q(W))^T, activations kept in bf16 (Table 1, W4A16).  Its tile computes 128 rows whatever M is:
    up to GEMV_MAX_TOKENS rows w4a16_gemv takes a third to a half of its time (3584 -> 37888: 8 rows 25 against 70 us,
    16 rows 33)."""
    _require_bf16_matrix(X, "X")
    M, K = X.shape
    N = w_codes.shape[0]
    if Y is None:
        ld = (N + 7) // 8 * 8
        Y = torch.empty((M, ld), dtype=out_dtype, device=X.device)[:, :N]
    if Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    if workspace is None:
        workspace = alloc_workspace(int(lib().resq_w4a16_workspace_bytes(M, N, K)), X.device)
    _check(_fn(fmt, "hif4_w4a16_linear", "mxfp4_w4a16_linear")(
        X.data_ptr(), M, K, X.stride(0), w_codes.data_ptr(), w_side.data_ptr(), N, Y.data_ptr(),
        OUT_BF16 if Y.dtype == torch.bfloat16 else OUT_F32, Y.stride(0), workspace.data_ptr(), workspace.numel(),
        _stream(stream)))
    return Y


def swiglu_resq_linear(GU: torch.Tensor, w_codes: torch.Tensor, w_side: torch.Tensor, pattern: int, fmt: str = "hif4",
                       out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_swiglu_resq_linear: Eq. (5) on X = bf16(SiLU(gate) * up) with GU = [gate | up], X never stored."""
    _require_bf16_matrix(GU, "GU")
    M, K2 = GU.shape
    K = K2 // 2
    N = w_codes.shape[0]
    if K2 % 2 or w_codes.shape[1] * 2 != K:
        raise ValueError("GU must be [M, 2K] for weights packed as [N, K/2]")
    if Y is None:
        ld = (N + 7) // 8 * 8
        Y = torch.empty((M, ld), dtype=out_dtype, device=GU.device)[:, :N]
    if Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    if workspace is None:
        workspace = alloc_workspace(resq_workspace_bytes(M, N, K, pattern, fmt), GU.device)
    _check(_fn(fmt, "hif4_swiglu_resq_linear", "mxfp4_swiglu_resq_linear")(
        GU.data_ptr(), M, K, GU.stride(0), w_codes.data_ptr(), w_side.data_ptr(), N, pattern, Y.data_ptr(),
        OUT_BF16 if Y.dtype == torch.bfloat16 else OUT_F32, Y.stride(0), workspace.data_ptr(), workspace.numel(),
        _stream(stream)))
    return Y


def rmsnorm_resq_linear(H: torch.Tensor, gamma: torch.Tensor, eps: float, w_codes: torch.Tensor, w_side: torch.Tensor,
                        pattern: int, fmt: str = "hif4", out_dtype: torch.dtype = torch.bfloat16,
                        Y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_rmsnorm_resq_linear: Eq. (5) on X = bf16(RMSNorm(H) * gamma), X never stored."""
    _require_bf16_matrix(H, "H")
    M, K = H.shape
    N = w_codes.shape[0]
    if gamma.dtype != torch.bfloat16 or gamma.numel() != K or not gamma.is_contiguous():
        raise ValueError("gamma must be a contiguous bf16 vector of K elements")
    if Y is None:
        ld = (N + 7) // 8 * 8
        Y = torch.empty((M, ld), dtype=out_dtype, device=H.device)[:, :N]
    if Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    if workspace is None:
        workspace = alloc_workspace(resq_workspace_bytes(M, N, K, pattern, fmt), H.device)
    _check(_fn(fmt, "hif4_rmsnorm_resq_linear", "mxfp4_rmsnorm_resq_linear")(
        H.data_ptr(), M, K, H.stride(0), gamma.data_ptr(), float(eps), w_codes.data_ptr(), w_side.data_ptr(), N, pattern,
        Y.data_ptr(), OUT_BF16 if Y.dtype == torch.bfloat16 else OUT_F32, Y.stride(0), workspace.data_ptr(),
        workspace.numel(), _stream(stream)))
    return Y


def w4a8_linear(X: torch.Tensor, w_codes: torch.Tensor, w_side: torch.Tensor, fmt: str = "hif4",
                out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_w4a8_linear: Y = deq(MXFP8-E4M3(X)) deq(Q(W))^T (Table 1, W4A8; the 8-bit format is this library's reading)."""
    _require_bf16_matrix(X, "X")
    M, K = X.shape
    N = w_codes.shape[0]
    if Y is None:
        ld = (N + 7) // 8 * 8
        Y = torch.empty((M, ld), dtype=out_dtype, device=X.device)[:, :N]
    if Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    if workspace is None:
        workspace = alloc_workspace(int(lib().resq_w4a8_workspace_bytes(M, N, K)), X.device)
    _check(_fn(fmt, "hif4_w4a8_linear", "mxfp4_w4a8_linear")(
        X.data_ptr(), M, K, X.stride(0), w_codes.data_ptr(), w_side.data_ptr(), N, Y.data_ptr(),
        OUT_BF16 if Y.dtype == torch.bfloat16 else OUT_F32, Y.stride(0), workspace.data_ptr(), workspace.numel(),
        _stream(stream)))
    return Y


def w16a4_linear(X: torch.Tensor, W: torch.Tensor, pattern: int = S_NONE, fmt: str = "hif4",
                 out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_w16a4_linear: Y = (deq Q(X) + S(deq Q(dX))) W^T with plain bf16 weights (Table 1, W16A4)."""
    _require_bf16_matrix(X, "X")
    _require_bf16_matrix(W, "W")
    M, K = X.shape
    N = W.shape[0]
    if W.shape[1] != K:
        raise ValueError("W must be [N, K]")
    if Y is None:
        ld = (N + 7) // 8 * 8
        Y = torch.empty((M, ld), dtype=out_dtype, device=X.device)[:, :N]
    if Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be bf16 or fp32")
    if workspace is None:
        workspace = alloc_workspace(resq_workspace_bytes(M, N, K, pattern, fmt), X.device)
    _check(_fn(fmt, "hif4_w16a4_linear", "mxfp4_w16a4_linear")(
        X.data_ptr(), M, K, X.stride(0), W.data_ptr(), N, W.stride(0), pattern, Y.data_ptr(),
        OUT_BF16 if Y.dtype == torch.bfloat16 else OUT_F32, Y.stride(0), workspace.data_ptr(), workspace.numel(),
        _stream(stream)))
    return Y


# ------------------------------------------------------------------ few-token product, residual stream, log-probabilities
#
# These calls run on the device of their first tensor (made current for the call) and on `stream` (default: that device's
# current stream).  What they allocate belongs to that stream.  At one token the call is host time: entering a device and a
# stream costs three times the launch, so that is done only where they are not the current ones already.

GEMV_MAX_TOKENS = 16
JOIN_MAX_K = 32768
MAX_TOP = 32
GATE_LINEAR, GATE_SIGMOID = 0, 1
_GATES = {"linear": GATE_LINEAR, "sigmoid": GATE_SIGMOID}
_OUT = {torch.bfloat16: OUT_BF16, torch.float32: OUT_F32}
_BF16, _F32 = torch.bfloat16, torch.float32
# the current stream's handle without a Stream object around it (0.1 instead of 3 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _elsewhere(index: int, stream, call):
    """call() with device `index` current and, if a stream is named, that stream current too: the allocator then ties what
    the call allocates to the stream its kernels run on."""
    if stream is not None and not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=index)
    if stream is not None and stream.device.index != index:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to cuda:{index}")
    with torch.cuda.device(index), torch.cuda.stream(stream):
        return call()


def _require(ok: bool, msg: str) -> None:
    if not ok:
        raise ValueError(msg)


def _first(t: torch.Tensor, name: str):
    """(M, K, row pitch in elements, type code, device index) of a call's first tensor: a matrix on a device with unit inner
    stride (a single row has no pitch of its own: any multiple of 8 that covers it will do)."""
    if t.dim() != 2 or not t.is_cuda or t.dtype not in _OUT:
        raise ValueError(f"{name} must be a 2-D CUDA tensor, bf16 or fp32")
    M, K = t.shape
    ld, inner = t.stride()
    if inner != 1 and K > 1:
        raise ValueError(f"{name} must have unit inner stride")
    return M, K, ld if M > 1 else (K + 7) // 8 * 8, _OUT[t.dtype], t.get_device()


def _rows(t: torch.Tensor, name: str, M: int, K: int, dtype, index: int) -> int:
    """Checks that t is an [M, K] matrix of one type on one device with unit inner stride; its row pitch as in _first."""
    if t.dtype is not dtype or t.shape != (M, K) or t.get_device() != index or (K > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a {dtype} tensor [{M}, {K}] on cuda:{index} with unit inner stride")
    return t.stride(0) if M > 1 else (K + 7) // 8 * 8


def _vector(t: torch.Tensor, name: str, n: int, dtype, index: int) -> int:
    """Checks that t is a contiguous vector of n elements on one device; its address."""
    if t.dtype is not dtype or t.shape != (n,) or t.get_device() != index or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {n} elements on cuda:{index}")
    return t.data_ptr()


def _new_rows(M: int, K: int, dtype, index: int) -> torch.Tensor:
    """A matrix whose rows start on 16-byte boundaries."""
    return torch.empty_strided((M, K), ((K + 7) // 8 * 8, 1), dtype=dtype, device=index)


def _new(M: int, K: int, dtype, index: int) -> torch.Tensor:
    """A contiguous matrix (0.8 us sooner than from torch.empty)."""
    return torch.empty_strided((M, K), (K, 1), dtype=dtype, device=index)


def _new_vector(n: int, dtype, index: int) -> torch.Tensor:
    return torch.empty_strided((n,), (1,), dtype=dtype, device=index)


def w4a16_gemv(X: torch.Tensor, w_codes: torch.Tensor, w_side: torch.Tensor, fmt: str = "hif4",
               out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """*_w4a16_gemv: Y = X deq(Q(W))^T for at most GEMV_MAX_TOKENS token rows, streaming the packed weights once."""
    fn = _fn(fmt, "hif4_w4a16_gemv", "mxfp4_w4a16_gemv")
    M, K, ldx, code, index = _first(X, "X")
    _require(code == OUT_BF16, "X must be bf16")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: w4a16_gemv(X, w_codes, w_side, fmt, out_dtype, Y))
    _require(w_codes.dim() == 2, "w_codes must be [N, K/2]")
    N = w_codes.shape[0]
    if w_codes.dtype is not torch.uint8 or w_codes.shape[1] * 2 != K or not w_codes.is_contiguous() or w_codes.get_device() != index:
        raise ValueError(f"w_codes must be contiguous uint8 [N, K/2] on cuda:{index} for the activations' K = {K}")
    block, side_type = (64, torch.int32) if fmt == "hif4" else (32, torch.uint8)
    if w_side.dtype is not side_type or w_side.shape != (N, K // block) or not w_side.is_contiguous() or w_side.get_device() != index:
        raise ValueError(f"w_meta / w_scale must be contiguous {side_type} [N, K/{block}] on cuda:{index}")
    out_dtype = out_dtype if Y is None else Y.dtype
    _require(out_dtype in _OUT, "Y must be bf16 or fp32")
    if Y is None:
        Y, ldy = _new_rows(M, N, out_dtype, index), (N + 7) // 8 * 8
    else:
        ldy = _rows(Y, "Y", M, N, out_dtype, index)
    _check(fn(X.data_ptr(), M, K, ldx, w_codes.data_ptr(), w_side.data_ptr(), N, Y.data_ptr(), _OUT[out_dtype], ldy, _raw_stream(index)))
    return Y


def _join_gate(gate, M: int, K: int, index: int):
    """(address, row pitch) of a gate; the pitch of a channel gate is 0."""
    if gate is None:
        return None, 0
    if gate.dim() == 1:
        return _vector(gate, "gate", K, _BF16, index), 0
    ldg = _rows(gate, "gate", M, K, _BF16, index)
    _require(ldg != 0, "a gate shared by all tokens is given as a vector of K elements")
    return gate.data_ptr(), ldg


def block_join(H: torch.Tensor, B: torch.Tensor, gamma_pre: Optional[torch.Tensor] = None, gamma_post: Optional[torch.Tensor] = None,
               gate: Optional[torch.Tensor] = None, act: str = "linear", alpha: float = 1.0, eps: float = 1e-6,
               H_out: Optional[torch.Tensor] = None, X: Optional[torch.Tensor] = None, stream=None):
    """resq_block_join: H' = H + alpha g(gate) norm(B), X = norm(H') -> (H', X).

    gamma_post None: the branch B is added as it is; gamma_pre None: X is None.  gate: None, [K] (one for all tokens) or
    [M, K]; act "linear" or "sigmoid".  H_out may be H."""
    M, K, ldh, code, index = _first(H, "H")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: block_join(H, B, gamma_pre, gamma_post, gate, act, alpha, eps, H_out, X))
    ldb = _rows(B, "B", M, K, _BF16, index)
    pre = None if gamma_pre is None else _vector(gamma_pre, "gamma_pre", K, _BF16, index)
    post = None if gamma_post is None else _vector(gamma_post, "gamma_post", K, _BF16, index)
    g, ldg = _join_gate(gate, M, K, index)
    _require(act in _GATES, f"unknown gate function {act!r}")
    _require(X is None or gamma_pre is not None, "X needs gamma_pre")

    ldho = ldx = (K + 7) // 8 * 8
    if H_out is None:
        H_out = _new_rows(M, K, H.dtype, index)
    else:
        ldho = _rows(H_out, "H_out", M, K, H.dtype, index)
    if X is not None:
        ldx = _rows(X, "X", M, K, _BF16, index)
    elif gamma_pre is not None:
        X = _new_rows(M, K, _BF16, index)
    _check(lib().resq_block_join(H.data_ptr(), code, B.data_ptr(), M, K, ldh, ldb, g, ldg, _GATES[act], post, pre, alpha, eps,
                                 H_out.data_ptr(), ldho, _ptr(X), ldx, _raw_stream(index)))
    return H_out, X


@functools.lru_cache(maxsize=1024)
def block_join_backward_workspace_bytes(M: int, K: int) -> int:
    return int(lib().resq_block_join_backward_workspace_bytes(M, K))


def block_join_backward(dH_out: Optional[torch.Tensor], dX: Optional[torch.Tensor], H_out: torch.Tensor, B: torch.Tensor,
                        gamma_pre: Optional[torch.Tensor] = None, gamma_post: Optional[torch.Tensor] = None,
                        gate: Optional[torch.Tensor] = None, act: str = "linear", alpha: float = 1.0, eps: float = 1e-6,
                        dH: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """resq_block_join_backward -> dict(dH, dB[, dgate][, dgamma_post][, dgamma_pre]) from the gradients of H' and X (either
    may be None) and the forward call's H' and inputs.  dgate has the gate's shape, fp32 for a channel gate [K], else bf16;
    the norms' gradients are fp32.  dH may be dH_out."""
    M, K, ldh, code, index = _first(H_out, "H_out")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: block_join_backward(dH_out, dX, H_out, B, gamma_pre, gamma_post, gate, act, alpha, eps, dH,
                                                                     workspace))
    ldb = _rows(B, "B", M, K, _BF16, index)
    _require(dH_out is not None or dX is not None, "one of dH_out and dX is needed")
    _require(dX is None or gamma_pre is not None, "dX needs gamma_pre")
    lddho = 0 if dH_out is None else _rows(dH_out, "dH_out", M, K, H_out.dtype, index)
    lddx = 0 if dX is None else _rows(dX, "dX", M, K, _BF16, index)
    pre = None if gamma_pre is None else _vector(gamma_pre, "gamma_pre", K, _BF16, index)
    post = None if gamma_post is None else _vector(gamma_post, "gamma_post", K, _BF16, index)
    g, ldg = _join_gate(gate, M, K, index)
    _require(act in _GATES, f"unknown gate function {act!r}")
    if workspace is not None and (workspace.get_device() != index or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{index}")
    lddh = ldn = (K + 7) // 8 * 8
    if dH is not None:
        lddh = _rows(dH, "dH", M, K, H_out.dtype, index)

    out = {"dH": _new_rows(M, K, H_out.dtype, index) if dH is None else dH, "dB": _new_rows(M, K, _BF16, index)}
    columns = [n for n, on in (("dgamma_pre", dX is not None), ("dgamma_post", post is not None), ("dgate", g is not None and ldg == 0)) if on]
    if columns:
        out.update(zip(columns, _new(len(columns), K, _F32, index).unbind()))
    if ldg:
        out["dgate"] = _new_rows(M, K, _BF16, index)
    if workspace is None:
        workspace = _new(1, max(block_join_backward_workspace_bytes(M, K), 256), torch.uint8, index)
    _check(lib().resq_block_join_backward(
        _ptr(dH_out), _ptr(dX), H_out.data_ptr(), code, B.data_ptr(), M, K, lddho, lddx, ldh, ldb, g, ldg, _GATES[act], post, pre,
        alpha, eps, out["dH"].data_ptr(), lddh, out["dB"].data_ptr(), ldn, _ptr(out.get("dgate")), ldn if ldg else 0,
        _ptr(out.get("dgamma_post")), _ptr(out.get("dgamma_pre")), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _raw_stream(index)))
    return out


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, temperature: float = 1.0, top: int = 0, stream=None):
    """resq_token_logprobs -> dict(logp, entropy, peak, log_sum[, top_ids, top_logp]) of the rows of logits [M, V] (bf16 or
    fp32) for tokens int64 [M] (outside 0 .. V - 1: none, logp 0).  top > 0: ids int32 [M, top] and log-probabilities of the
    largest logits, largest first, equal ones by lower id."""
    M, V, ld, code, index = _first(logits, "logits")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: token_logprobs(logits, tokens, temperature, top))
    tok = _vector(tokens, "tokens", M, torch.int64, index)
    top = min(max(top, -1), MAX_TOP + 1)  # a C int would keep the low bits of a larger number; the library refuses both ends
    values = _new(4, M, _F32, index)
    logp, entropy, peak, log_sum = values.unbind()
    out = {"logp": logp, "entropy": entropy, "peak": peak, "log_sum": log_sum}
    ids = top_logp = None
    if top > 0:
        ids = out["top_ids"] = _new(M, top, torch.int32, index)
        top_logp = out["top_logp"] = _new(M, top, _F32, index)
    at = values.data_ptr()
    _check(lib().resq_token_logprobs(logits.data_ptr(), code, M, V, ld, tok, temperature, top, at, at + 4 * M, at + 8 * M, at + 12 * M,
                                     _ptr(ids), _ptr(top_logp), _raw_stream(index)))
    return out


def token_logprobs_backward(logits: torch.Tensor, tokens: torch.Tensor, logp: torch.Tensor, peak: torch.Tensor, log_sum: torch.Tensor,
                            entropy: Optional[torch.Tensor], dlogp: torch.Tensor, dentropy: Optional[torch.Tensor] = None,
                            temperature: float = 1.0, dlogits: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """resq_token_logprobs_backward: the gradient of the logits from token_logprobs' results and the gradients of logp and
    (optionally) entropy; dlogits may be the logits tensor itself."""
    M, V, ld, code, index = _first(logits, "logits")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: token_logprobs_backward(logits, tokens, logp, peak, log_sum, entropy, dlogp, dentropy,
                                                                         temperature, dlogits))
    _require(logp is not None and peak is not None and log_sum is not None and dlogp is not None, "logp, peak, log_sum and dlogp are needed")
    _require(dentropy is None or entropy is not None, "dentropy needs entropy")
    values = [_vector(tokens, "tokens", M, torch.int64, index)]
    values += [None if t is None else _vector(t, name, M, _F32, index)
               for name, t in (("logp", logp), ("peak", peak), ("log_sum", log_sum), ("entropy", entropy), ("dlogp", dlogp), ("dentropy", dentropy))]
    if dlogits is None:
        dlogits, ldd = _new_rows(M, V, logits.dtype, index), (V + 7) // 8 * 8
    else:
        ldd = _rows(dlogits, "dlogits", M, V, logits.dtype, index)
    _check(lib().resq_token_logprobs_backward(logits.data_ptr(), code, M, V, ld, values[0], temperature, *values[1:], dlogits.data_ptr(), ldd,
                                              _raw_stream(index)))
    return dlogits


# ------------------------------------------------------------------ paged cache, attention, verification of drafts
#
# As above: on the device of the first tensor, on `stream` or that device's current one.  A cache is a pair of tensors [pages,
# page_size, kv_heads, head_dim] with any strides that keep 16-byte rows (a transposed view of [pages, kv_heads, page_size,
# head_dim], or one half of a joint buffer).

MAX_SEQUENCES = 4096
MAX_GROUP_HEADS = 128


# The structs resq_paged_cache and resq_sequences, packed (a quarter of the time of filling a ctypes.Structure): addresses of k and v,
# then pages, page_size, kv_heads, head_dim and the strides of k and of v; addresses of q_start, kv_len and page_table, then count,
# max_pages and ld_table.
_PAGED_CACHE, _SEQUENCES = struct.Struct("2Q10q"), struct.Struct("3Q3q")


def _paged(k_cache: torch.Tensor, v_cache: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor, index: int):
    """The two structs of a paged call, and its kv_heads, head_dim and number of sequences."""
    shape = k_cache.shape
    if (k_cache.dtype is not _BF16 or v_cache.dtype is not _BF16 or len(shape) != 4 or v_cache.shape != shape or k_cache.get_device() != index
            or v_cache.get_device() != index):
        raise ValueError(f"k_cache and v_cache must be bf16 tensors of one shape [pages, page_size, kv_heads, head_dim] on cuda:{index}")
    kp, kr, kh, ki = k_cache.stride()
    vp, vr, vh, vi = v_cache.stride()
    if ki != 1 or vi != 1:
        raise ValueError("k_cache and v_cache must have unit inner stride")
    table = page_table.shape
    if page_table.dtype is not torch.int32 or len(table) != 2 or page_table.get_device() != index or (table[1] > 1 and page_table.stride(1) != 1):
        raise ValueError(f"page_table must be an int32 tensor [sequences, pages per sequence] on cuda:{index} with unit inner stride")
    count, per_seq = table
    at_start, at_len = _vector(q_start, "q_start", count + 1, torch.int32, index), _vector(kv_len, "kv_len", count, torch.int32, index)
    pages, page, heads, dim = shape
    return (_PAGED_CACHE.pack(k_cache.data_ptr(), v_cache.data_ptr(), pages, page, heads, dim, kp, kr, kh, vp, vr, vh),
            _SEQUENCES.pack(at_start, at_len, page_table.data_ptr(), count, per_seq, page_table.stride(0) if count > 1 else per_seq),
            heads, dim, count)


def rope_append(qkv: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor,
                page_table: torch.Tensor, inv_freq: torch.Tensor, bias: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                pairs: bool = False, q: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """resq_rope_append: rows of qkv [T, (Hq + 2 Hkv) D] (bf16 or fp32) plus bias -> the rotated queries q [T, Hq D] bf16 (returned);
    rotated keys and the values go to their slots of the cache.

    q_start int32 [B + 1], kv_len int32 [B] (keys of each sequence, the new ones among them), page_table int32 [B, pages per
    sequence].  inv_freq fp64 [rot / 2]; pairs: neighbouring elements turn into each other, not those rot / 2 apart.  q may be
    qkv[:, :Hq * D] of a bf16 qkv."""
    T, W, ld, code, index = _first(qkv, "qkv")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: rope_append(qkv, k_cache, v_cache, q_start, kv_len, page_table, inv_freq, bias, positions, pairs, q))
    cache, seqs, Hkv, D, _ = _paged(k_cache, v_cache, q_start, kv_len, page_table, index)
    _require(D > 0 and W % D == 0 and W > 2 * Hkv * D, f"qkv must have (Hq + 2 * {Hkv}) heads of {D} columns")
    Hq = W // D - 2 * Hkv
    half = inv_freq.shape[0] if inv_freq.dim() == 1 else -1
    freq = _vector(inv_freq, "inv_freq", half, torch.float64, index)
    at_bias = None if bias is None else _vector(bias, "bias", W, _BF16, index)
    at_pos = None if positions is None else _vector(positions, "positions", T, torch.int32, index)
    if q is None:
        q, ldq = _new(T, Hq * D, _BF16, index), Hq * D
    else:
        ldq = _rows(q, "q", T, Hq * D, _BF16, index)
    _check(lib().resq_rope_append(qkv.data_ptr(), code, T, ld, Hq, Hkv, D, at_bias, freq, 2 * half, 1 if pairs else 0, at_pos,
                                  cache, seqs, q.data_ptr(), ldq, _raw_stream(index)))
    return q


@functools.lru_cache(maxsize=1024)
def paged_attention_workspace_bytes(T: int, count: int, Hq: int, Hkv: int, D: int, max_new: int = 0) -> int:
    return int(lib().resq_paged_attention_workspace_bytes(T, count, Hq, Hkv, D, max_new))


def paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor,
                    page_table: torch.Tensor, scale: Optional[float] = None, max_new: Optional[int] = None, lse: bool = False,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """resq_paged_attention: attention of the new tokens' queries q [T, Hq D] over the cache -> out [T, Hq D] bf16, or (out,
    lse [T, Hq] fp32).

    scale: 1 / sqrt(head_dim) unless given.  max_new: the largest number of new tokens per sequence if the host knows it; it
    chooses the kernel."""
    T, W, ldq, code, index = _first(q, "q")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: paged_attention(q, k_cache, v_cache, q_start, kv_len, page_table, scale, max_new, lse, out,
                                                                 workspace))
    _require(code == OUT_BF16, "q must be bf16")
    cache, seqs, Hkv, D, count = _paged(k_cache, v_cache, q_start, kv_len, page_table, index)
    _require(D > 0 and W % D == 0, f"q must have heads of {D} columns")
    Hq = W // D
    max_new = 0 if max_new is None else min(max(int(max_new), 0), T)
    if out is None:
        out, ldo = _new(T, W, _BF16, index), W
    else:
        ldo = _rows(out, "out", T, W, _BF16, index)
    values = _new(T, Hq, _F32, index) if lse else None
    if workspace is None:
        workspace = _new(1, max(paged_attention_workspace_bytes(T, count, Hq, Hkv, D, max_new), 256), torch.uint8, index)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{index}")
    _check(lib().resq_paged_attention(q.data_ptr(), T, ldq, Hq, Hkv, D, cache, seqs, max_new,
                                      D ** -0.5 if scale is None else scale, out.data_ptr(), ldo, _ptr(values), workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), _raw_stream(index)))
    return (out, values) if lse else out


@functools.lru_cache(maxsize=1024)
def verify_drafts_workspace_bytes(R: int) -> int:
    return int(lib().resq_verify_drafts_workspace_bytes(R))


def verify_drafts(logits: torch.Tensor, row_start: torch.Tensor, drafts: torch.Tensor, u: Optional[torch.Tensor] = None,
                  noise: Optional[torch.Tensor] = None, draft_logits: Optional[torch.Tensor] = None, draft_peak: Optional[torch.Tensor] = None,
                  draft_log_sum: Optional[torch.Tensor] = None, temperature: float = 1.0, out: Optional[dict] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None):
    """resq_verify_drafts -> dict(accepted int32 [B], tokens int64 [R], logp fp32 [R]): of each sequence's rows row_start[b] ..
    row_start[b + 1] - 1 of the target's logits [R, V] the drafts that are kept, then the token that follows them, then -1.

    drafts int64 [R] (a sequence's last row proposes none); u fp32 [R] uniform, noise fp32 [B, V] exponential.  draft_logits
    with the draft's peak and log_sum (from token_logprobs at the same temperature), or None for drafts without probabilities.
    temperature 0: the largest logits, without random numbers.  out: the dict of an earlier call of the same sizes, written anew."""
    R, V, ld, code, index = _first(logits, "logits")
    if stream is not None or _current_device() != index:
        return _elsewhere(index, stream, lambda: verify_drafts(logits, row_start, drafts, u, noise, draft_logits, draft_peak, draft_log_sum,
                                                               temperature, out, workspace))
    count = row_start.shape[0] - 1 if row_start.dim() == 1 else -1
    _require(count >= 1, "row_start must be a vector of at least 2 elements")
    start, at_drafts = _vector(row_start, "row_start", count + 1, torch.int32, index), _vector(drafts, "drafts", R, torch.int64, index)
    at_u = at_noise = at_draft = at_peak = at_sum = None
    lde = ldd = 0
    if temperature != 0:
        _require(1e-6 <= temperature <= 1e6, "temperature must be 0 or lie in 1e-6 .. 1e6")  # (one of 1e-50 would arrive as 0)
        _require(u is not None and noise is not None, "u and noise are needed to draw tokens")
        at_u = _vector(u, "u", R, _F32, index)
        lde, at_noise = _rows(noise, "noise", count, V, _F32, index), noise.data_ptr()
        if draft_logits is not None:
            _require(draft_peak is not None and draft_log_sum is not None, "draft_logits needs draft_peak and draft_log_sum")
            ldd, at_draft = _rows(draft_logits, "draft_logits", R, V, logits.dtype, index), draft_logits.data_ptr()
            at_peak, at_sum = _vector(draft_peak, "draft_peak", R, _F32, index), _vector(draft_log_sum, "draft_log_sum", R, _F32, index)
    if out is None:
        out = {"accepted": _new_vector(count, torch.int32, index), "tokens": _new_vector(R, torch.int64, index), "logp": _new_vector(R, _F32, index)}
    if workspace is None:
        workspace = _new(1, verify_drafts_workspace_bytes(R), torch.uint8, index)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{index}")
    _check(lib().resq_verify_drafts(
        logits.data_ptr(), code, R, V, ld, start, count, at_drafts, at_u, at_noise, lde, at_draft, ldd, at_peak, at_sum, temperature,
        _vector(out["accepted"], "accepted", count, torch.int32, index), _vector(out["tokens"], "tokens", R, torch.int64, index),
        _vector(out["logp"], "logp", R, _F32, index), workspace.data_ptr(), workspace.numel() * workspace.element_size(), _raw_stream(index)))
    return out


def check(workspace: torch.Tensor, stream=None) -> int:
    """resq_check: synchronize and return the device status word."""
    return int(lib().resq_check(workspace.data_ptr(), _stream(stream)))


# ------------------------------------------------------------------ diagnostics

KERNEL_KINDS = ("quantize", "select", "gemm", "splitk_reduce")


def kernel_launches() -> int:
    """resq_kernel_launches: kernels launched by the library in this process so far."""
    return int(lib().resq_kernel_launches())


def debug_expire_next_wait(on: bool = True, attention: bool = False) -> None:
    """resq_debug_expire_next_wait: the next decode-sized GEMM launch, or the next attention of long chunks, lets its bounded wait
    run out (test hook)."""
    _check(lib().resq_debug_expire_next_wait((2 if attention else 1) if on else 0))


def profile_enable(on: bool) -> None:
    _check(lib().resq_profile_enable(1 if on else 0))


def profile_read():
    """resq_profile_read -> {kind: (device ms, launches)} since the last read."""
    ms = (ctypes.c_double * 4)()
    n = (ctypes.c_int64 * 4)()
    _check(lib().resq_profile_read(ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(n, ctypes.c_void_p)))
    return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(KERNEL_KINDS)}
