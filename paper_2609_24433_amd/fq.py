"""Python binding of libfq (the C ABI in include/fq.h), over torch device tensors.

Argument marshalling only: tensors are used for their device pointers and torch's
current HIP stream; every step of the projection runs in the library's kernels.
If libfq.so is missing the import fails loudly; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
import struct
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfq.so")

FQ_OK, FQ_ERR_ALIAS = 0, 7
_STATUS = {1: "FQ_ERR_NULL", 2: "FQ_ERR_SHAPE", 3: "FQ_ERR_UNSUPPORTED", 4: "FQ_ERR_ALIGN",
           5: "FQ_ERR_WORKSPACE", 6: "FQ_ERR_HIP", FQ_ERR_ALIAS: "FQ_ERR_ALIAS"}

EXPORTED = ["fq_fwht_quant", "fq_quantize_weights", "fq_packed_weight_bytes", "fq_pack_weights",
            "fq_unpack_weights", "fq_gemm_workspace_bytes", "fq_gemm_w4a4", "fq_gemm_w8a8",
            "fq_linear_workspace_bytes", "fq_linear", "fq_gemm_w4a16_workspace_bytes", "fq_gemm_w4a16",
            "fq_rotate_quant_workspace_bytes", "fq_rotate_quant", "fq_quantize_weights_rotated",
            "fq_transform", "fq_gptq_hessian", "fq_gptq_factor_workspace_bytes", "fq_gptq_factor",
            "fq_gptq_sweep_workspace_bytes", "fq_gptq_sweep",
            "fq_linear_static_max_workspace_bytes", "fq_linear_static",
            "fq_rope_table", "fq_qk_rope", "fq_cache_append", "fq_cache_read",
            "fq_cache_attention_workspace_bytes", "fq_cache_attention",
            "fq_cross_attention_workspace_bytes", "fq_cross_attention",
            "fq_norm_quant", "fq_norm_mx_quant", "fq_read_codes", "fq_mx_quant", "fq_mx_read", "fq_mx_packed_bytes", "fq_mx_pack",
            "fq_mx_unpack", "fq_mx_gemm_workspace_bytes", "fq_mx_gemm", "fq_mx_linear_workspace_bytes", "fq_mx_linear",
            "fq_status_string", "fq_last_error"]


class FQError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "(python -m paper_2609_24433_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    # descriptors (fq_heads and its kin) come as packed bytes
    desc = ctypes.c_char_p
    vp, i64, i32, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    sig = {
        "fq_fwht_quant": [vp, i64, vp, vp, i64, i64, i32, i32, f32, vp, vp, vp],
        "fq_quantize_weights": [vp, i64, vp, vp, i64, i64, i32, i32, vp, vp, vp],
        "fq_pack_weights": [vp, i64, i64, i32, vp, vp],
        "fq_unpack_weights": [vp, i64, i64, i32, vp, vp],
        "fq_gemm_w4a4": [vp, vp, vp, vp, vp, vp, i64, vp, i64, i64, i64, vp, sz, vp],
        "fq_gemm_w8a8": [vp, vp, vp, vp, vp, vp, i64, vp, i64, i64, i64, vp, sz, vp],
        "fq_linear": [vp, i64, vp, vp, i64, i64, i64, i32, i32, f32, vp, vp, vp, vp, i64, vp, sz, vp],
        "fq_gemm_w4a16": [vp, i64, vp, vp, vp, vp, i64, vp, i64, i64, i64, vp, sz, vp],
        "fq_rotate_quant": [vp, i64, vp, vp, vp, vp, i64, i64, i32, i32, f32, vp, vp, vp, sz, vp],
        "fq_quantize_weights_rotated": [vp, i64, vp, vp, vp, vp, i64, i64, i32, i32, vp, vp, vp, sz, vp],
        "fq_transform": [vp, i32, i64, vp, vp, i64, i64, i32, vp, vp],
        "fq_gptq_hessian": [vp, i64, i64, i64, vp, i32, vp],
        "fq_gptq_factor": [vp, i64, ctypes.c_double, vp, vp, sz, vp],
        "fq_gptq_sweep": [vp, i64, vp, i64, i64, i32, i32, vp, vp, vp, sz, vp],
        "fq_linear_static": [vp, i64, vp, vp, i64, i64, i64, i32, i32, f32, vp, vp, vp, vp, i64, vp],
        "fq_rope_table": [vp, ctypes.c_double, i64, i64, vp, vp],
        "fq_qk_rope": [desc, i32, desc, i32, desc, i64, i32, vp, vp, vp],
        "fq_cache_append": [desc, desc, desc, desc, desc, i32, desc, i64, vp, vp],
        "fq_cache_read": [desc, vp, i64, vp, vp, i64, i64, vp, vp, vp],
        "fq_cache_attention": [desc, i32, i64, desc, desc, f32, i32, vp, vp, sz, vp],
        "fq_cross_attention": [desc, desc, desc, vp, vp, i64, i64, i64, i64, i32, i32, i32, f32, vp, vp, sz, vp],
        "fq_norm_quant": [vp, i64, vp, i64, vp, f32, vp, i64, i64, i32, i32, f32, vp, i64, vp, vp, vp],
        "fq_norm_mx_quant": [vp, i64, vp, i64, vp, f32, vp, i64, i64, i32, vp, i64, vp, vp, vp],
        "fq_read_codes": [vp, vp, i64, i64, i32, vp, i64, vp],
        "fq_mx_quant": [vp, i32, i64, vp, vp, i64, i64, i32, vp, vp, vp],
        "fq_mx_read": [vp, vp, i64, i64, vp, i64, vp],
        "fq_mx_pack": [vp, i64, i64, vp, vp],
        "fq_mx_unpack": [vp, i64, i64, vp, vp],
        "fq_mx_gemm": [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, vp, sz, vp],
        "fq_mx_linear": [vp, i64, vp, vp, i64, i64, i64, i32, vp, vp, vp, vp, i64, vp, sz, vp],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    for name, args in {"fq_packed_weight_bytes": [i64, i64, i32],
                       "fq_gemm_workspace_bytes": [i64, i64, i64, i32],
                       "fq_linear_workspace_bytes": [i64, i64, i64, i32],
                       "fq_gemm_w4a16_workspace_bytes": [i64, i64, i64],
                       "fq_rotate_quant_workspace_bytes": [i64, i64],
                       "fq_gptq_factor_workspace_bytes": [i64],
                       "fq_gptq_sweep_workspace_bytes": [i64, i64],
                       "fq_linear_static_max_workspace_bytes": [],
                       "fq_cache_attention_workspace_bytes": [i64, i32, i32, i32, i64, i64, i64],
                       "fq_cross_attention_workspace_bytes": [i64, i64, i64, i32, i32, i32],
                       "fq_mx_packed_bytes": [i64, i64], "fq_mx_gemm_workspace_bytes": [i64, i64, i64],
                       "fq_mx_linear_workspace_bytes": [i64, i64, i64]}.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = sz
    lib.fq_status_string.argtypes = [ctypes.c_int]
    lib.fq_status_string.restype = ctypes.c_char_p
    lib.fq_last_error.argtypes = []
    lib.fq_last_error.restype = ctypes.c_char_p
    return lib


LIB = _load()


def _check(rc: int) -> None:
    if rc != FQ_OK:
        raise FQError(rc, LIB.fq_last_error().decode())


def _p(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream: Optional[torch.cuda.Stream] = None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


# The entry points that a serving loop calls eagerly hand plain integers to ctypes (no c_void_p
# objects) and take the current stream's handle without building a Stream object: a small
# projection's call is bound by the host, and the marshalling was most of it (fq.linear at
# M 64, K = N = 1024: 12.8 us a call with them, 8.0 without, 3.9 of it the kernel).

def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_handle() -> int:
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


# ---------------------------------------------------------------- raw C-ABI calls (pointers)

def fwht_quant_raw(x_ptr, ldx, smooth_ptr, M, K, b, bits, clip_ratio, codes_ptr, delta_ptr, stream_ptr,
                   post_ptr=None):
    _check(LIB.fq_fwht_quant(x_ptr, ldx, smooth_ptr, post_ptr, M, K, b, bits, clip_ratio, codes_ptr, delta_ptr,
                             stream_ptr))


# ---------------------------------------------------------------- tensor API

def code_bytes(K: int, bits: int) -> int:
    return K * bits // 8


def _require(cond: bool, msg: str) -> None:
    if not cond:
        raise ValueError(msg)


def _check_out(out: Optional[torch.Tensor], M: int, N: int) -> None:
    """A caller-supplied output must be what the library writes: bf16 [M, N] rows with unit
    column stride (the row stride is passed on as ldy)."""
    if out is not None:
        _require(out.dtype == torch.bfloat16 and tuple(out.shape) == (M, N) and (M == 0 or out.stride(1) == 1),
                 "out: bf16 [M, N] with unit column stride")


def fwht_quant(x: torch.Tensor, b: int, bits: int, clip_ratio: float = 1.0,
               smooth_inv: Optional[torch.Tensor] = None, out_codes: Optional[torch.Tensor] = None,
               out_delta: Optional[torch.Tensor] = None,
               post_inv: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Prologue: x bf16 [M, K] (row stride x.stride(0)) -> (codes uint8 [M, K*bits/8], delta fp32 [M]).
    smooth_inv: fold-before S^-1 (before the rotation); post_inv: fold-after P^-1 (after it)."""
    M, K = x.shape
    assert x.dtype == torch.bfloat16 and (M == 0 or x.stride(1) == 1)
    if out_codes is not None:
        _require(out_codes.dtype in (torch.uint8, torch.int8) and out_codes.is_contiguous()
                 and tuple(out_codes.shape) == (M, code_bytes(K, bits)), "out_codes: contiguous [M, K*bits/8] bytes")
    if out_delta is not None:
        _require(out_delta.dtype == torch.float32 and out_delta.is_contiguous() and out_delta.numel() == M,
                 "out_delta: contiguous fp32 [M]")
    codes = out_codes if out_codes is not None else torch.empty((M, code_bytes(K, bits)), dtype=torch.uint8, device=x.device)
    delta = out_delta if out_delta is not None else torch.empty((M,), dtype=torch.float32, device=x.device)
    _check(LIB.fq_fwht_quant(x.data_ptr(), x.stride(0) if M else K, _ptr(smooth_inv), _ptr(post_inv), M, K, b, bits,
                             clip_ratio, codes.data_ptr(), delta.data_ptr(), _stream_handle()))
    return codes, delta


def quantize_weights(w: torch.Tensor, b: int, bits: int, col_scale: Optional[torch.Tensor] = None,
                     post_scale: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Offline fold + RTN: w fp32 [N, K] -> (codes int8 [N, K], scales fp32 [N]).
    col_scale: fold-before S (before the rotation); post_scale: fold-after P (after it)."""
    N, K = w.shape
    assert w.dtype == torch.float32 and w.stride(1) == 1
    codes = torch.empty((N, K), dtype=torch.int8, device=w.device)
    scale = torch.empty((N,), dtype=torch.float32, device=w.device)
    _check(LIB.fq_quantize_weights(_p(w), w.stride(0), _p(col_scale), _p(post_scale), N, K, b, bits, _p(codes),
                                   _p(scale), _stream()))
    return codes, scale


def packed_weight_bytes(N: int, K: int, bits: int) -> int:
    return int(LIB.fq_packed_weight_bytes(N, K, bits))


def pack_weights(codes: torch.Tensor, bits: int) -> torch.Tensor:
    N, K = codes.shape
    assert codes.dtype == torch.int8 and codes.is_contiguous()
    out = torch.empty((packed_weight_bytes(N, K, bits),), dtype=torch.uint8, device=codes.device)
    _check(LIB.fq_pack_weights(_p(codes), N, K, bits, _p(out), _stream()))
    return out


def unpack_weights(packed: torch.Tensor, N: int, K: int, bits: int) -> torch.Tensor:
    out = torch.empty((N, K), dtype=torch.int8, device=packed.device)
    _check(LIB.fq_unpack_weights(_p(packed), N, K, bits, _p(out), _stream()))
    return out


def gemm_workspace_bytes(M: int, N: int, K: int, bits: int) -> int:
    return int(LIB.fq_gemm_workspace_bytes(M, N, K, bits))


def linear_workspace_bytes(M: int, N: int, K: int, bits: int) -> int:
    return int(LIB.fq_linear_workspace_bytes(M, N, K, bits))


def workspace(nbytes: int, device) -> torch.Tensor:
    """Scratch for the GEMM / fused-linear entry points (no initialization needed)."""
    return torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=device)


def _scratch(nbytes: int, device) -> Optional[torch.Tensor]:
    """A call's own workspace, or None where the shape needs none."""
    return workspace(nbytes, device) if nbytes else None


def gemm(a_codes: torch.Tensor, delta: torch.Tensor, w_packed: torch.Tensor, w_scale: torch.Tensor,
         N: int, K: int, bits: int, bias: Optional[torch.Tensor] = None, want_acc: bool = False,
         ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
    """Integer GEMM + eq. (8) epilogue.  Returns y bf16 [M, N] (and int32 acc if want_acc)."""
    M = a_codes.shape[0]
    _require(a_codes.dtype in (torch.uint8, torch.int8) and tuple(a_codes.shape) == (M, code_bytes(K, bits))
             and a_codes.is_contiguous(), "a_codes: canonical contiguous [M, K*bits/8] bytes")
    _check_out(out, M, N)
    y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=a_codes.device)
    acc = torch.empty((M, N), dtype=torch.int32, device=a_codes.device) if want_acc else None
    ws = _scratch(LIB.fq_gemm_workspace_bytes(M, N, K, bits), a_codes.device) if ws is None else ws
    fn = LIB.fq_gemm_w4a4 if bits == 4 else LIB.fq_gemm_w8a8
    _check(fn(a_codes.data_ptr(), _ptr(delta), _ptr(w_packed), _ptr(w_scale), _ptr(bias), y.data_ptr(),
              y.stride(0) if M else N, _ptr(acc), M, N, K, _ptr(ws), 0 if ws is None else ws.numel(), _stream_handle()))
    return (y, acc) if want_acc else y


def linear(x: torch.Tensor, w_packed: torch.Tensor, w_scale: torch.Tensor, N: int, b: int, bits: int,
           clip_ratio: float = 1.0, smooth_inv: Optional[torch.Tensor] = None,
           bias: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
           out: Optional[torch.Tensor] = None, post_inv: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Fused projection: bf16 x [M, K] -> bf16 y [M, N]."""
    M, K = x.shape
    assert x.dtype == torch.bfloat16 and (M == 0 or x.stride(1) == 1)
    _check_out(out, M, N)
    if out is not None:
        y = out
    elif type(x) is torch.Tensor:
        y = x.new_empty((M, N))  # (0.2 us less than torch.empty, but a subclass would give its own kind)
    else:
        y = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    ws = _scratch(LIB.fq_linear_workspace_bytes(M, N, K, bits), x.device) if ws is None else ws
    _check(LIB.fq_linear(x.data_ptr(), x.stride(0) if M else K, _ptr(smooth_inv), _ptr(post_inv), M, K, N, b, bits,
                         clip_ratio, None if w_packed is None else w_packed.data_ptr(),
                         None if w_scale is None else w_scale.data_ptr(), _ptr(bias), y.data_ptr(),
                         y.stride(0) if M else N, _ptr(ws), 0 if ws is None else ws.numel(), _stream_handle()))
    return y


def linear_static(x: torch.Tensor, w_packed: torch.Tensor, w_scale: torch.Tensor, N: int, b: int, bits: int,
                  clip_ratio: float = 1.0, smooth_inv: Optional[torch.Tensor] = None,
                  bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  post_inv: Optional[torch.Tensor] = None) -> torch.Tensor:
    """fq_linear without a workspace argument: the library's own device scratch (calls that
    overlap on one device race)."""
    M, K = x.shape
    _require(x.dtype == torch.bfloat16 and (M == 0 or x.stride(1) == 1), "x: bf16 [M, K] with unit column stride")
    _check_out(out, M, N)
    y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    _check(LIB.fq_linear_static(x.data_ptr(), x.stride(0) if M else K, _ptr(smooth_inv), _ptr(post_inv), M, K, N, b, bits,
                                clip_ratio, _ptr(w_packed), _ptr(w_scale), _ptr(bias), y.data_ptr(),
                                y.stride(0) if M else N, _stream_handle()))
    return y


def rotate_quant(x: torch.Tensor, perm: Optional[torch.Tensor], blocks: torch.Tensor, b: int, bits: int,
                 clip_ratio: float = 1.0, smooth_inv: Optional[torch.Tensor] = None,
                 post_inv: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Prologue with the stored composite rotation (permutation int32 [K] or None, blocks fp32
    [K/b, b, b]): x bf16 [M, K] -> (codes [M, K*bits/8], delta fp32 [M])."""
    M, K = x.shape
    assert x.dtype == torch.bfloat16 and (M == 0 or x.stride(1) == 1)
    codes = torch.empty((M, code_bytes(K, bits)), dtype=torch.uint8, device=x.device)
    delta = torch.empty((M,), dtype=torch.float32, device=x.device)
    ws = workspace(LIB.fq_rotate_quant_workspace_bytes(M, K), x.device)
    _check(LIB.fq_rotate_quant(x.data_ptr(), x.stride(0) if M else K, _ptr(perm), _ptr(blocks), _ptr(smooth_inv),
                               _ptr(post_inv), M, K, b, bits, clip_ratio, codes.data_ptr(), delta.data_ptr(),
                               ws.data_ptr(), ws.numel(), _stream_handle()))
    return codes, delta


def quantize_weights_rotated(w: torch.Tensor, perm: Optional[torch.Tensor], blocks: torch.Tensor, b: int,
                             bits: int, col_scale: Optional[torch.Tensor] = None,
                             post_scale: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Offline fold + RTN for the composite rotation: w fp32 [N, K] -> (codes int8 [N, K], scales fp32 [N])."""
    N, K = w.shape
    assert w.dtype == torch.float32 and w.stride(1) == 1
    codes = torch.empty((N, K), dtype=torch.int8, device=w.device)
    scale = torch.empty((N,), dtype=torch.float32, device=w.device)
    ws = workspace(int(LIB.fq_rotate_quant_workspace_bytes(N, K)), w.device)
    _check(LIB.fq_quantize_weights_rotated(_p(w), w.stride(0), _p(perm), _p(blocks), _p(col_scale),
                                           _p(post_scale), N, K, b, bits, _p(codes), _p(scale), _p(ws),
                                           ws.numel(), _stream()))
    return codes, scale


def transform(x: torch.Tensor, b: int, pre_mult: Optional[torch.Tensor] = None,
              post_mult: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The prologue's transform without quantization: bf16 or fp32 rows [M, K] -> fp32 [M, K]
    (unnormalized blockwise butterfly between the optional multipliers)."""
    M, K = x.shape
    assert x.dtype in (torch.bfloat16, torch.float32) and (M == 0 or x.stride(1) == 1)
    z = torch.empty((M, K), dtype=torch.float32, device=x.device)
    _check(LIB.fq_transform(_p(x), int(x.dtype == torch.float32), x.stride(0) if M else K, _p(pre_mult),
                            _p(post_mult), M, K, b, _p(z), _stream()))
    return z


def gptq_hessian(z: torch.Tensor, G: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
    """G (+)= z^T z in fp64 for transformed tokens z fp32 [T, K]."""
    T, K = z.shape
    assert z.dtype == torch.float32 and (T == 0 or z.stride(1) == 1)
    if G is None:
        G = torch.empty((K, K), dtype=torch.float64, device=z.device)
    _check(LIB.fq_gptq_hessian(_p(z), z.stride(0) if T else K, T, K, _p(G), int(accumulate), _stream()))
    return G


def gptq_factor(G: torch.Tensor, damp: float = 0.01) -> torch.Tensor:
    """U fp64 [K, K] upper triangular with (G + damp * mean(diag G) I)^-1 = U^T U."""
    K = G.shape[0]
    assert G.dtype == torch.float64 and G.is_contiguous()
    U = torch.empty((K, K), dtype=torch.float64, device=G.device)
    ws = workspace(int(LIB.fq_gptq_factor_workspace_bytes(K)), G.device)
    _check(LIB.fq_gptq_factor(_p(G), K, damp, _p(U), _p(ws), ws.numel(), _stream()))
    return U


def gptq_sweep(w_t: torch.Tensor, U: torch.Tensor, b: int, bits: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """GPTQ column sweep on weight rows w_t fp32 [N, K] transformed with block size b ->
    (codes int8 [N, K], scales fp32 [N])."""
    N, K = w_t.shape
    assert w_t.dtype == torch.float32 and w_t.stride(1) == 1 and U.dtype == torch.float64 and U.is_contiguous()
    codes = torch.empty((N, K), dtype=torch.int8, device=w_t.device)
    scales = torch.empty((N,), dtype=torch.float32, device=w_t.device)
    ws = workspace(int(LIB.fq_gptq_sweep_workspace_bytes(N, K)), w_t.device)
    _check(LIB.fq_gptq_sweep(_p(w_t), w_t.stride(0), _p(U), N, K, b, bits, _p(codes), _p(scales), _p(ws),
                             ws.numel(), _stream()))
    return codes, scales


def gptq_quantize_weights(w: torch.Tensor, calib: torch.Tensor, b: int, bits: int,
                          col_scale: Optional[torch.Tensor] = None, post_scale: Optional[torch.Tensor] = None,
                          smooth_inv: Optional[torch.Tensor] = None, post_inv: Optional[torch.Tensor] = None,
                          damp: float = 0.01) -> Tuple[torch.Tensor, torch.Tensor]:
    """Eq. (7) on the GPU: calibration tokens (bf16 [T, K]) through the runtime transform,
    G = Z Z^T, the damped factor, and the sweep over the folded weight rows (fp32 [N, K]).
    Returns (codes int8 [N, K], scales fp32 [N]) in the layout of quantize_weights."""
    z = transform(calib, b, smooth_inv, post_inv)
    U = gptq_factor(gptq_hessian(z), damp)
    w_t = transform(w, b, col_scale, post_scale)
    return gptq_sweep(w_t, U, b, bits)


def w4a16_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(LIB.fq_gemm_w4a16_workspace_bytes(M, N, K))


def gemm_w4a16(x: torch.Tensor, w_packed: torch.Tensor, w_scale: torch.Tensor, N: int,
               bias: Optional[torch.Tensor] = None, want_acc: bool = False, ws: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None):
    """Weight-only INT4 projection: bf16 x [M, K] times packed INT4 weights -> bf16 y [M, N]
    (and the fp32 sums if want_acc)."""
    M, K = x.shape
    assert x.dtype == torch.bfloat16 and (M == 0 or x.stride(1) == 1)
    _check_out(out, M, N)
    y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    acc = torch.empty((M, N), dtype=torch.float32, device=x.device) if want_acc else None
    ws = _scratch(LIB.fq_gemm_w4a16_workspace_bytes(M, N, K), x.device) if ws is None else ws
    _check(LIB.fq_gemm_w4a16(x.data_ptr(), x.stride(0) if M else K, _ptr(w_packed), _ptr(w_scale), _ptr(bias),
                             y.data_ptr(), y.stride(0) if M else N, _ptr(acc), M, N, K, _ptr(ws),
                             0 if ws is None else ws.numel(), _stream_handle()))
    return (y, acc) if want_acc else y


class QuantLinear:
    """One consumer projection: folded, rounded and packed weights kept resident on the device."""

    def __init__(self, w: torch.Tensor, b: int, bits: int, col_scale: Optional[torch.Tensor] = None,
                 bias: Optional[torch.Tensor] = None, post_scale: Optional[torch.Tensor] = None):
        self.N, self.K = w.shape
        self.b, self.bits = b, bits
        codes, self.w_scale = quantize_weights(w, b, bits, col_scale, post_scale)
        self.w_packed = pack_weights(codes, bits)
        self.bias = bias

    def __call__(self, x: torch.Tensor, clip_ratio: float = 1.0, smooth_inv: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 post_inv: Optional[torch.Tensor] = None) -> torch.Tensor:
        return linear(x, self.w_packed, self.w_scale, self.N, self.b, self.bits, clip_ratio, smooth_inv,
                      self.bias, ws, out, post_inv)


# ---------------------------------------------------------------- attention between the projections

_HEADS = struct.Struct("=Qqqq").pack          # fq_heads
_ROPE = struct.Struct("=QqQQQfiii").pack      # fq_head_rope
_CACHE = struct.Struct("=QQQQqiiii").pack     # fq_kv_cache
_BATCH = struct.Struct("=QQQqqqq").pack       # fq_kv_batch


class KVCache(NamedTuple):
    """Pages of keys and values in 8 bits, one scale per page and head (kv_cache makes them)."""
    k_codes: torch.Tensor  # int8 [pages, heads, P, D]
    k_scale: torch.Tensor  # fp32 [pages, heads]
    v_codes: torch.Tensor  # int8 [pages, heads, P/16, D, 16]
    v_scale: torch.Tensor  # fp32 [pages, heads]


def kv_cache(pages: int, heads: int, page_tokens: int, head_dim: int, device="cuda") -> KVCache:
    """A pool of empty cache pages of page_tokens = 16, 32, 64 or 128 tokens."""
    return KVCache(torch.zeros((pages, heads, page_tokens, head_dim), dtype=torch.int8, device=device),
                   torch.zeros((pages, heads), dtype=torch.float32, device=device),
                   torch.zeros((pages, heads, page_tokens // 16, head_dim, 16), dtype=torch.int8, device=device),
                   torch.zeros((pages, heads), dtype=torch.float32, device=device))


# A decoding step's calls are bound by the host: these helpers build no message unless a check
# fails and read each property of a tensor once.  `dev` is the device of the call's first tensor (Tensor.get_device():
# -1 is the host): every other tensor's address is only good for a kernel on the same one.

_BF16, _F32, _I32, _I8 = torch.bfloat16, torch.float32, torch.int32, torch.int8


def _elsewhere(name: str, t: torch.Tensor, dev: int) -> ValueError:
    return ValueError(f"{name} is on {t.device}, the call's first tensor on {'the host' if dev < 0 else f'GPU {dev}'}")


def _refuse(rc: int, dev: int) -> None:
    """A failed call.  Where the tensors are on the host, the caller gave the library an output that overlaps an input: its
    other checks come first, with their errors, and nothing is launched on addresses that a kernel must not see."""
    if dev < 0 and rc == FQ_ERR_ALIAS:
        raise ValueError("the tensors are on the host, not on a GPU")
    _check(rc)


def _heads(x: torch.Tensor, name: str, dev: int) -> bytes:
    s = x.stride()
    if x.dtype is not _BF16 or s[-1] != 1:
        raise ValueError(f"{name}: bf16 with unit stride of the last dim")
    if x.get_device() != dev:
        raise _elsewhere(name, x, dev)
    return _HEADS(x.data_ptr(), s[0] if len(s) == 4 else 0, s[-3], s[-2])


def _index(t: Optional[torch.Tensor], n: int, name: str, dev: int) -> int:
    if t is None:
        return 0
    if t.dtype is not _I32 or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: contiguous int32 [{n}]")
    if t.get_device() != dev:
        raise _elsewhere(name, t, dev)
    return t.data_ptr()


def _weight(w: Optional[torch.Tensor], D: int, name: str, dev: int) -> int:
    if w is None:
        return 0
    if w.dtype is not _F32 or w.shape != (D,) or w.stride(0) != 1:
        raise ValueError(f"{name}: contiguous fp32 [{D}]")
    if w.get_device() != dev:
        raise _elsewhere(name, w, dev)
    return w.data_ptr()


def _cache_desc(c: KVCache, dev: int, growth: int = 0) -> Tuple[bytes, int, int, int]:
    kc, ks, vc, vs = c
    pages, H, P, D = kc.shape
    if (kc.dtype is not _I8 or vc.dtype is not _I8 or vc.shape != (pages, H, P // 16, D, 16) or not kc.is_contiguous()
            or not vc.is_contiguous()):
        raise ValueError("cache codes: contiguous int8 [pages, heads, P, D] and [pages, heads, P/16, D, 16]")
    if (ks.dtype is not _F32 or vs.dtype is not _F32 or ks.shape != (pages, H) or vs.shape != (pages, H)
            or not ks.is_contiguous() or not vs.is_contiguous()):
        raise ValueError("cache scales: contiguous fp32 [pages, heads]")
    if kc.get_device() != dev or ks.get_device() != dev or vc.get_device() != dev or vs.get_device() != dev:
        raise _elsewhere("the cache", next(t for t in c if t.get_device() != dev), dev)
    return _CACHE(kc.data_ptr(), ks.data_ptr(), vc.data_ptr(), vs.data_ptr(), pages, H, P, D, growth), H, P, D


def _table_shape(page_table: torch.Tensor, dev: int) -> Tuple[int, int]:
    shape = page_table.shape
    if page_table.dtype is not _I32 or len(shape) != 2 or not page_table.is_contiguous():
        raise ValueError("page_table: contiguous int32 [seqs, pages]")
    if page_table.get_device() != dev:
        raise _elsewhere("page_table", page_table, dev)
    return shape


def _batch_desc(page_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, max_new: int, max_kv: int, dev: int) -> bytes:
    B, width = _table_shape(page_table, dev)
    return _BATCH(_index(q_start, B + 1, "q_start", dev), _index(kv_len, B, "kv_len", dev), page_table.data_ptr(), width, B, max_new,
                  max_kv)


def _rope_desc(table, positions, T, q_weight, k_weight, D, eps, interleaved, dev) -> bytes:
    length = pairs = at = 0
    if table is not None:
        shape = table.shape
        if table.dtype is not _F32 or len(shape) != 3 or shape[2] != 2 or not table.is_contiguous():
            raise ValueError("table: contiguous fp32 [length, R/2, 2]")
        if table.get_device() != dev:
            raise _elsewhere("table", table, dev)
        length, pairs, at = shape[0], shape[1], table.data_ptr()
    return _ROPE(at, length, _index(positions, T, "positions", dev), _weight(q_weight, D, "q_weight", dev),
                 _weight(k_weight, D, "k_weight", dev), eps, 2 * pairs, interleaved, 0)


def _rows(out: Optional[torch.Tensor], like: torch.Tensor, shape: Tuple[int, ...], name: str, dev: int) -> torch.Tensor:
    """A contiguous bf16 output, the caller's or a new one on the device of `like` (bf16)."""
    if out is None:
        return like.new_empty(shape) if type(like) is torch.Tensor else torch.empty(shape, dtype=_BF16, device=like.device)
    if out.dtype is not _BF16 or out.shape != shape or not out.is_contiguous():
        raise ValueError(f"{name}: contiguous bf16 {tuple(shape)}")
    if out.get_device() != dev:
        raise _elsewhere(name, out, dev)
    return out


def _room(ws: Optional[torch.Tensor], dev: int) -> Tuple[Optional[int], int]:
    """Address and bytes of a workspace."""
    if ws is None:
        return None, 0
    if ws.get_device() != dev:
        raise _elsewhere("ws", ws, dev)
    return ws.data_ptr(), ws.numel()


def rope_frequencies(rot: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     original_length: int = 0, fast: float = 32.0, slow: float = 1.0) -> Tuple[torch.Tensor, float]:
    """(radians per position fp64 [rot/2], magnitude of the rotation) of base^(-2i/rot), as they are
    or scaled for contexts `factor` times longer than `original_length`:
      "linear"    every frequency divided by factor (positions compressed)
      "base"      the base raised by factor^(rot/(rot-2)): the fastest pair stays, the slowest is divided by factor
      "by_parts"  pairs that turn more than `fast` times within original_length stay, those under `slow` turns are
                  divided by factor, those between in proportion; magnitude 1 + 0.1 ln(factor)"""
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    if scaling == "base":
        _require(rot > 2, "a scaled base needs more than one pair")
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-i / rot)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "by_parts":
        _require(original_length > 0 and fast > slow, "by_parts needs original_length and fast > slow")
        turns = f * original_length / (2 * math.pi)
        keep = ((turns - slow) / (fast - slow)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1 - keep), 1.0 + 0.1 * math.log(factor) if factor > 1 else 1.0
    _require(scaling in (None, "base"), f"unknown scaling {scaling!r}")
    return f, 1.0


def rope_table(length: int, inv_freq: torch.Tensor, magnitude: float = 1.0, device="cuda") -> torch.Tensor:
    """cos and sin of m * inv_freq[i] for m < length, angles in fp64: fp32 [length, pairs, 2]."""
    f = inv_freq.to(device=device, dtype=torch.float64).contiguous()
    _require(f.get_device() >= 0, "a table is made on a GPU")
    table = torch.empty((length, f.numel(), 2), dtype=torch.float32, device=f.device)
    _check(LIB.fq_rope_table(_p(f), magnitude, length, f.numel(), _p(table), _stream()))
    return table


def qk_rope(q: torch.Tensor, k: Optional[torch.Tensor], table: Optional[torch.Tensor],
            positions: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
            k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
            q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Norms of queries and keys per head (where a weight fp32 [D] is given) and the rotation of their first
    2 * table.shape[1] dims, halves or (interleaved) adjacent pairs: bf16 q [T, Hq, D], k [T, Hk, D], any strides of
    multiples of 8 -> contiguous (q_out, k_out).  positions int32 [T] (None: 0, 1, ...)."""
    shape = q.shape
    T, Hq, D = shape
    dev = q.get_device()
    rope = _rope_desc(table, positions, T, q_weight, k_weight, D, eps, interleaved, dev)
    hq, hk, Hk, yk = _heads(q, "q", dev), None, 0, None
    yq = _rows(q_out, q, shape, "q_out", dev)
    if k is not None:
        shape = k.shape
        Hk = shape[1]
        if shape != (T, Hk, D):
            raise ValueError("k: [T, Hk, D] of q's T and D")
        hk, yk = _heads(k, "k", dev), _rows(k_out, k, shape, "k_out", dev)
    to_q, to_k = (yq, yk) if dev >= 0 else (q, k)  # (_refuse)
    rc = LIB.fq_qk_rope(hq, Hq, hk, Hk, rope, T, D, to_q.data_ptr(), None if to_k is None else to_k.data_ptr(), _stream_handle())
    if rc:
        _refuse(rc, dev)
    return yq, yk


def cache_append(cache: KVCache, page_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, max_new: int,
                 k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
                 table: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 interleaved: bool = False, q_out: Optional[torch.Tensor] = None, growth: int = 0) -> Optional[torch.Tensor]:
    """Appends the tokens of a ragged batch (rows q_start[b] .. q_start[b+1] - 1 of k, v [T, Hk, D] are the last ones of
    the kv_len[b] tokens of sequence b) to its pages: keys normed and rotated as by qk_rope, keys and values rounded to 8
    bits under a scale per page and head.  q [T, Hq, D] is normed and rotated in the same launch and returned.
    max_new: the most rows of a sequence.  positions: None for a token's place in its sequence.
    growth: percent that a page's scale grows at least, where it has to grow over earlier tokens.  Every growth rounds
    the earlier tokens again: a page filled token by token errs by up to half a step for each with 0 (2 steps for
    normal values, tens for values that keep rising a little), by 2.5 steps at most with 25."""
    shape = k.shape
    T, H, D = shape
    dev = k.get_device()
    desc, ch, P, cd = _cache_desc(cache, dev, growth)
    if H != ch or D != cd or v.shape != shape:
        raise ValueError("k, v: [T, heads, D] of the cache's heads and D")
    batch = _batch_desc(page_table, q_start, kv_len, max_new, page_table.shape[1] * P if page_table.dim() == 2 else 0, dev)
    y, Hq, hq = None, 0, None
    if q is not None:
        shape = q.shape
        Hq = shape[1]
        if shape != (T, Hq, D):
            raise ValueError("q: [T, Hq, D] of k's T and D")
        hq, y = _heads(q, "q", dev), _rows(q_out, q, shape, "q_out", dev)
    rope = _rope_desc(table, positions, T, q_weight, k_weight, D, eps, interleaved, dev)
    hk, hv = _heads(k, "k", dev), _heads(v, "v", dev)
    if dev < 0:
        raise ValueError("the tensors are on the host, not on a GPU")
    rc = LIB.fq_cache_append(desc, batch, hk, hv, hq, Hq, rope, T, None if y is None else y.data_ptr(), _stream_handle())
    if rc:
        _check(rc)
    return y


def cache_read(cache: KVCache, page_table: torch.Tensor, first: torch.Tensor, last: torch.Tensor, max_tokens: int,
               k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Tokens first[b] .. last[b] - 1 of every sequence as values: bf16 k, v [seqs, max_tokens, heads, D], zeros beyond."""
    dev = page_table.get_device()
    desc, H, _, D = _cache_desc(cache, dev)
    B, width = _table_shape(page_table, dev)
    shape = (B, max_tokens, H, D)
    if k_out is None and v_out is None:
        k_out, v_out = torch.empty((2, *shape), dtype=_BF16, device=page_table.device)
    else:
        given = v_out if k_out is None else k_out
        k_out, v_out = _rows(k_out, given, shape, "k_out", dev), _rows(v_out, given, shape, "v_out", dev)
    lo, hi = _index(first, B, "first", dev), _index(last, B, "last", dev)
    if dev < 0:
        raise ValueError("the tensors are on the host, not on a GPU")
    rc = LIB.fq_cache_read(desc, page_table.data_ptr(), width, lo, hi, B, max_tokens, k_out.data_ptr(), v_out.data_ptr(),
                           _stream_handle())
    if rc:
        _check(rc)
    return k_out, v_out


def cache_attention_workspace_bytes(T: int, Hq: int, Hk: int, D: int, seqs: int, max_new: int, max_kv: int) -> int:
    return int(LIB.fq_cache_attention_workspace_bytes(T, Hq, Hk, D, seqs, max_new, max_kv))


def cache_attention(q: torch.Tensor, cache: KVCache, page_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor,
                    max_new: int, max_kv: int, scale: Optional[float] = None, causal: bool = True,
                    ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(scale q k^T) v of a ragged batch of queries bf16 [T, Hq, D] over its sequences' tokens in the cache (see
    cache_append; append first) -> [T, Hq, D].  max_new, max_kv: the most rows and tokens of a sequence; scale: None for
    1/sqrt(D); causal: a row sees the tokens up to its own place, otherwise all kv_len[b]."""
    shape = q.shape
    T, Hq, D = shape
    dev = q.get_device()
    desc, H, _, cd = _cache_desc(cache, dev)
    if D != cd:
        raise ValueError("q: [T, Hq, D] of the cache's D")
    batch = _batch_desc(page_table, q_start, kv_len, max_new, max_kv, dev)
    hq, y = _heads(q, "q", dev), _rows(out, q, shape, "out", dev)
    if ws is None:
        ws = _scratch(LIB.fq_cache_attention_workspace_bytes(T, Hq, H, D, page_table.shape[0], max_new, max_kv), q.device)
    room, size = _room(ws, dev)
    to = y if dev >= 0 else q  # (_refuse)
    rc = LIB.fq_cache_attention(hq, Hq, T, desc, batch, D ** -0.5 if scale is None else scale, causal, to.data_ptr(), room, size,
                                _stream_handle())
    if rc:
        _refuse(rc, dev)
    return y


def cross_attention_workspace_bytes(B: int, Sq: int, Sk: int, Hq: int, Hk: int, D: int) -> int:
    return int(LIB.fq_cross_attention_workspace_bytes(B, Sq, Sk, Hq, Hk, D))


def cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, kv_len: Optional[torch.Tensor] = None,
                    key_mask: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                    ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(scale q k^T) v of queries bf16 [B, Sq, Hq, D] over an encoder's states k, v [B, Sk, Hk, D] (any strides of
    multiples of 8) -> [B, Sq, Hq, D].  kv_len int32 [B]: states in use; key_mask bool [B, Sk]: True = seen.  What lies in
    unseen places has no effect; a sample that sees nothing gives zeros."""
    shape, ks = q.shape, k.shape
    B, Sq, Hq, D = shape
    dev = q.get_device()
    _, Sk, Hk, _ = ks
    if ks != (B, Sk, Hk, D) or v.shape != ks:
        raise ValueError("k, v: [B, Sk, Hk, D] of q's B and D")
    mask = stride = 0
    if key_mask is not None:
        if (key_mask.dtype not in (torch.bool, torch.uint8) or key_mask.shape != (B, Sk)
                or (Sk > 1 and key_mask.stride(1) != 1)):
            raise ValueError("key_mask: bool [B, Sk] with unit stride of the last dim")
        if key_mask.get_device() != dev:
            raise _elsewhere("key_mask", key_mask, dev)
        mask, stride = key_mask.data_ptr(), key_mask.stride(0)
    hq, hk, hv, y = _heads(q, "q", dev), _heads(k, "k", dev), _heads(v, "v", dev), _rows(out, q, shape, "out", dev)
    if ws is None:
        ws = _scratch(LIB.fq_cross_attention_workspace_bytes(B, Sq, Sk, Hq, Hk, D), q.device)
    room, size = _room(ws, dev)
    to = y if dev >= 0 else q  # (_refuse)
    rc = LIB.fq_cross_attention(hq, hk, hv, _index(kv_len, B, "kv_len", dev) or None, mask or None, stride, B, Sq, Sk, Hq, Hk, D,
                                D ** -0.5 if scale is None else scale, to.data_ptr(), room, size, _stream_handle())
    if rc:
        _refuse(rc, dev)
    return y


# ---------------------------------------------------------------- microscaled 4-bit codes, and the norm before a projection

_U8 = torch.uint8


def _plain(t: torch.Tensor, dtype, shape, name: str, dev: int) -> int:
    """Address of a contiguous tensor of this type and shape."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous {str(dtype)[6:]} {list(shape)}")
    if t.get_device() != dev:
        raise _elsewhere(name, t, dev)
    return t.data_ptr()


def _matrix(t: torch.Tensor, dtype, shape, name: str, dev: int) -> Tuple[int, int]:
    """Address and row stride of rows with unit column stride."""
    ld, step = t.stride()
    if t.dtype is not dtype or t.shape != shape or (step != 1 and t.numel()):
        raise ValueError(f"{name}: {str(dtype)[6:]} {list(shape)} with unit column stride")
    if t.get_device() != dev:
        raise _elsewhere(name, t, dev)
    return t.data_ptr(), ld


def _new(like: torch.Tensor, shape, dtype) -> torch.Tensor:
    return like.new_empty(*shape, dtype=dtype) if type(like) is torch.Tensor else torch.empty(shape, dtype=dtype, device=like.device)


def _gpu_stream(dev: int) -> int:
    """The current stream, on which a call's kernels see the current device's tensors only."""
    if dev < 0:
        raise ValueError("the tensors are on the host, not on a GPU")
    here = torch._C._cuda_getDevice()
    if dev != here:
        raise ValueError(f"the tensors are on GPU {dev}, the current device is GPU {here}")
    return torch._C._cuda_getCurrentRawStream(here)


def _norm_args(x, weight, residual, sum_out, post_inv, M, K, dev):
    """The arguments that both norms begin with, and the stream of hidden states after the addition."""
    at, ld = _matrix(x, _BF16, (M, K), "x", dev)
    post = None if post_inv is None else _weight(post_inv, K, "post_inv", dev)
    w = _weight(weight, K, "weight", dev)
    if residual is None:
        if sum_out is not None:
            raise ValueError("sum_out needs a residual")
        return at, ld, None, 0, w, post, None, 0, x
    r, ldr = _matrix(residual, _BF16, (M, K), "residual", dev)
    if sum_out is None:
        total = _new(x, (M, K), _BF16)
        return at, ld, r, ldr, w, post, total.data_ptr(), K, total
    return (at, ld, r, ldr, w, post, *_matrix(sum_out, _BF16, (M, K), "sum_out", dev), sum_out)


def norm_quant(x: torch.Tensor, weight: torch.Tensor, b: int, bits: int, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
               clip_ratio: float = 1.0, post_inv: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None,
               out_codes: Optional[torch.Tensor] = None,
               out_delta: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The residual's addition, the root-mean-square norm with its gain `weight` fp32 [K] and the prologue's rotation and
    rounding, bf16 x, residual [M, K] -> (codes uint8 [M, K*bits/8], delta fp32 [M], the sum bf16 [M, K]; x where there is no
    residual).  sum_out may be x or the residual itself.  The codes are gemm's."""
    M, K = x.shape
    dev, width = x.get_device(), K * bits // 8
    at, ld, r, ldr, w, post, total, lds, states = _norm_args(x, weight, residual, sum_out, post_inv, M, K, dev)
    codes = _new(x, (M, width), _U8) if out_codes is None else out_codes
    delta = _new(x, (M,), _F32) if out_delta is None else out_delta
    c = codes.data_ptr() if out_codes is None else _plain(codes, _U8, (M, width), "out_codes", dev)
    d = delta.data_ptr() if out_delta is None else _plain(delta, _F32, (M,), "out_delta", dev)
    rc = LIB.fq_norm_quant(at, ld, r, ldr, w, eps, post, M, K, b, bits, clip_ratio, total, lds, c, d, _gpu_stream(dev))
    if rc:
        _check(rc)
    return codes, delta, states


def norm_mx_quant(x: torch.Tensor, weight: torch.Tensor, b: int = 1, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  post_inv: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None,
                  out_codes: Optional[torch.Tensor] = None,
                  out_scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """norm_quant with microscaled codes: (codes uint8 [M, K/2], scales uint8 [K/128, M, 4], the sum).  The codes are
    mx_gemm's."""
    M, K = x.shape
    dev = x.get_device()
    at, ld, r, ldr, w, post, total, lds, states = _norm_args(x, weight, residual, sum_out, post_inv, M, K, dev)
    codes, c, scales, s = _mx_out(x, M, K, out_codes, out_scales, dev)
    rc = LIB.fq_norm_mx_quant(at, ld, r, ldr, w, eps, post, M, K, b, total, lds, c, s, _gpu_stream(dev))
    if rc:
        _check(rc)
    return codes, scales, states


def _values_out(out: Optional[torch.Tensor], codes: torch.Tensor, M: int, K: int, dev: int):
    if out is None:
        out = _new(codes, (M, K), _BF16)
        return out, out.data_ptr(), K
    return (out, *_matrix(out, _BF16, (M, K), "out", dev))


def read_codes(codes: torch.Tensor, delta: torch.Tensor, bits: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Codes of fwht_quant or norm_quant, uint8 [M, K*bits/8] with delta fp32 [M], as values bf16 [M, K]: the fp32 product
    of code and delta, rounded."""
    if bits != 8 and bits != 4:
        raise ValueError("bits: 4 or 8")
    shape = codes.shape
    M, width = shape
    K, dev = width * 8 // bits, codes.get_device()
    c = _plain(codes, _I8 if codes.dtype is _I8 else _U8, shape, "codes", dev)
    d = _plain(delta, _F32, (M,), "delta", dev)
    out, at, ld = _values_out(out, codes, M, K, dev)
    rc = LIB.fq_read_codes(c, d, M, K, bits, at, ld, _gpu_stream(dev))
    if rc:
        _check(rc)
    return out


def _mx_out(x, M, K, codes, scales, dev):
    """Outputs of a microscaled rounding, the caller's or new ones, with their addresses."""
    if codes is None:
        codes = _new(x, (M, K // 2), _U8)
        c = codes.data_ptr()
    else:
        c = _plain(codes, _U8, (M, K // 2), "out_codes", dev)
    if scales is None:
        scales = _new(x, (K // 128, M, 4), _U8)
        return codes, c, scales, scales.data_ptr()
    return codes, c, scales, _plain(scales, _U8, (K // 128, M, 4), "out_scales", dev)


def mx_quant(x: torch.Tensor, b: int = 1, pre_mult: Optional[torch.Tensor] = None, post_mult: Optional[torch.Tensor] = None,
             out_codes: Optional[torch.Tensor] = None,
             out_scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows bf16 (tokens) or fp32 (weights) [M, K] through the folds and the block Hadamard, rounded to microscaled codes:
    (codes uint8 [M, K/2], scales uint8 [K/128, M, 4]).  Tokens: pre_mult = S^-1, post_mult = P^-1; weights: S and P."""
    shape = x.shape
    M, K = shape
    dev, f32 = x.get_device(), x.dtype is _F32
    at, ld = _matrix(x, _F32 if f32 else _BF16, shape, "x", dev)
    pre = None if pre_mult is None else _weight(pre_mult, K, "pre_mult", dev)
    post = None if post_mult is None else _weight(post_mult, K, "post_mult", dev)
    codes, c, scales, s = _mx_out(x, M, K, out_codes, out_scales, dev)
    rc = LIB.fq_mx_quant(at, f32, ld, pre, post, M, K, b, c, s, _gpu_stream(dev))
    if rc:
        _check(rc)
    return codes, scales


def _mx_codes(codes, scales, name, dev) -> Tuple[int, int, int, int]:
    """(M, K, address of the codes, of the scales) of microscaled rows."""
    shape = codes.shape
    M, half = shape
    return M, 2 * half, _plain(codes, _U8, shape, name, dev), _plain(scales, _U8, (half // 64, M, 4), name + "'s scales", dev)


def mx_read(codes: torch.Tensor, scales: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Microscaled codes as values: bf16 [M, K], exactly."""
    dev = codes.get_device()
    M, K, c, s = _mx_codes(codes, scales, "codes", dev)
    out, at, ld = _values_out(out, codes, M, K, dev)
    rc = LIB.fq_mx_read(c, s, M, K, at, ld, _gpu_stream(dev))
    if rc:
        _check(rc)
    return out


def mx_pack(codes: torch.Tensor) -> torch.Tensor:
    """Weight codes uint8 [N, K/2] in the product's order: uint8 [N/16, K/128, 4, 16, 16].  The scales stay as they are."""
    N, half = codes.shape
    dev = codes.get_device()
    c = _plain(codes, _U8, (N, half), "codes", dev)
    out = _new(codes, (N // 16, half // 64, 4, 16, 16), _U8)
    _check(LIB.fq_mx_pack(c, N, 2 * half, out.data_ptr(), _gpu_stream(dev)))
    return out


def mx_unpack(packed: torch.Tensor) -> torch.Tensor:
    """mx_pack's inverse."""
    n, ks = packed.shape[:2]
    dev = packed.get_device()
    p = _plain(packed, _U8, (n, ks, 4, 16, 16), "packed", dev)
    out = _new(packed, (16 * n, 64 * ks), _U8)
    _check(LIB.fq_mx_unpack(p, 16 * n, 128 * ks, out.data_ptr(), _gpu_stream(dev)))
    return out


def _mx_operands(w: torch.Tensor, scales: torch.Tensor, bias, out, like, M: int, K: int, dev: int):
    """(N, addresses of packed weights, their scales and the bias, the output, its address and row stride)."""
    n = w.shape[0]
    N = 16 * n
    at = _plain(w, _U8, (n, K // 128, 4, 16, 16), "w_packed", dev)
    s = _plain(scales, _U8, (K // 128, N, 4), "w_scales", dev)
    b = None if bias is None else _weight(bias, N, "bias", dev)
    if out is None:
        out = _new(like, (M, N), _BF16)
        return N, at, s, b, out, out.data_ptr(), N
    return (N, at, s, b, out, *_matrix(out, _BF16, (M, N), "out", dev))


@functools.lru_cache(4096)  # a call asks every time
def mx_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(LIB.fq_mx_gemm_workspace_bytes(M, N, K))


def mx_gemm(a_codes: torch.Tensor, a_scales: torch.Tensor, w_packed: torch.Tensor, w_scales: torch.Tensor,
            bias: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Product of microscaled tokens [M, K] and packed weights [N, K] (mx_pack), plus bias fp32 [N]: bf16 [M, N]."""
    dev = a_codes.get_device()
    M, K, a, sa = _mx_codes(a_codes, a_scales, "a_codes", dev)
    N, w, sw, b, out, y, ldy = _mx_operands(w_packed, w_scales, bias, out, a_codes, M, K, dev)
    stream = _gpu_stream(dev)
    if ws is None:
        ws = _scratch(mx_gemm_workspace_bytes(M, N, K), a_codes.device)
    room, size = _room(ws, dev)
    rc = LIB.fq_mx_gemm(a, sa, w, sw, b, y, ldy, M, N, K, room, size, stream)
    if rc:
        _check(rc)
    return out


@functools.lru_cache(4096)  # a call asks every time
def mx_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(LIB.fq_mx_linear_workspace_bytes(M, N, K))


def mx_linear(x: torch.Tensor, w_packed: torch.Tensor, w_scales: torch.Tensor, b: int = 1, smooth_inv: Optional[torch.Tensor] = None,
              post_inv: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """mx_quant of bf16 x [M, K], then mx_gemm: bf16 [M, N]."""
    shape = x.shape
    M, K = shape
    dev = x.get_device()
    at, ld = _matrix(x, _BF16, shape, "x", dev)
    pre = None if smooth_inv is None else _weight(smooth_inv, K, "smooth_inv", dev)
    post = None if post_inv is None else _weight(post_inv, K, "post_inv", dev)
    N, w, sw, bias_at, out, y, ldy = _mx_operands(w_packed, w_scales, bias, out, x, M, K, dev)
    stream = _gpu_stream(dev)
    if ws is None:
        ws = _scratch(mx_linear_workspace_bytes(M, N, K), x.device)
    room, size = _room(ws, dev)
    rc = LIB.fq_mx_linear(at, ld, pre, post, M, K, N, b, w, sw, bias_at, y, ldy, room, size, stream)
    if rc:
        _check(rc)
    return out


class MXLinear:
    """One projection with microscaled weights: w fp32 [N, K] folded, rounded and packed, kept on the device."""

    def __init__(self, w: torch.Tensor, b: int = 1, col_scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                 post_scale: Optional[torch.Tensor] = None):
        self.N, self.K = w.shape
        self.b, self.bias = b, bias
        codes, self.w_scales = mx_quant(w, b, col_scale, post_scale)
        self.w_packed = mx_pack(codes)

    def __call__(self, x: torch.Tensor, smooth_inv: Optional[torch.Tensor] = None, post_inv: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        return mx_linear(x, self.w_packed, self.w_scales, self.b, smooth_inv, post_inv, self.bias, ws, out)

    def product(self, codes: torch.Tensor, scales: torch.Tensor, ws: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The product alone, for tokens that norm_mx_quant or mx_quant rounded (several projections of one site)."""
        return mx_gemm(codes, scales, self.w_packed, self.w_scales, self.bias, ws, out)
