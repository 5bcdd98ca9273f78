"""ctypes binding of the C-ABI library (include/fedrag.h), one Python function per entry point.

Argument marshalling only: tensors are torch CUDA tensors used as device memory, the stream is torch's
current HIP stream.  Every step of the path runs in the library's kernels; there is no fallback: if the
library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
from operator import attrgetter, index
from typing import Optional

import torch  # noqa: F401  (imported before the library so that both share one HIP runtime)

from . import build as _build

OK, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_ALIAS, ERR_DEVICE = range(7)
F32, BF16, F16 = 0, 1, 2
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

STATIC_SCRATCH_BYTES = 16 << 20  # FEDRAG_STATIC_SCRATCH_BYTES

EXPORTS = ("fedrag_scramble_kv", "fedrag_scramble_q", "fedrag_partial_attn", "fedrag_partial_attn_static",
           "fedrag_partial_attn_workspace_bytes", "fedrag_partial_attn_shards",
           "fedrag_partial_attn_shards_workspace_bytes", "fedrag_lse_merge", "fedrag_unscramble", "fedrag_unscramble_merge",
           "fedrag_scramble_kv_structured", "fedrag_scramble_q_structured", "fedrag_unscramble_structured",
           "fedrag_local_attn", "fedrag_unpermute_lse", "fedrag_partial_attn_varlen", "fedrag_quantize_rows",
           "fedrag_dequantize_rows", "fedrag_scramble_kv_quantized", "fedrag_scramble_kv_structured_quantized",
           "fedrag_partial_attn_quantized", "fedrag_partial_attn_varlen_quantized", "fedrag_paged_map",
           "fedrag_paged_write", "fedrag_paged_attn", "fedrag_paged_attn_workspace_bytes", "fedrag_tree_map",
           "fedrag_paged_tree_attn", "fedrag_paged_tree_attn_workspace_bytes", "fedrag_tree_verify",
           "fedrag_tree_verify_workspace_bytes", "fedrag_paged_keep", "fedrag_paged_trim", "fedrag_invert_perm",
           "fedrag_validate_perm", "fedrag_status_string",
           "fedrag_version")

# what fedrag_paged_map's flags are the sum of
MAP_NO_PAGES, MAP_NO_COLUMNS, MAP_NO_ROWS, MAP_BAD_LENGTH = 1, 2, 4, 8
# fedrag_tree_map's flags of a request, fedrag_paged_trim's
TREE_BAD_PARENT, TREE_NO_WORDS = 1, 2
TRIM_NO_ROOM, TRIM_BAD_LENGTH = 1, 2
TREE_WORDS, KEEP_CACHES = 64, 64  # FEDRAG_TREE_WORDS, FEDRAG_KEEP_CACHES


class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("d_head", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class StructuredKey(ctypes.Structure):
    """fedrag_structured_key: host struct of four device pointers, [Hkv, d] each."""
    _fields_ = [("scale_in", ctypes.c_void_p), ("perm_in", ctypes.c_void_p), ("perm_out", ctypes.c_void_p),
                ("scale_out", ctypes.c_void_p)]


class PagedCache(ctypes.Structure):
    """fedrag_paged_cache: host struct of two device pointers and the pages' sizes."""
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("page_stride", ctypes.c_int64),
                ("page_tokens", ctypes.c_int32)]


class Rows(ctypes.Structure):
    """fedrag_rows: host struct of a device pointer and two strides, in elements."""
    _fields_ = [("data", ctypes.c_void_p), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64)]


class FedragError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib_path() -> str:
    return _build.LIB_PATH


def load() -> ctypes.CDLL:
    """Load libfedrag.so (built in-tree by paper_2605_25716_amd.build).  Raises if it is missing."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise FileNotFoundError(
                f"{path} not found: build it first (python -m paper_2605_25716_amd.build); "
                "this package has no fallback path")
        lib = ctypes.CDLL(path)
        vp, i64, i32, f32p = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
        sp = ctypes.POINTER(Shape)
        lib.fedrag_scramble_kv.argtypes = [sp, i64, vp, vp, vp, vp, vp, i32, vp, vp, vp]
        lib.fedrag_scramble_q.argtypes = [sp, i64, vp, vp, vp, vp, vp]
        lib.fedrag_partial_attn.argtypes = [sp, i64, i64, vp, vp, vp, ctypes.c_float, f32p, f32p, vp,
                                            ctypes.c_size_t, vp]
        lib.fedrag_local_attn.argtypes = lib.fedrag_partial_attn.argtypes
        lib.fedrag_partial_attn_static.argtypes = [sp, i64, i64, vp, vp, vp, ctypes.c_float, f32p, f32p, vp]
        lib.fedrag_partial_attn_shards.argtypes = [sp, i64, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64),
                                                   ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p),
                                                   vp, ctypes.c_float, f32p, f32p, vp, ctypes.c_size_t, vp]
        lib.fedrag_partial_attn_shards_workspace_bytes.argtypes = [sp, i64, ctypes.c_int32,
                                                                   ctypes.POINTER(ctypes.c_int64)]
        lib.fedrag_partial_attn_shards_workspace_bytes.restype = ctypes.c_size_t
        lib.fedrag_unscramble_merge.argtypes = [sp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.fedrag_partial_attn_varlen.argtypes = [sp, i64, i64, vp, vp, vp, vp, vp, ctypes.c_float, f32p, f32p, vp,
                                                   ctypes.c_size_t, vp]
        lib.fedrag_unpermute_lse.argtypes = [sp, i64, f32p, vp, f32p, vp]
        lib.fedrag_partial_attn_workspace_bytes.argtypes = [sp, i64, i64]
        lib.fedrag_partial_attn_workspace_bytes.restype = ctypes.c_size_t
        lib.fedrag_lse_merge.argtypes = [sp, i64, i32, f32p, f32p, f32p, f32p, vp]
        lib.fedrag_unscramble.argtypes = [sp, i64, f32p, f32p, vp, f32p, vp]
        kp = ctypes.POINTER(StructuredKey)
        lib.fedrag_scramble_kv_structured.argtypes = [sp, i64, vp, vp, kp, kp, vp, i32, vp, vp, vp]
        lib.fedrag_scramble_q_structured.argtypes = [sp, i64, vp, kp, vp, vp, vp]
        lib.fedrag_unscramble_structured.argtypes = [sp, i64, f32p, kp, vp, f32p, vp]
        lib.fedrag_quantize_rows.argtypes = [i64, i32, ctypes.c_int, i32, vp, vp, vp, vp]
        lib.fedrag_dequantize_rows.argtypes = [i64, i32, ctypes.c_int, i32, vp, vp, vp, vp]
        lib.fedrag_scramble_kv_quantized.argtypes = [sp, i64, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
        lib.fedrag_scramble_kv_structured_quantized.argtypes = [sp, i64, vp, vp, kp, kp, vp, i32, i32, vp, vp, vp, vp, vp]
        lib.fedrag_partial_attn_quantized.argtypes = [sp, i64, i64, vp, vp, vp, vp, vp, i32, ctypes.c_float, f32p, f32p,
                                                      vp, ctypes.c_size_t, vp]
        lib.fedrag_partial_attn_varlen_quantized.argtypes = [sp, i64, i64, vp, vp, vp, vp, vp, i32, vp, vp,
                                                             ctypes.c_float, f32p, f32p, vp, ctypes.c_size_t, vp]
        cp, rp = ctypes.POINTER(PagedCache), ctypes.POINTER(Rows)
        lib.fedrag_paged_map.argtypes = [i32, i64, i32, i64, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.fedrag_paged_write.argtypes = [sp, i64, rp, rp, vp, cp, vp]
        lib.fedrag_paged_attn.argtypes = [sp, i64, rp, cp, vp, i64, vp, vp, i64, i32, ctypes.c_float, f32p, f32p, vp,
                                          ctypes.c_size_t, vp]
        lib.fedrag_paged_attn_workspace_bytes.argtypes = [sp, i64, i64, i32, i64]
        lib.fedrag_paged_attn_workspace_bytes.restype = ctypes.c_size_t
        lib.fedrag_tree_map.argtypes = [i32, i64, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.fedrag_paged_tree_attn.argtypes = [sp, i64, rp, cp, vp, i64, vp, vp, vp, i32, i64, ctypes.c_float, f32p, f32p, vp,
                                               ctypes.c_size_t, vp]
        lib.fedrag_paged_tree_attn_workspace_bytes.argtypes = lib.fedrag_paged_attn_workspace_bytes.argtypes
        lib.fedrag_paged_tree_attn_workspace_bytes.restype = ctypes.c_size_t
        lib.fedrag_tree_verify.argtypes = [i32, i64, i64, i32, vp, vp, vp, vp, i64, vp, i64, vp, vp, i64, vp, vp, vp, vp,
                                           ctypes.c_size_t, vp]
        lib.fedrag_tree_verify_workspace_bytes.argtypes = [i32, i64, i32]
        lib.fedrag_tree_verify_workspace_bytes.restype = ctypes.c_size_t
        lib.fedrag_paged_keep.argtypes = [sp, i32, cp, vp, i64, vp, vp, vp, i64, vp, vp]
        lib.fedrag_paged_trim.argtypes = [i32, i32, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp]
        lib.fedrag_invert_perm.argtypes = [vp, i64, vp, vp]
        lib.fedrag_validate_perm.argtypes = [vp, i32, i64, vp, vp, vp]
        lib.fedrag_status_string.argtypes = [ctypes.c_int]
        lib.fedrag_status_string.restype = ctypes.c_char_p
        lib.fedrag_version.restype = ctypes.c_int
        for name in ("fedrag_scramble_kv", "fedrag_scramble_q", "fedrag_partial_attn", "fedrag_partial_attn_static",
                     "fedrag_partial_attn_shards", "fedrag_unscramble_merge", "fedrag_lse_merge",
                     "fedrag_unscramble", "fedrag_invert_perm", "fedrag_validate_perm", "fedrag_scramble_kv_structured",
                     "fedrag_scramble_q_structured", "fedrag_unscramble_structured", "fedrag_local_attn",
                     "fedrag_unpermute_lse", "fedrag_partial_attn_varlen", "fedrag_quantize_rows",
                     "fedrag_dequantize_rows", "fedrag_scramble_kv_quantized",
                     "fedrag_scramble_kv_structured_quantized", "fedrag_partial_attn_quantized",
                     "fedrag_partial_attn_varlen_quantized", "fedrag_paged_map", "fedrag_paged_write",
                     "fedrag_paged_attn", "fedrag_tree_map", "fedrag_paged_tree_attn", "fedrag_tree_verify",
                     "fedrag_paged_keep", "fedrag_paged_trim"):
            getattr(lib, name).restype = ctypes.c_int
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().fedrag_status_string(int(status)).decode()


def version() -> int:
    return int(load().fedrag_version())


def _check(status: int, where: str) -> None:
    if status != OK:
        raise FedragError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    """A tensor's device address (ctypes makes a pointer of the integer itself)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("the library works on device memory: pass CUDA tensors")
    if not t.is_contiguous():
        raise ValueError("tensors must be dense row-major (contiguous)")
    return t.data_ptr()


def _stream():
    # the current stream of the current device, as its handle: torch.cuda.current_stream() builds a Stream object by way
    # of a device lookup, which took 2 us of a 9 us call
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def make_shape(batch: int, n_q_heads: int, n_kv_heads: int, d_head: int, dtype) -> Shape:
    code = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    return Shape(batch, n_q_heads, n_kv_heads, d_head, code)


@functools.lru_cache(maxsize=256)
def _shape_ref(batch: int, n_q_heads: int, n_kv_heads: int, d_head: int, dtype):
    """A reference to the shape struct of these numbers, for the calls' `const fedrag_shape*` (read during the call
    only): small calls spend as long on building ctypes objects as on the device.  For sizes of tensors and numbers passed
    through `index`: the cache would take 8.0 for 8, which the struct refuses, and an integer tensor for itself whatever it
    holds by now."""
    return ctypes.byref(make_shape(batch, n_q_heads, n_kv_heads, d_head, dtype))


def _shape_ref_of_numbers(batch, n_q_heads, n_kv_heads, d_head, dtype):
    return _shape_ref(index(batch), index(n_q_heads), index(n_kv_heads), index(d_head),
                      dtype if isinstance(dtype, torch.dtype) else int(dtype))


def _shape_of(q_like: torch.Tensor, n_kv_heads: int, dtype=None) -> Shape:
    B, Hq, _, d = q_like.shape
    return make_shape(B, Hq, n_kv_heads, d, q_like.dtype if dtype is None else dtype)


# ----------------------------------------------------------------------------------------------- entry points
def fedrag_scramble_kv(K, V, phi_k, phi_v, perm_kv=None, n_q_heads: Optional[int] = None,
                       K_out=None, V_out=None):
    """K' = P_KV K Phi_KQ^{-T}, V' = P_KV V Phi_V for one shard.  K, V [B,Hkv,L,d]; perm_kv [n_perm,L] or [L]."""
    B, Hkv, L, d = K.shape
    shape = _shape_ref(B, index(n_q_heads or Hkv), Hkv, d, K.dtype)
    K_out = torch.empty_like(K) if K_out is None else K_out
    V_out = torch.empty_like(V) if V_out is None else V_out
    n_perm = 0
    if perm_kv is not None:
        n_perm = 1 if perm_kv.dim() == 1 else perm_kv.shape[0]
    st = load().fedrag_scramble_kv(shape, L, _ptr(K), _ptr(V), _ptr(phi_k), _ptr(phi_v),
                                   _ptr(perm_kv), n_perm, _ptr(K_out), _ptr(V_out), _stream())
    _check(st, "fedrag_scramble_kv")
    return K_out, V_out


def _workspace(workspace, like, query: str, *sizes):
    """(tensor or None, its bytes): the caller's, whose size the call itself checks, or one of the size that it asks for."""
    if workspace is None:
        need = int(getattr(load(), query)(*sizes))
        if need == 0:
            return None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
    return workspace, workspace.numel() * workspace.element_size()


def fedrag_scramble_q(Q, phi_q, perm_q=None, Q_out=None):
    """Q' = P_Q Q Phi_KQ.  Q [B,Hq,Lq,d]; phi_q [Hkv,d,d]."""
    B, Hq, Lq, d = Q.shape
    shape = _shape_ref(B, Hq, phi_q.shape[0], d, Q.dtype)
    Q_out = torch.empty_like(Q) if Q_out is None else Q_out
    st = load().fedrag_scramble_q(shape, Lq, _ptr(Q), _ptr(phi_q), _ptr(perm_q), _ptr(Q_out), _stream())
    _check(st, "fedrag_scramble_q")
    return Q_out


def fedrag_partial_attn_workspace_bytes(batch, n_q_heads, n_kv_heads, d_head, dtype, L_q, L_kv) -> int:
    shape = _shape_ref_of_numbers(batch, n_q_heads, n_kv_heads, d_head, dtype)
    return int(load().fedrag_partial_attn_workspace_bytes(shape, L_q, L_kv))


def fedrag_partial_attn(Qs, Ks, Vs, softmax_scale: Optional[float] = None, O_part=None, lse=None, workspace=None):
    """One shard's (O_i, lse_i).  Qs [B,Hq,Lq,d], Ks/Vs [B,Hkv,L,d] -> fp32 [B,Hq,Lq,d], fp32 [B,Hq,Lq]."""
    B, Hq, Lq, d = Qs.shape
    Hkv, L = Ks.shape[1], Ks.shape[2]
    shape = _shape_ref(B, Hq, Hkv, d, Qs.dtype)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O_part = torch.empty((B, Hq, Lq, d), dtype=torch.float32, device=Qs.device) if O_part is None else O_part
    lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=Qs.device) if lse is None else lse
    workspace, ws_bytes = _workspace(workspace, Qs, "fedrag_partial_attn_workspace_bytes", shape, Lq, L)
    st = load().fedrag_partial_attn(shape, Lq, L, _ptr(Qs), _ptr(Ks) if L > 0 else None,
                                    _ptr(Vs) if L > 0 else None, softmax_scale, _ptr(O_part),
                                    _ptr(lse), _ptr(workspace), ws_bytes, _stream())
    _check(st, "fedrag_partial_attn")
    return O_part, lse


def fedrag_partial_attn_static(Qs, Ks, Vs, O_part, lse, softmax_scale: Optional[float] = None):
    """fedrag_partial_attn without a workspace argument (the library's static scratch array); the caller passes the
    outputs, so that the call allocates nothing."""
    B, Hq, Lq, d = Qs.shape
    Hkv, L = Ks.shape[1], Ks.shape[2]
    shape = _shape_ref(B, Hq, Hkv, d, Qs.dtype)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    st = load().fedrag_partial_attn_static(shape, Lq, L, _ptr(Qs), _ptr(Ks) if L > 0 else None,
                                           _ptr(Vs) if L > 0 else None, softmax_scale, _ptr(O_part),
                                           _ptr(lse), _stream())
    _check(st, "fedrag_partial_attn_static")
    return O_part, lse


def fedrag_partial_attn_shards_workspace_bytes(batch, n_q_heads, n_kv_heads, d_head, dtype, L_q, L_kv_list) -> int:
    shape = _shape_ref_of_numbers(batch, n_q_heads, n_kv_heads, d_head, dtype)
    n = len(L_kv_list)
    Ls = (ctypes.c_int64 * n)(*[int(x) for x in L_kv_list])
    return int(load().fedrag_partial_attn_shards_workspace_bytes(shape, L_q, n, Ls))


def fedrag_partial_attn_shards(Qs, Ks_list, Vs_list, softmax_scale: Optional[float] = None, O=None, lse=None,
                               workspace=None):
    """Per-shard attention and its aggregation over the shards in one call.  Qs [B,Hq,Lq,d];
    Ks_list[i], Vs_list[i] [B,Hkv,L_i,d] -> fp32 [B,Hq,Lq,d], fp32 [B,Hq,Lq] over all shards' keys."""
    B, Hq, Lq, d = Qs.shape
    n = len(Ks_list)
    Hkv = Ks_list[0].shape[1]
    shape = _shape_ref(B, Hq, Hkv, d, Qs.dtype)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O = torch.empty((B, Hq, Lq, d), dtype=torch.float32, device=Qs.device) if O is None else O
    lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=Qs.device) if lse is None else lse
    Ls = (ctypes.c_int64 * n)(*[int(k.shape[2]) for k in Ks_list])
    Kp = (ctypes.c_void_p * n)(*[_ptr(k) if k.shape[2] > 0 else None for k in Ks_list])
    Vp = (ctypes.c_void_p * n)(*[_ptr(v) if v.shape[2] > 0 else None for v in Vs_list])
    workspace, ws_bytes = _workspace(workspace, Qs, "fedrag_partial_attn_shards_workspace_bytes", shape, Lq, n, Ls)
    st = load().fedrag_partial_attn_shards(shape, Lq, n, Ls, Kp, Vp, _ptr(Qs),
                                           softmax_scale, _ptr(O), _ptr(lse), _ptr(workspace),
                                           ws_bytes, _stream())
    _check(st, "fedrag_partial_attn_shards")
    return O, lse


def fedrag_partial_attn_varlen(Qs, Ks, Vs, kv_lens, softmax_scale: Optional[float] = None, O_part=None, lse=None,
                               workspace=None, q_lens=None):
    """fedrag_partial_attn over a padded batch: sequence b attends to its first kv_lens[b] keys.  kv_lens int32 [B]."""
    B, Hq, Lq, d = Qs.shape
    Hkv, L = Ks.shape[1], Ks.shape[2]
    if kv_lens.dtype != torch.int32 or kv_lens.shape != (B,):
        raise ValueError("kv_lens: int32 [B]")
    shape = _shape_ref(B, Hq, Hkv, d, Qs.dtype)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O_part = torch.empty((B, Hq, Lq, d), dtype=torch.float32, device=Qs.device) if O_part is None else O_part
    lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=Qs.device) if lse is None else lse
    workspace, ws_bytes = _workspace(workspace, Qs, "fedrag_partial_attn_workspace_bytes", shape, Lq, L)
    st = load().fedrag_partial_attn_varlen(shape, Lq, L, _ptr(Qs), _ptr(Ks) if L > 0 else None,
                                           _ptr(Vs) if L > 0 else None, _ptr(kv_lens), _ptr(q_lens),
                                           softmax_scale,
                                           _ptr(O_part), _ptr(lse), _ptr(workspace), ws_bytes, _stream())
    _check(st, "fedrag_partial_attn_varlen")
    return O_part, lse


def fedrag_partial_attn_quantized(Qs, K_codes, K_params, V_codes, V_params, bits: int,
                                  softmax_scale: Optional[float] = None, O_part=None, lse=None, workspace=None):
    """fedrag_partial_attn reading K', V' as transport-codec codes (any query count; 16-bit storage)."""
    B, Hq, Lq, d = Qs.shape
    Hkv, L = K_codes.shape[1], K_codes.shape[2]
    shape = _shape_ref(B, Hq, Hkv, d, Qs.dtype)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O_part = torch.empty((B, Hq, Lq, d), dtype=torch.float32, device=Qs.device) if O_part is None else O_part
    lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=Qs.device) if lse is None else lse
    workspace, ws_bytes = _workspace(workspace, Qs, "fedrag_partial_attn_workspace_bytes", shape, Lq, L)
    nz = L > 0
    st = load().fedrag_partial_attn_quantized(shape, Lq, L, _ptr(Qs), _ptr(K_codes) if nz else None,
                                              _ptr(K_params) if nz else None, _ptr(V_codes) if nz else None,
                                              _ptr(V_params) if nz else None, bits, softmax_scale,
                                              _ptr(O_part), _ptr(lse), _ptr(workspace), ws_bytes, _stream())
    _check(st, "fedrag_partial_attn_quantized")
    return O_part, lse


def fedrag_partial_attn_varlen_quantized(Qs, K_codes, K_params, V_codes, V_params, bits: int, kv_lens,
                                         softmax_scale: Optional[float] = None, O_part=None, lse=None, workspace=None,
                                         q_lens=None):
    """fedrag_partial_attn_varlen reading K', V' as transport-codec codes: sequence b attends to its first kv_lens[b]
    keys; q_lens (optional) gives the real query rows per sequence."""
    B, Hq, Lq, d = Qs.shape
    Hkv, L = K_codes.shape[1], K_codes.shape[2]
    if kv_lens.dtype != torch.int32 or kv_lens.shape != (B,):
        raise ValueError("kv_lens: int32 [B]")
    shape = _shape_ref(B, Hq, Hkv, d, Qs.dtype)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O_part = torch.empty((B, Hq, Lq, d), dtype=torch.float32, device=Qs.device) if O_part is None else O_part
    lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=Qs.device) if lse is None else lse
    workspace, ws_bytes = _workspace(workspace, Qs, "fedrag_partial_attn_workspace_bytes", shape, Lq, L)
    nz = L > 0
    st = load().fedrag_partial_attn_varlen_quantized(
        shape, Lq, L, _ptr(Qs), _ptr(K_codes) if nz else None, _ptr(K_params) if nz else None,
        _ptr(V_codes) if nz else None, _ptr(V_params) if nz else None, bits, _ptr(kv_lens), _ptr(q_lens),
        softmax_scale, _ptr(O_part), _ptr(lse), _ptr(workspace), ws_bytes, _stream())
    _check(st, "fedrag_partial_attn_varlen_quantized")
    return O_part, lse


def fedrag_local_attn(Q, K, V, softmax_scale: Optional[float] = None, O_part=None, lse=None, workspace=None):
    """The Inquirer's own part (Section 5.3): the Lq queries are the last Lq of the L local tokens, each sees itself
    and what comes before.  Q [B,Hq,Lq,d], K/V [B,Hkv,L,d] plaintext -> fp32 [B,Hq,Lq,d], fp32 [B,Hq,Lq]."""
    B, Hq, Lq, d = Q.shape
    Hkv, L = K.shape[1], K.shape[2]
    shape = _shape_ref(B, Hq, Hkv, d, Q.dtype)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O_part = torch.empty((B, Hq, Lq, d), dtype=torch.float32, device=Q.device) if O_part is None else O_part
    lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=Q.device) if lse is None else lse
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if Lq == 1:
        workspace, ws_bytes = _workspace(workspace, Q, "fedrag_partial_attn_workspace_bytes", shape, Lq, L)
    st = load().fedrag_local_attn(shape, Lq, L, _ptr(Q), _ptr(K) if L > 0 else None,
                                  _ptr(V) if L > 0 else None, softmax_scale, _ptr(O_part), _ptr(lse),
                                  _ptr(workspace), ws_bytes, _stream())
    _check(st, "fedrag_local_attn")
    return O_part, lse


def fedrag_unscramble_merge(O_scr, lse_scr, phi_v_inv, perm_q, O_local, lse_local, O_out=None, lse_out=None,
                            n_kv_heads: Optional[int] = None):
    """Dec of the remote result and its aggregation with the Inquirer's own partial, in one call."""
    B, Hq, Lq, d = O_scr.shape
    shape = _shape_ref(B, Hq, index(n_kv_heads or phi_v_inv.shape[0]), d, F32)
    O_out = torch.empty_like(O_scr) if O_out is None else O_out
    lse_out = torch.empty_like(lse_scr) if lse_out is None else lse_out
    st = load().fedrag_unscramble_merge(shape, Lq, _ptr(O_scr), _ptr(lse_scr), _ptr(phi_v_inv),
                                        _ptr(perm_q), _ptr(O_local), _ptr(lse_local), _ptr(O_out), _ptr(lse_out),
                                        _stream())
    _check(st, "fedrag_unscramble_merge")
    return O_out, lse_out


def fedrag_unpermute_lse(lse_scr, perm_q=None, lse_out=None):
    """lse_out[b,h,perm_q[i]] = lse_scr[b,h,i]: the log-sum-exps back in the query rows' own order."""
    B, Hq, Lq = lse_scr.shape
    shape = _shape_ref(B, Hq, Hq, 128, F32)
    lse_out = torch.empty_like(lse_scr) if lse_out is None else lse_out
    st = load().fedrag_unpermute_lse(shape, Lq, _ptr(lse_scr), _ptr(perm_q), _ptr(lse_out), _stream())
    _check(st, "fedrag_unpermute_lse")
    return lse_out


def fedrag_lse_merge(O_parts, lses, n_kv_heads: Optional[int] = None, O_out=None, lse_out=None):
    """Aggregation over shards.  O_parts fp32 [S,B,Hq,Lq,d], lses fp32 [S,B,Hq,Lq]."""
    S, B, Hq, Lq, d = O_parts.shape
    shape = _shape_ref(B, Hq, index(n_kv_heads or Hq), d, F32)
    O_out = torch.empty((B, Hq, Lq, d), dtype=torch.float32, device=O_parts.device) if O_out is None else O_out
    lse_out = torch.empty((B, Hq, Lq), dtype=torch.float32, device=O_parts.device) if lse_out is None else lse_out
    st = load().fedrag_lse_merge(shape, Lq, S, _ptr(O_parts), _ptr(lses), _ptr(O_out), _ptr(lse_out),
                                 _stream())
    _check(st, "fedrag_lse_merge")
    return O_out, lse_out


def fedrag_unscramble(O_scr, phi_v_inv, perm_q=None, O_out=None):
    """Dec: out[b,h,perm_q[i]] = O_scr[b,h,i] @ phi_v_inv[h // G].  O_scr fp32 [B,Hq,Lq,d]; phi_v_inv fp32 [Hkv,d,d]."""
    B, Hq, Lq, d = O_scr.shape
    shape = _shape_ref(B, Hq, phi_v_inv.shape[0], d, F32)
    O_out = torch.empty_like(O_scr) if O_out is None else O_out
    st = load().fedrag_unscramble(shape, Lq, _ptr(O_scr), _ptr(phi_v_inv), _ptr(perm_q), _ptr(O_out),
                                  _stream())
    _check(st, "fedrag_unscramble")
    return O_out


def _key(key) -> StructuredKey:
    """key = (scale_in fp32, perm_in int32, perm_out int32, scale_out fp32), CUDA tensors [Hkv, d]."""
    a, g1, g2, b = key
    if a.dtype != torch.float32 or b.dtype != torch.float32 or g1.dtype != torch.int32 or g2.dtype != torch.int32:
        raise ValueError("structured key: scales are fp32, permutations int32")
    if not (a.shape == g1.shape == g2.shape == b.shape and a.dim() == 2):
        raise ValueError("structured key: four [Hkv, d] arrays")
    return StructuredKey(_ptr(a), _ptr(g1), _ptr(g2), _ptr(b))


def fedrag_scramble_kv_structured(K, V, key_k, key_v, perm_kv=None, n_q_heads: Optional[int] = None,
                                  K_out=None, V_out=None):
    """fedrag_scramble_kv with Phi_KQ^{-T} and Phi_V given as S1 P1 H P2 S2 factors (Section 4.2)."""
    B, Hkv, L, d = K.shape
    if key_k[0].shape != (Hkv, d) or key_v[0].shape != (Hkv, d):
        raise ValueError("structured key does not match [Hkv, d]")
    shape = _shape_ref(B, index(n_q_heads or Hkv), Hkv, d, K.dtype)
    K_out = torch.empty_like(K) if K_out is None else K_out
    V_out = torch.empty_like(V) if V_out is None else V_out
    n_perm = 0
    if perm_kv is not None:
        n_perm = 1 if perm_kv.dim() == 1 else perm_kv.shape[0]
    kk, kv = _key(key_k), _key(key_v)
    st = load().fedrag_scramble_kv_structured(shape, L, _ptr(K), _ptr(V), ctypes.byref(kk),
                                              ctypes.byref(kv), _ptr(perm_kv), n_perm, _ptr(K_out), _ptr(V_out),
                                              _stream())
    _check(st, "fedrag_scramble_kv_structured")
    return K_out, V_out


def fedrag_scramble_q_structured(Q, key_q, perm_q=None, Q_out=None):
    B, Hq, Lq, d = Q.shape
    if key_q[0].dim() != 2 or key_q[0].shape[1] != d:
        raise ValueError("structured key does not match [Hkv, d]")
    shape = _shape_ref(B, Hq, key_q[0].shape[0], d, Q.dtype)
    Q_out = torch.empty_like(Q) if Q_out is None else Q_out
    kq = _key(key_q)
    st = load().fedrag_scramble_q_structured(shape, Lq, _ptr(Q), ctypes.byref(kq), _ptr(perm_q),
                                             _ptr(Q_out), _stream())
    _check(st, "fedrag_scramble_q_structured")
    return Q_out


def fedrag_unscramble_structured(O_scr, key_v_inv, perm_q=None, O_out=None):
    B, Hq, Lq, d = O_scr.shape
    if key_v_inv[0].dim() != 2 or key_v_inv[0].shape[1] != d:
        raise ValueError("structured key does not match [Hkv, d]")
    shape = _shape_ref(B, Hq, key_v_inv[0].shape[0], d, F32)
    O_out = torch.empty_like(O_scr) if O_out is None else O_out
    kv = _key(key_v_inv)
    st = load().fedrag_unscramble_structured(shape, Lq, _ptr(O_scr), ctypes.byref(kv), _ptr(perm_q),
                                             _ptr(O_out), _stream())
    _check(st, "fedrag_unscramble_structured")
    return O_out


def fedrag_quantize_rows(X, bits: int, codes=None, params=None):
    """Transport codec (Section 7.5), per row of the last dimension.  X [..., d] -> (codes uint8 [..., d*bits/8],
    params fp32 [..., 2] = (scale, lo))."""
    d = X.shape[-1]
    n = X.numel() // d
    codes = torch.empty(X.shape[:-1] + (d * bits // 8,), dtype=torch.uint8, device=X.device) if codes is None else codes
    params = torch.empty(X.shape[:-1] + (2,), dtype=torch.float32, device=X.device) if params is None else params
    st = load().fedrag_quantize_rows(n, d, _DTYPES[X.dtype], bits, _ptr(X), _ptr(codes), _ptr(params), _stream())
    _check(st, "fedrag_quantize_rows")
    return codes, params


def fedrag_dequantize_rows(codes, params, bits: int, dtype, X_out=None):
    """Inverse map: codes uint8 [..., d*bits/8], params fp32 [..., 2] -> X [..., d] of `dtype`."""
    d = codes.shape[-1] * 8 // bits
    n = codes.numel() // codes.shape[-1]
    X_out = torch.empty(codes.shape[:-1] + (d,), dtype=dtype, device=codes.device) if X_out is None else X_out
    st = load().fedrag_dequantize_rows(n, d, _DTYPES[dtype], bits, _ptr(codes), _ptr(params), _ptr(X_out), _stream())
    _check(st, "fedrag_dequantize_rows")
    return X_out


def fedrag_scramble_kv_quantized(K, V, phi_k, phi_v, perm_kv, bits: int, n_q_heads: Optional[int] = None,
                                 structured: bool = False, out=None):
    """Enc of a KV shard with the transport codec as epilogue.  phi_k / phi_v: dense matrices, or structured keys
    with structured=True.  Returns (K_codes, K_params, V_codes, V_params)."""
    B, Hkv, L, d = K.shape
    shape = _shape_ref(B, index(n_q_heads or Hkv), Hkv, d, K.dtype)
    mk_c = lambda: torch.empty((B, Hkv, L, d * bits // 8), dtype=torch.uint8, device=K.device)
    mk_p = lambda: torch.empty((B, Hkv, L, 2), dtype=torch.float32, device=K.device)
    Kc, Kp, Vc, Vp = (mk_c(), mk_p(), mk_c(), mk_p()) if out is None else out
    n_perm = 0
    if perm_kv is not None:
        n_perm = 1 if perm_kv.dim() == 1 else perm_kv.shape[0]
    if structured:
        kk, kv = _key(phi_k), _key(phi_v)
        st = load().fedrag_scramble_kv_structured_quantized(shape, L, _ptr(K), _ptr(V), ctypes.byref(kk),
                                                            ctypes.byref(kv), _ptr(perm_kv), n_perm, bits, _ptr(Kc),
                                                            _ptr(Kp), _ptr(Vc), _ptr(Vp), _stream())
    else:
        st = load().fedrag_scramble_kv_quantized(shape, L, _ptr(K), _ptr(V), _ptr(phi_k), _ptr(phi_v),
                                                 _ptr(perm_kv), n_perm, bits, _ptr(Kc), _ptr(Kp), _ptr(Vc), _ptr(Vp),
                                                 _stream())
    _check(st, "fedrag_scramble_kv_quantized")
    return Kc, Kp, Vc, Vp


# ------------------------------------------------------------------------------------------- the paged cache
# Small calls spend more time here than on the device, so what is checked is checked once, in one expression per tensor, and
# put into words only when it fails (a call over one request's 192 tokens: 9.4 us of host time, 13.0 with a function per check).
def _device(t) -> int:
    """The index of the tensor's device, which has to be the current one: the call goes to its current stream."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError("the library works on device memory: pass CUDA tensors")
    if dev != torch.cuda.current_device():
        raise ValueError(f"the tensors are on device {dev}, which is not the current one")
    return dev


def _refuse(name, t, dtype, dev, what):
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on the device of the others")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: {dtype}, not {t.dtype}")
    raise ValueError(f"{name}: {what}, dense, not {list(t.shape)} with strides {list(t.stride())}")


def _values(name, t, dtype, dev, least):
    """The address of a dense tensor of at least `least` values."""
    if t.get_device() != dev or t.dtype is not dtype or t.numel() < least or not t.is_contiguous():
        _refuse(name, t, dtype, dev, f"at least {least} values")
    return t.data_ptr()


def _exactly(name, t, dtype, dev, shape):
    if t.get_device() != dev or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _refuse(name, t, dtype, dev, f"shape {list(shape)}")
    return t.data_ptr()


def _rows(name, X, dtype, dev):
    """(H, T, d) and the struct of rows [H, T, d] or [1, H, T, d] of any strides but the last one's: for rows kept [T, H, d] pass
    X.transpose(0, 1)."""
    shape, stride = X.shape, X.stride()
    if len(shape) == 4 and shape[0] == 1:
        shape, stride = shape[1:], stride[1:]
    if len(shape) != 3 or X.get_device() != dev or X.dtype is not dtype or (stride[2] != 1 and shape[2] > 1):
        if len(shape) == 3 and X.get_device() == dev and X.dtype is dtype:
            raise ValueError(f"{name}: the channels of a row have to lie side by side")
        _refuse(name, X, dtype, dev, "[H, T, d] or [1, H, T, d]")
    H, T, d = shape
    # (the stride of a dimension of one entry says nothing)
    return (H, T, d), ctypes.byref(Rows(X.data_ptr(), stride[0] if H > 1 else 0, stride[1] if T > 1 else 0))


@functools.lru_cache(maxsize=64)
def _page_stride(shape, stride) -> int:
    if len(shape) != 4:
        raise ValueError("K_pages, V_pages: [n_pages, Hkv, page_tokens, d]")
    n, H, P, d = shape
    if any(size > 1 and have != want for have, size, want in ((stride[1], H, P * d), (stride[2], P, d), (stride[3], d, 1))):
        raise ValueError("a page has to be dense: [Hkv, page_tokens, d] without gaps")
    if n > 1 and stride[0] == 0:  # (which to the library means that the pages lie side by side)
        raise ValueError("K_pages, V_pages: every page has memory of its own, not one that is expanded")
    return stride[0] if n > 1 else 0


def _pages(K_pages, V_pages, dev):
    shape, stride, dtype = K_pages.shape, K_pages.stride(), K_pages.dtype
    if V_pages.shape != shape or V_pages.stride() != stride or V_pages.dtype is not dtype or V_pages.get_device() != dev:
        raise ValueError("K_pages and V_pages: alike in shape, type, strides and device")
    page_stride = _page_stride(shape, stride)
    return shape, ctypes.byref(PagedCache(K_pages.data_ptr(), V_pages.data_ptr(), shape[0], page_stride, shape[2]))


def fedrag_paged_map(cached_lens, new_lens, block_table, free_pages, free_count, page_tokens: int, n_rows: int, q_start=None,
                     kv_lens=None, slots=None, positions=None, free_left=None, flags=None):
    """Plans a step over the paged cache from the requests' lengths: (q_start int32 [B+1], kv_lens int32 [B], slots int64
    [n_rows], positions int32 [n_rows], free_left int32 [1], flags int32 [1]); new pages are taken from the top of the stack
    free_pages[:free_count] and entered in block_table int32 [B, max_pages], in place.  kv_lens may be cached_lens and
    free_left may be free_count: the state then advances in place.  flags: 0 or a sum of MAP_*."""
    if block_table.dim() != 2:
        raise ValueError("block_table: int32 [B, max_pages]")
    dev, i32 = _device(block_table), torch.int32
    (B, columns), n_rows, page_tokens = block_table.shape, index(n_rows), index(page_tokens)
    if n_rows < 0:
        raise ValueError("n_rows is not negative")
    new = lambda n, dt=i32: torch.empty(n, dtype=dt, device=block_table.device)  # noqa: E731
    q_start = new(B + 1) if q_start is None else q_start
    kv_lens = new(B) if kv_lens is None else kv_lens
    slots = new(n_rows, torch.int64) if slots is None else slots
    positions = new(n_rows) if positions is None else positions
    free_left = new(1) if free_left is None else free_left
    flags = new(1) if flags is None else flags
    st = load().fedrag_paged_map(
        B, n_rows, page_tokens, columns, _exactly("cached_lens", cached_lens, i32, dev, (B,)),
        _exactly("new_lens", new_lens, i32, dev, (B,)), _values("free_pages", free_pages, i32, dev, 0), free_pages.numel(),
        _values("free_count", free_count, i32, dev, 1), _exactly("block_table", block_table, i32, dev, (B, columns)),
        _values("q_start", q_start, i32, dev, B + 1), _exactly("kv_lens", kv_lens, i32, dev, (B,)),
        _values("slots", slots, torch.int64, dev, n_rows), _values("positions", positions, i32, dev, n_rows),
        _values("free_left", free_left, i32, dev, 1), _values("flags", flags, i32, dev, 1), torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_paged_map")
    return q_start, kv_lens, slots, positions, free_left, flags


def fedrag_paged_write(K, V, slots, K_pages, V_pages):
    """Rows K, V ([Hkv, T, d] or [1, Hkv, T, d], any strides) into the pages [n_pages, Hkv, page_tokens, d], row t to slots[t]
    (int64 [T]); rows whose slot lies outside the pages are left out."""
    dev, dtype = _device(K_pages), K_pages.dtype
    shape, cache = _pages(K_pages, V_pages, dev)
    of_k, rk = _rows("K", K, dtype, dev)
    of_v, rv = _rows("V", V, dtype, dev)
    H, T, d = of_k
    if of_v != of_k or H != shape[1] or d != shape[3]:
        raise ValueError("K, V [Hkv, T, d] and the pages [n_pages, Hkv, page_tokens, d] do not match")
    st = load().fedrag_paged_write(_shape_ref(1, H, H, d, dtype), T, rk, rv, _values("slots", slots, torch.int64, dev, T), cache,
                                   torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_paged_write")
    return K_pages, V_pages


def fedrag_paged_attn_workspace_bytes(batch, n_q_heads, n_kv_heads, d_head, dtype, n_rows, max_pages, page_tokens, max_q_len) -> int:
    """Bytes for one call of these sizes (more rows can need less); 69 MiB are enough for any on 256 compute units."""
    shape = _shape_ref_of_numbers(batch, n_q_heads, n_kv_heads, d_head, dtype)
    return int(load().fedrag_paged_attn_workspace_bytes(shape, n_rows, max_pages, page_tokens, max_q_len))


@functools.lru_cache(maxsize=256)
def _paged_need(dev, *sizes) -> int:  # (of one device the answer is always the same)
    return fedrag_paged_attn_workspace_bytes(*sizes)


def fedrag_paged_attn(Q, K_pages, V_pages, block_table, q_start, kv_lens, max_q_len: int = 0, causal: bool = True,
                      softmax_scale: Optional[float] = None, O_part=None, lse=None, workspace=None):
    """A step's rows over the paged cache.  Q [Hq, T, d] or [1, Hq, T, d], any strides; request b's rows are
    q_start[b] .. q_start[b+1]-1 and see its first kv_lens[b] tokens, causal: up to themselves.  -> fp32 [1, Hq, T, d],
    fp32 [1, Hq, T]; rows behind the last request are not written.  max_q_len: the most rows of a request, 0 if not known
    (speed only)."""
    dev, dtype, i32, f32 = _device(K_pages), K_pages.dtype, torch.int32, torch.float32
    (_, Hkv, P, dk), cache = _pages(K_pages, V_pages, dev)
    (Hq, T, d), rq = _rows("Q", Q, dtype, dev)
    if d != dk:
        raise ValueError("Q [Hq, T, d] and the pages [n_pages, Hkv, page_tokens, d] do not match")
    if block_table.dim() != 2:
        raise ValueError("block_table: int32 [B, max_pages]")
    B, columns = block_table.shape
    max_q_len = index(max_q_len)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O_part = torch.empty((1, Hq, T, d), dtype=f32, device=Q.device) if O_part is None else O_part
    lse = torch.empty((1, Hq, T), dtype=f32, device=Q.device) if lse is None else lse
    if workspace is None:
        ws, ws_bytes = None, _paged_need(dev, B, Hq, Hkv, d, dtype, T, columns, P, max_q_len)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=Q.device)
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _values("workspace", workspace, workspace.dtype, dev, 0), workspace.numel() * workspace.element_size()
    st = load().fedrag_paged_attn(
        _shape_ref(B, Hq, Hkv, d, dtype), T, rq, cache, _exactly("block_table", block_table, i32, dev, (B, columns)), columns,
        _values("q_start", q_start, i32, dev, B + 1), _exactly("kv_lens", kv_lens, i32, dev, (B,)), max_q_len, 1 if causal else 0,
        softmax_scale, _values("O_part", O_part, f32, dev, Hq * T * d), _values("lse", lse, f32, dev, Hq * T), ws, ws_bytes,
        torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_paged_attn")
    return O_part, lse


def fedrag_tree_map(parents, q_start, kv_lens, mask_words: int, tree_mask=None, positions=None, flags=None):
    """Masks and positions of a drafted step's rows from the nodes' parents (int32 [n_rows], indices within the request, -1 for none):
    (tree_mask int64 [n_rows, mask_words], positions int32 [n_rows], flags int32 [B]: 0 or a sum of TREE_* for each request).
    Bit j % 64 of a row's word j / 64: node j is the row's own or an ancestor."""
    dev, i32 = _device(parents), torch.int32
    n_rows, B, mask_words = parents.numel(), kv_lens.numel(), index(mask_words)
    if mask_words < 1:
        raise ValueError("mask_words: at least one for every 64 nodes")
    new = lambda *n, dt=i32: torch.empty(n, dtype=dt, device=parents.device)  # noqa: E731
    tree_mask = new(n_rows, mask_words, dt=torch.int64) if tree_mask is None else tree_mask
    positions = new(n_rows) if positions is None else positions
    flags = new(B) if flags is None else flags
    st = load().fedrag_tree_map(
        B, n_rows, mask_words, _values("q_start", q_start, i32, dev, B + 1), _values("kv_lens", kv_lens, i32, dev, B),
        _values("parents", parents, i32, dev, n_rows), _exactly("tree_mask", tree_mask, torch.int64, dev, (n_rows, mask_words)),
        _values("positions", positions, i32, dev, n_rows), _values("flags", flags, i32, dev, B), torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_tree_map")
    return tree_mask, positions, flags


def fedrag_paged_tree_attn_workspace_bytes(batch, n_q_heads, n_kv_heads, d_head, dtype, n_rows, max_pages, page_tokens, max_q_len) -> int:
    """Bytes for one call of these sizes; 73 MiB are enough for any on 256 compute units."""
    shape = _shape_ref_of_numbers(batch, n_q_heads, n_kv_heads, d_head, dtype)
    return int(load().fedrag_paged_tree_attn_workspace_bytes(shape, n_rows, max_pages, page_tokens, max_q_len))


@functools.lru_cache(maxsize=256)
def _tree_need(dev, *sizes) -> int:
    return fedrag_paged_tree_attn_workspace_bytes(*sizes)


def fedrag_paged_tree_attn(Q, K_pages, V_pages, block_table, q_start, kv_lens, tree_mask, max_q_len: int = 0,
                           softmax_scale: Optional[float] = None, O_part=None, lse=None, workspace=None):
    """fedrag_paged_attn with a mask for each row: a request's rows q_start[b] .. q_start[b+1]-1 are the last of its kv_lens[b] tokens; a
    row sees all tokens before them, and of them those whose bit is set in its words of tree_mask (int64 [T, words], as
    fedrag_tree_map makes them)."""
    dev, dtype, i32, f32 = _device(K_pages), K_pages.dtype, torch.int32, torch.float32
    (_, Hkv, P, dk), cache = _pages(K_pages, V_pages, dev)
    (Hq, T, d), rq = _rows("Q", Q, dtype, dev)
    if d != dk:
        raise ValueError("Q [Hq, T, d] and the pages [n_pages, Hkv, page_tokens, d] do not match")
    if block_table.dim() != 2:
        raise ValueError("block_table: int32 [B, max_pages]")
    if tree_mask.dim() != 2:
        raise ValueError("tree_mask: int64 [T, words]")
    (B, columns), words = block_table.shape, tree_mask.shape[1]
    max_q_len = index(max_q_len)
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    O_part = torch.empty((1, Hq, T, d), dtype=f32, device=Q.device) if O_part is None else O_part
    lse = torch.empty((1, Hq, T), dtype=f32, device=Q.device) if lse is None else lse
    if workspace is None:
        ws, ws_bytes = None, _tree_need(dev, B, Hq, Hkv, d, dtype, T, columns, P, max_q_len)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=Q.device)
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _values("workspace", workspace, workspace.dtype, dev, 0), workspace.numel() * workspace.element_size()
    st = load().fedrag_paged_tree_attn(
        _shape_ref(B, Hq, Hkv, d, dtype), T, rq, cache, _exactly("block_table", block_table, i32, dev, (B, columns)), columns,
        _values("q_start", q_start, i32, dev, B + 1), _exactly("kv_lens", kv_lens, i32, dev, (B,)),
        _exactly("tree_mask", tree_mask, torch.int64, dev, (T, words)), words, max_q_len, softmax_scale,
        _values("O_part", O_part, f32, dev, Hq * T * d), _values("lse", lse, f32, dev, Hq * T), ws, ws_bytes,
        torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_paged_tree_attn")
    return O_part, lse


def fedrag_tree_verify_workspace_bytes(batch: int, vocab: int, dtype) -> int:
    """Bytes for one call of these sizes; none for rows of up to 128 KiB."""
    code = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    return int(load().fedrag_tree_verify_workspace_bytes(index(batch), index(vocab), code))


@functools.lru_cache(maxsize=256)
def _verify_need(*sizes) -> int:  # (the same on every device)
    return fedrag_tree_verify_workspace_bytes(*sizes)


def _vocab_rows(name, X, dtype, dev, n_rows, vocab):
    """(address, elements from a row to the next) of [n_rows, vocab] with any row stride that is not smaller."""
    if X.get_device() != dev or X.dtype is not dtype or X.shape != (n_rows, vocab):
        _refuse(name, X, dtype, dev, f"shape {[n_rows, vocab]}")
    if (vocab > 1 and X.stride(1) != 1) or (n_rows > 1 and X.stride(0) < vocab):
        raise ValueError(f"{name}: the values of a row have to lie side by side, and rows apart")
    return X.data_ptr(), X.stride(0) if n_rows > 1 else vocab


def fedrag_tree_verify(target, tokens, parents, q_start, u, u_next, draft=None, max_kept: int = 0, kept=None, n_kept=None,
                       next_token=None, workspace=None):
    """The walk over a drafted step's trees: (kept int32 [B, max_kept]: the accepted nodes of each request, node 0 first; n_kept int32
    [B]; next_token int32 [B]).  target [n_rows, vocab]: the probabilities that follow each node; draft: those that its children were
    drawn from, or None if they were not drawn; tokens, parents int32 [n_rows]; u float64 [n_rows], u_next float64 [B]: uniform in
    [0, 1).  max_kept: 16 if neither it nor kept is given."""
    dev, i32, f64 = _device(target), torch.int32, torch.float64
    if target.dim() != 2 or target.dtype not in _DTYPES:
        raise ValueError("target: [n_rows, vocab] in fp32, bf16 or fp16")
    (n_rows, vocab), B = target.shape, u_next.numel()
    new = lambda *n: torch.empty(n, dtype=i32, device=target.device)  # noqa: E731
    kept = new(B, index(max_kept) or 16) if kept is None else kept
    if kept.dim() != 2:
        raise ValueError("kept: int32 [B, max_kept]")
    columns = kept.shape[1]
    if max_kept and index(max_kept) != columns:
        raise ValueError("max_kept is the number of kept's columns")
    n_kept = new(B) if n_kept is None else n_kept
    next_token = new(B) if next_token is None else next_token
    target_at, target_stride = _vocab_rows("target", target, target.dtype, dev, n_rows, vocab)
    draft_at, draft_stride = (None, 0) if draft is None else _vocab_rows("draft", draft, target.dtype, dev, n_rows, vocab)
    if workspace is None:
        ws, ws_bytes = None, _verify_need(B, vocab, target.dtype)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=target.device)
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _values("workspace", workspace, workspace.dtype, dev, 0), workspace.numel() * workspace.element_size()
    st = load().fedrag_tree_verify(
        B, n_rows, vocab, _DTYPES[target.dtype], _values("q_start", q_start, i32, dev, B + 1), _values("parents", parents, i32, dev, n_rows),
        _values("tokens", tokens, i32, dev, n_rows), target_at, target_stride, draft_at, draft_stride, _values("u", u, f64, dev, n_rows),
        _values("u_next", u_next, f64, dev, B), columns, _exactly("kept", kept, i32, dev, (B, columns)),
        _values("n_kept", n_kept, i32, dev, B), _values("next_token", next_token, i32, dev, B), ws, ws_bytes,
        torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_tree_verify")
    return kept, n_kept, next_token


_size, _strides, _dense = torch.Tensor.size, torch.Tensor.stride, torch.Tensor.is_contiguous
_address, _index = torch.Tensor.data_ptr, torch.Tensor.get_device
_dtype = attrgetter("dtype")


@functools.lru_cache(maxsize=64)
def _cache_structs(n) -> struct.Struct:
    """An array of n fedrag_paged_cache."""
    return struct.Struct("@" + "PPqqi4x" * n)


def fedrag_paged_keep(caches, block_table, q_start, kv_lens, kept, n_kept):
    """Moves the K, V of the rows that stay to the front of each request's rows, in place, in every one of the caches, a list of (K_pages,
    V_pages) of one shape and type but for their numbers of pages.  kept int32 [B, max_kept], rising; n_kept int32 [B]."""
    if not caches:
        raise ValueError("caches: a list of (K_pages, V_pages)")
    first, i32 = caches[0][0], torch.int32
    dev, dtype = _device(first), first.dtype
    # All tensors in one sweep of each property (a loop in Python over 32 layers took 40 us, the launch takes 6).
    K, V = zip(*caches)
    tensors, n = K + V, len(K)
    shapes = list(map(_size, tensors))
    if all(map(_dense, tensors)):
        page_strides = [0] * n
    else:
        strides = list(map(_strides, tensors))
        page_strides = [_page_stride(*x) for x in zip(shapes, strides[:n])] if strides[:n] == strides[n:] else []
    if (not page_strides or shapes[:n] != shapes[n:] or (shapes.count(shapes[0]) != 2 * n and any(x[1:] != shapes[0][1:] for x in shapes))
            or len(shapes[0]) != 4 or set(map(_dtype, tensors)) != {dtype} or set(map(_index, tensors)) != {dev}):
        raise ValueError("caches: K_pages and V_pages [n_pages, Hkv, page_tokens, d], alike in shape, type, strides and device, and all of them "
                         "but for n_pages")
    numbers = [shapes[0][2]] * (5 * n)
    numbers[0::5], numbers[1::5] = map(_address, K), map(_address, V)
    numbers[2::5], numbers[3::5] = [x[0] for x in shapes[:n]], page_strides
    structs = _cache_structs(n).pack(*numbers)
    if block_table.dim() != 2 or kept.dim() != 2:
        raise ValueError("block_table: int32 [B, max_pages], kept: int32 [B, max_kept]")
    (B, columns), (_, H, _, d), most = block_table.shape, first.shape, kept.shape[1]
    st = load().fedrag_paged_keep(
        _shape_ref(B, H, H, d, dtype), len(caches), ctypes.cast(structs, ctypes.POINTER(PagedCache)), _exactly("block_table", block_table, i32, dev, (B, columns)), columns,
        _values("q_start", q_start, i32, dev, B + 1), _exactly("kv_lens", kv_lens, i32, dev, (B,)), _exactly("kept", kept, i32, dev, (B, most)),
        most, _exactly("n_kept", n_kept, i32, dev, (B,)), torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_paged_keep")
    return caches


def fedrag_paged_trim(kv_lens, n_kept, block_table, free_pages, free_count, page_tokens: int, q_start=None, lens_out=None, free_left=None,
                      flags=None):
    """What is left of the requests: (lens_out int32 [B], free_left int32 [1], flags int32 [1]).  Request b keeps kv_lens[b] - n + n_kept[b]
    of its tokens, n = q_start[b+1] - q_start[b] (without q_start: n_kept[b]), and its other pages go on the stack
    free_pages[:free_count], in place.  lens_out may be kv_lens and free_left may be free_count.  flags: 0 or a sum of TRIM_*."""
    if block_table.dim() != 2:
        raise ValueError("block_table: int32 [B, max_pages]")
    dev, i32 = _device(block_table), torch.int32
    (B, columns), page_tokens = block_table.shape, index(page_tokens)
    new = lambda n: torch.empty(n, dtype=i32, device=block_table.device)  # noqa: E731
    lens_out = new(B) if lens_out is None else lens_out
    free_left = new(1) if free_left is None else free_left
    flags = new(1) if flags is None else flags
    st = load().fedrag_paged_trim(
        B, page_tokens, columns, _exactly("kv_lens", kv_lens, i32, dev, (B,)),
        None if q_start is None else _values("q_start", q_start, i32, dev, B + 1), _exactly("n_kept", n_kept, i32, dev, (B,)),
        _exactly("block_table", block_table, i32, dev, (B, columns)), _values("free_pages", free_pages, i32, dev, 0), free_pages.numel(),
        _values("free_count", free_count, i32, dev, 1), _exactly("lens_out", lens_out, i32, dev, (B,)),
        _values("free_left", free_left, i32, dev, 1), _values("flags", flags, i32, dev, 1), torch._C._cuda_getCurrentRawStream(dev))
    if st != OK:
        raise FedragError(st, "fedrag_paged_trim")
    return lens_out, free_left, flags


def fedrag_invert_perm(perm, inv_out=None):
    inv_out = torch.empty_like(perm) if inv_out is None else inv_out
    st = load().fedrag_invert_perm(_ptr(perm), perm.numel(), _ptr(inv_out), _stream())
    _check(st, "fedrag_invert_perm")
    return inv_out


def fedrag_validate_perm(perm, flag_out=None, marks=None):
    """Debug aid: device int32 flag, 0 when every row of perm ([L] or [n_perm, L] int32) is a permutation of 0..L-1,
    else bit 0 = an index out of range, bit 1 = an index repeated.  Read it after synchronising."""
    n_perm = 1 if perm.dim() == 1 else perm.shape[0]
    L = perm.shape[-1]
    flag_out = torch.empty(1, dtype=torch.int32, device=perm.device) if flag_out is None else flag_out
    marks = torch.empty(max(1, n_perm * L), dtype=torch.int32, device=perm.device) if marks is None else marks
    st = load().fedrag_validate_perm(_ptr(perm), n_perm, L, _ptr(marks), _ptr(flag_out), _stream())
    _check(st, "fedrag_validate_perm")
    return flag_out
