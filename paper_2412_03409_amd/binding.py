"""ctypes binding of include/prefixkv.h.  Argument marshalling only.

The wrappers have the names of the C entry points.  Tensors must live on the GPU; outputs and the
workspace are allocated here with torch (the library itself never allocates) unless passed in.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from functools import lru_cache
from operator import index
from pathlib import Path
from typing import Optional

import torch

_HERE = Path(__file__).resolve().parent
_LIB_PATH = _HERE / "libprefixkv.so"

PKV_F32, PKV_BF16 = 0, 1
_ERR_WORKSPACE = 5   # PKV_ERR_WORKSPACE
OP_IMPORTANCE, OP_SELECT, OP_COMPACT, OP_DECODE, OP_MERGE_FEATURE = 0, 1, 2, 3, 4


class PrefixKVError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: status {code} ({prefixkv_status_string(code)})")
        self.code = code


class _Shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "L", "H", "Hkv", "N", "D", "dtype")]


class _Strides(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("b", "l", "h", "n")]


class _SelectParams(C.Structure):
    _fields_ = [("budget_tokens", C.c_int64), ("tol_tokens", C.c_int64), ("max_iters", C.c_int32),
                ("fixup", C.c_int32)]


class _Packed(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("S", "L", "H", "Hkv", "T", "D", "dtype")]


class _Paging(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("num_pages", "page_size", "max_pages", "layers")]


class _Rope(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("axis", C.c_void_p), ("rot_dim", C.c_int32), ("axes", C.c_int32),
                ("interleaved", C.c_int32)]


_lib = None


def lib_path() -> Path:
    return _LIB_PATH


def load(path: Optional[str] = None) -> C.CDLL:
    """Load libprefixkv.so (or another build of it at `path`); raises if it has not been built
    (no fallback exists)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or os.environ.get("PKV_LIB_PATH")   # an alternative build of the same library
    lib_file = Path(path) if path else _LIB_PATH
    if not lib_file.exists():
        raise ImportError(f"{lib_file} is missing: build it with `python -m paper_2412_03409_amd.build` "
                          "(hipcc, gfx950); there is no CPU path")
    L = C.CDLL(str(lib_file))
    vp, i32, i64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
    L.prefixkv_version.restype = C.c_int
    L.prefixkv_status_string.restype = C.c_char_p
    L.prefixkv_status_string.argtypes = [C.c_int]
    L.prefixkv_workspace_bytes.restype = sz
    L.prefixkv_workspace_bytes.argtypes = [i32, C.POINTER(_Shape), i32]
    L.prefixkv_importance.restype = C.c_int
    L.prefixkv_importance.argtypes = [C.POINTER(_Shape), vp, _Strides, vp, _Strides, vp, vp, vp, vp, sz, vp]
    L.prefixkv_prefill_attn.restype = C.c_int
    L.prefixkv_prefill_attn.argtypes = [C.POINTER(_Shape), vp, _Strides, vp, _Strides, vp, _Strides, vp, vp, vp, vp]
    L.prefixkv_select.restype = C.c_int
    L.prefixkv_select.argtypes = [i32, i32, i32, vp, C.POINTER(_SelectParams), vp, vp, vp, vp, vp, vp, vp,
                                  vp, vp, sz, vp]
    L.prefixkv_select_static.restype = C.c_int
    L.prefixkv_select_static.argtypes = [i32, i32, i32, vp, C.POINTER(_SelectParams), vp, vp, vp, vp, vp, vp, vp,
                                         vp, vp]
    L.prefixkv_static_scratch_segments.restype = C.c_int
    L.prefixkv_rank.restype = C.c_int
    L.prefixkv_rank.argtypes = [i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    L.prefixkv_offline_config.restype = C.c_int
    L.prefixkv_offline_config.argtypes = [i32, i32, i32, vp, i64, i32, vp, vp]
    L.prefixkv_gini.restype = C.c_int
    L.prefixkv_gini.argtypes = [i32, i32, i32, vp, vp, vp]
    L.prefixkv_merge_position.restype = C.c_int
    L.prefixkv_merge_position.argtypes = [C.POINTER(_Shape), vp, _Strides, vp, _Strides, vp, vp, vp, vp, vp, vp, vp]
    L.prefixkv_merge_feature.restype = C.c_int
    L.prefixkv_merge_feature.argtypes = [C.POINTER(_Shape), vp, _Strides, vp, _Strides, vp, vp, vp, vp, vp, vp, vp,
                                         vp, sz, vp]
    L.prefixkv_compact.restype = C.c_int
    L.prefixkv_compact.argtypes = [C.POINTER(_Shape), vp, _Strides, vp, _Strides, vp, vp, i32, vp, vp, vp,
                                   vp, vp, vp, vp, sz, vp]
    L.prefixkv_cache_tokens_upper_bound.restype = i64
    L.prefixkv_cache_tokens_upper_bound.argtypes = [i32, i64, i32, i32]
    L.prefixkv_decode_attn.restype = C.c_int
    L.prefixkv_decode_attn.argtypes = [C.POINTER(_Shape), i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                       vp, sz, vp]
    L.prefixkv_decode_attn_evict.restype = C.c_int
    L.prefixkv_decode_attn_evict.argtypes = [C.POINTER(_Shape), i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                             vp, vp, i32, i32, vp, vp, sz, vp]
    packed, paging, rope = C.POINTER(_Packed), C.POINTER(_Paging), C.POINTER(_Rope)
    L.prefixkv_page_workspace_bytes.restype = sz
    L.prefixkv_page_workspace_bytes.argtypes = [i32, i32]
    L.prefixkv_page_resize.restype = C.c_int
    L.prefixkv_page_resize.argtypes = [i32, paging, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.prefixkv_page_append.restype = C.c_int
    L.prefixkv_page_append.argtypes = [i32, i32, paging, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.prefixkv_rope_freq.restype = C.c_int
    L.prefixkv_rope_freq.argtypes = [i32, C.c_double, vp]
    L.prefixkv_rope.restype = C.c_int
    L.prefixkv_rope.argtypes = [packed, rope, vp, vp, _Strides, vp, _Strides, vp, _Strides, vp, _Strides, vp]
    L.prefixkv_rope_store.restype = C.c_int
    L.prefixkv_rope_store.argtypes = [packed, rope, vp, vp, _Strides, vp, _Strides, vp, _Strides, vp, _Strides, vp, paging,
                                      vp, vp, vp]
    L.prefixkv_compact_paged.restype = C.c_int
    L.prefixkv_compact_paged.argtypes = [C.POINTER(_Shape), vp, _Strides, vp, _Strides, vp, vp, paging, i32, vp, vp, vp, vp, vp]
    L.prefixkv_attn_workspace_bytes.restype = sz
    L.prefixkv_attn_workspace_bytes.argtypes = [packed, i32]
    L.prefixkv_prefill_attn_packed.restype = C.c_int
    L.prefixkv_prefill_attn_packed.argtypes = [packed, vp, _Strides, vp, _Strides, vp, _Strides, vp, vp, vp, _Strides, vp, vp,
                                               sz, vp]
    L.prefixkv_chunk_attn.restype = C.c_int
    L.prefixkv_chunk_attn.argtypes = [packed, vp, _Strides, vp, paging, i32, vp, vp, vp, vp, vp, i32, vp, _Strides, vp, sz, vp]
    L.prefixkv_calibration_copy.restype = C.c_int
    L.prefixkv_calibration_copy.argtypes = [vp, vp, sz, vp]
    _lib = L
    return L


def prefixkv_version() -> int:
    return int(load().prefixkv_version())


def prefixkv_status_string(code: int) -> str:
    return load().prefixkv_status_string(int(code)).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return PKV_F32
    if t.dtype == torch.bfloat16:
        return PKV_BF16
    raise TypeError(f"unsupported storage dtype {t.dtype}")


@lru_cache(maxsize=256, typed=True)
def _shape_of(B, L, H, Hkv, N, D, dtype) -> _Shape:
    return _Shape(B, L, H, Hkv, N, D, dtype)


def _shape(B, L, H, Hkv, N, D, dtype) -> _Shape:
    """The argument struct of a shape (only read, so one object per value serves every call).  Any integer of the caller's
    will do, an array or tensor of no dimension too: the cache is asked for its value.  (_shape_of: sizes of tensors.)"""
    return _shape_of(index(B), index(L), index(H), index(Hkv), index(N), index(D), index(dtype))


@lru_cache(maxsize=256, typed=True)
def _decode_shape_of(B, L, H, Hkv, N, D, dtype):
    """A decode step's argument struct by reference, and its workspace: pure functions of the shape, asked for in every step."""
    s = C.byref(_shape(B, L, H, Hkv, N, D, dtype))
    return s, int(load().prefixkv_workspace_bytes(OP_DECODE, s, 0))


def _strides5(t: torch.Tensor) -> _Strides:
    if t.stride(4) != 1:
        raise ValueError("the head dimension must be contiguous")
    return _Strides(t.stride(0), t.stride(1), t.stride(2), t.stride(3))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The current stream's handle without a Stream object around it (1.2 us a call), where torch has that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    # with an index: without one torch looks the device up through four layers of its own (4 us a call)
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream(torch.cuda.current_device()).cuda_stream


def _need_cuda(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("all tensors must be on the GPU")


def _ws(nbytes: int, device, ws: Optional[torch.Tensor]) -> torch.Tensor:
    if ws is not None:
        if ws.numel() * ws.element_size() < nbytes:
            raise ValueError("workspace too small")
        return ws
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def prefixkv_workspace_bytes(op: int, B, L, H, Hkv, N, D, dtype, has_lse: bool = False) -> int:
    s = _shape(B, L, H, Hkv, N, D, dtype)
    return int(load().prefixkv_workspace_bytes(op, C.byref(s), int(has_lse)))


@lru_cache(maxsize=256, typed=True)
def _select_ws_bytes_of(B, L, N) -> int:
    return select_workspace_bytes(B, L, N)


def select_workspace_bytes(B: int, L: int, N: int) -> int:
    # stages 2 and 3 do not depend on the head geometry: any valid one serves for the size query
    s = _shape(B, L, 1, 1, N, 128, PKV_BF16)
    return int(load().prefixkv_workspace_bytes(OP_SELECT, C.byref(s), 0))


def prefixkv_cache_tokens_upper_bound(B: int, budget_tokens: int, L: int, decode_capacity: int) -> int:
    return int(load().prefixkv_cache_tokens_upper_bound(B, budget_tokens, L, decode_capacity))


def prefixkv_importance(q: torch.Tensor, k: torch.Tensor, scale: torch.Tensor,
                        lse: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q [B,L,H,N,D], k [B,L,Hkv,N,D] (bf16 or f32), scale [L] f32, optional lse [B,L,H,N] f32
    -> importance [B,L,N] f32."""
    _need_cuda(q, k, scale, lse, out, ws)
    B, L, H, N, D = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, L, Hkv, N, D) or k.dtype != q.dtype:
        raise ValueError("k must be [B,L,Hkv,N,D] with q's dtype")
    if scale.dtype != torch.float32 or scale.shape != (L,) or not scale.is_contiguous():
        raise ValueError("scale must be contiguous f32 [L]")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (B, L, H, N) or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous f32 [B,L,H,N]")
    s = _shape_of(B, L, H, Hkv, N, D, _dtype_code(q))
    if out is None:
        out = torch.empty((B, L, N), dtype=torch.float32, device=q.device)
    # a workspace of the caller's may be smaller than the recommended one: the library says what it accepts
    w = ws if ws is not None else _ws(load().prefixkv_workspace_bytes(OP_IMPORTANCE, C.byref(s), int(lse is not None)),
                                      q.device, None)
    rc = load().prefixkv_importance(C.byref(s), _ptr(q), _strides5(q), _ptr(k), _strides5(k), _ptr(scale),
                                    _ptr(lse), _ptr(out), _ptr(w), w.numel() * w.element_size(), _stream())
    if rc == _ERR_WORKSPACE:
        raise ValueError("workspace too small")
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_importance")
    return out


def prefixkv_prefill_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: torch.Tensor,
                          out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
    """Causal attention over the prompt: q [B,L,H,N,D], k/v [B,L,Hkv,N,D] (bf16), scale [L] f32
    -> (out [B,L,H,N,D] bf16, lse [B,L,H,N] f32, ready to be passed to prefixkv_importance)."""
    _need_cuda(q, k, v, scale, out, lse)
    B, L, H, N, D = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, L, Hkv, N, D) or v.shape != k.shape or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("k, v must be [B,L,Hkv,N,D] with q's dtype")
    if scale.dtype != torch.float32 or scale.shape != (L,) or not scale.is_contiguous():
        raise ValueError("scale must be contiguous f32 [L]")
    if out is None:
        out = torch.empty((B, L, H, N, D), dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((B, L, H, N), dtype=torch.float32, device=q.device)
    s = _shape_of(B, L, H, Hkv, N, D, _dtype_code(q))
    rc = load().prefixkv_prefill_attn(C.byref(s), _ptr(q), _strides5(q), _ptr(k), _strides5(k), _ptr(v),
                                      _strides5(v), _ptr(scale), _ptr(out), _ptr(lse), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_prefill_attn")
    return out, lse


@dataclass
class SelectResult:
    order: torch.Tensor      # [B,L,N] i32
    cum: torch.Tensor        # [B,L,N] i64 holding the u64 bit pattern
    prefix: Optional[torch.Tensor]  # [B,L,N] f32
    lengths: torch.Tensor    # [B,L] i32
    p: torch.Tensor          # [B] f64
    iters: torch.Tensor      # [B] i32
    raw_total: torch.Tensor  # [B] i64
    status: torch.Tensor     # [B] i32


def prefixkv_select(importance: torch.Tensor, budget_tokens: int, tol_tokens: int = 0,
                    max_iters: int = 64, fixup: bool = True, want_prefix: bool = True,
                    out: Optional[SelectResult] = None, ws: Optional[torch.Tensor] = None) -> SelectResult:
    """importance [B,L,N] f32 -> SelectResult (all on the device; nothing is read back)."""
    _need_cuda(importance, ws)
    if importance.dtype != torch.float32 or importance.dim() != 3 or not importance.is_contiguous():
        raise ValueError("importance must be contiguous f32 [B,L,N]")
    B, L, N = importance.shape
    dev = importance.device
    if out is None:
        out = SelectResult(
            order=torch.empty((B, L, N), dtype=torch.int32, device=dev),
            cum=torch.empty((B, L, N), dtype=torch.int64, device=dev),
            prefix=torch.empty((B, L, N), dtype=torch.float32, device=dev) if want_prefix else None,
            lengths=torch.empty((B, L), dtype=torch.int32, device=dev),
            p=torch.empty(B, dtype=torch.float64, device=dev),
            iters=torch.empty(B, dtype=torch.int32, device=dev),
            raw_total=torch.empty(B, dtype=torch.int64, device=dev),
            status=torch.empty(B, dtype=torch.int32, device=dev))
    prm = _SelectParams(int(budget_tokens), int(tol_tokens), int(max_iters), int(bool(fixup)))
    w = _ws(_select_ws_bytes_of(B, L, N), dev, ws)
    rc = load().prefixkv_select(B, L, N, _ptr(importance), C.byref(prm), _ptr(out.order), _ptr(out.cum),
                                _ptr(out.prefix), _ptr(out.lengths), _ptr(out.p), _ptr(out.iters),
                                _ptr(out.raw_total), _ptr(out.status), _ptr(w),
                                w.numel() * w.element_size(), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_select")
    return out


def prefixkv_select_static(importance: torch.Tensor, budget_tokens: int, out: SelectResult, tol_tokens: int = 0,
                           max_iters: int = 64, fixup: bool = True) -> SelectResult:
    """prefixkv_select without a workspace and without any allocation: `out` must be pre-allocated
    (all eight tensors; prefix may be None).  B*L <= prefixkv_static_scratch_segments()."""
    _need_cuda(importance, out.order, out.cum, out.prefix, out.lengths, out.p, out.iters, out.raw_total, out.status)
    if importance.dtype != torch.float32 or importance.dim() != 3 or not importance.is_contiguous():
        raise ValueError("importance must be contiguous f32 [B,L,N]")
    B, L, N = importance.shape
    prm = _SelectParams(int(budget_tokens), int(tol_tokens), int(max_iters), int(bool(fixup)))
    rc = load().prefixkv_select_static(B, L, N, _ptr(importance), C.byref(prm), _ptr(out.order), _ptr(out.cum),
                                       _ptr(out.prefix), _ptr(out.lengths), _ptr(out.p), _ptr(out.iters),
                                       _ptr(out.raw_total), _ptr(out.status), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_select_static")
    return out


def prefixkv_static_scratch_segments() -> int:
    return int(load().prefixkv_static_scratch_segments())


@dataclass
class RankResult:
    order: torch.Tensor      # [B,L,N] i32
    cum: torch.Tensor        # [B,L,N] i64 holding the u64 bit pattern
    prefix: Optional[torch.Tensor]  # [B,L,N] f32
    status: torch.Tensor     # [B] i32


def prefixkv_rank(importance: torch.Tensor, want_prefix: bool = True, out: Optional[RankResult] = None,
                  ws: Optional[torch.Tensor] = None) -> RankResult:
    """importance [B,L,N] f32 -> per-layer ranking and cumulative priority, without the search."""
    _need_cuda(importance, ws)
    if importance.dtype != torch.float32 or importance.dim() != 3 or not importance.is_contiguous():
        raise ValueError("importance must be contiguous f32 [B,L,N]")
    B, L, N = importance.shape
    dev = importance.device
    if out is None:
        out = RankResult(
            order=torch.empty((B, L, N), dtype=torch.int32, device=dev),
            cum=torch.empty((B, L, N), dtype=torch.int64, device=dev),
            prefix=torch.empty((B, L, N), dtype=torch.float32, device=dev) if want_prefix else None,
            status=torch.empty(B, dtype=torch.int32, device=dev))
    w = _ws(select_workspace_bytes(B, L, N), dev, ws)
    rc = load().prefixkv_rank(B, L, N, _ptr(importance), _ptr(out.order), _ptr(out.cum), _ptr(out.prefix),
                              _ptr(out.status), _ptr(w), w.numel() * w.element_size(), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_rank")
    return out


def prefixkv_offline_config(sample_lengths: torch.Tensor, N: int, budget_tokens: int, B_out: int = 1,
                            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """sample_lengths [S,L] i32 (device) -> shared per-layer lengths, repeated: [B_out,L] i32."""
    _need_cuda(sample_lengths, out)
    if sample_lengths.dtype != torch.int32 or sample_lengths.dim() != 2 or not sample_lengths.is_contiguous():
        raise ValueError("sample_lengths must be contiguous i32 [S,L]")
    S, L = sample_lengths.shape
    if out is None:
        out = torch.empty((B_out, L), dtype=torch.int32, device=sample_lengths.device)
    elif out.dtype != torch.int32 or out.shape != (B_out, L) or not out.is_contiguous():
        raise ValueError("out must be contiguous i32 [B_out,L]")
    rc = load().prefixkv_offline_config(S, L, int(N), _ptr(sample_lengths), int(budget_tokens), int(B_out),
                                        _ptr(out), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_offline_config")
    return out


@dataclass
class CompactResult:
    kc: torch.Tensor         # flat [cache_tokens*Hkv*D] storage dtype
    vc: torch.Tensor
    kept_pos: torch.Tensor   # [cache_tokens] i32
    seg_off: torch.Tensor    # [B,L] i64 (tokens)
    caps: torch.Tensor       # [B,L] i32
    lens: torch.Tensor       # [B,L] i32
    cache_tokens: int
    Hkv: int
    D: int


def prefixkv_compact(k: torch.Tensor, v: torch.Tensor, order: torch.Tensor, lengths: torch.Tensor,
                     decode_capacity: int, cache_tokens: int,
                     out: Optional[CompactResult] = None) -> CompactResult:
    """k,v [B,L,Hkv,N,D]; order [B,L,N] i32; lengths [B,L] i32 -> ragged compressed cache.
    cache_tokens: token slots to allocate (prefixkv_cache_tokens_upper_bound)."""
    _need_cuda(k, v, order, lengths)
    B, L, Hkv, N, D = k.shape
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("v must match k")
    if order.dtype != torch.int32 or order.shape != (B, L, N) or not order.is_contiguous():
        raise ValueError("order must be contiguous i32 [B,L,N]")
    if lengths.dtype != torch.int32 or lengths.shape != (B, L) or not lengths.is_contiguous():
        raise ValueError("lengths must be contiguous i32 [B,L]")
    dev = k.device
    if out is None:
        out = CompactResult(
            kc=torch.empty(cache_tokens * Hkv * D, dtype=k.dtype, device=dev),
            vc=torch.empty(cache_tokens * Hkv * D, dtype=k.dtype, device=dev),
            kept_pos=torch.empty(cache_tokens, dtype=torch.int32, device=dev),
            seg_off=torch.empty((B, L), dtype=torch.int64, device=dev),
            caps=torch.empty((B, L), dtype=torch.int32, device=dev),
            lens=torch.empty((B, L), dtype=torch.int32, device=dev),
            cache_tokens=int(cache_tokens), Hkv=Hkv, D=D)
    s = _shape_of(B, L, Hkv, Hkv, N, D, _dtype_code(k))
    rc = load().prefixkv_compact(C.byref(s), _ptr(k), _strides5(k), _ptr(v), _strides5(v), _ptr(order),
                                 _ptr(lengths), int(decode_capacity), _ptr(out.seg_off), _ptr(out.caps),
                                 _ptr(out.kc), _ptr(out.vc), _ptr(out.kept_pos), _ptr(out.lens), None, 0,
                                 _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_compact")
    return out


def prefixkv_merge_position(cache: CompactResult, k: torch.Tensor, v: torch.Tensor) -> CompactResult:
    """Average every pruned position into the nearest kept one, in place on a freshly compacted cache."""
    _need_cuda(k, v)
    B, L, Hkv, N, D = k.shape
    if v.shape != k.shape or v.dtype != k.dtype or k.dtype != cache.kc.dtype or D != cache.D or Hkv != cache.Hkv:
        raise ValueError("k, v must be the [B,L,Hkv,N,D] tensors the cache was compacted from")
    s = _shape_of(B, L, Hkv, Hkv, N, D, _dtype_code(k))
    rc = load().prefixkv_merge_position(C.byref(s), _ptr(k), _strides5(k), _ptr(v), _strides5(v),
                                        _ptr(cache.seg_off), _ptr(cache.caps), _ptr(cache.kept_pos),
                                        _ptr(cache.lens), _ptr(cache.kc), _ptr(cache.vc), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_merge_position")
    return cache


def prefixkv_merge_feature(cache: CompactResult, k: torch.Tensor, v: torch.Tensor,
                           match: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Average every pruned vector into the most similar (cosine) retained vector of its head, keys by key
    similarity and values by value similarity, in place on a freshly compacted bf16 cache.  Returns the
    assignment match [2,B,L,Hkv,N] i32 (plane 0 keys, 1 values; -1 at retained positions)."""
    _need_cuda(k, v, match, ws)
    B, L, Hkv, N, D = k.shape
    if v.shape != k.shape or v.dtype != k.dtype or k.dtype != cache.kc.dtype or D != cache.D or Hkv != cache.Hkv:
        raise ValueError("k, v must be the [B,L,Hkv,N,D] tensors the cache was compacted from")
    if match is None:
        match = torch.empty((2, B, L, Hkv, N), dtype=torch.int32, device=k.device)
    elif match.dtype != torch.int32 or tuple(match.shape) != (2, B, L, Hkv, N) or not match.is_contiguous():
        raise ValueError("match must be contiguous i32 [2,B,L,Hkv,N]")
    s = _shape_of(B, L, Hkv, Hkv, N, D, _dtype_code(k))
    w = _ws(load().prefixkv_workspace_bytes(OP_MERGE_FEATURE, C.byref(s), 0), k.device, ws)
    rc = load().prefixkv_merge_feature(C.byref(s), _ptr(k), _strides5(k), _ptr(v), _strides5(v),
                                       _ptr(cache.seg_off), _ptr(cache.caps), _ptr(cache.kept_pos),
                                       _ptr(cache.lens), _ptr(cache.kc), _ptr(cache.vc), _ptr(match), _ptr(w),
                                       w.numel() * w.element_size(), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_merge_feature")
    return match


def prefixkv_gini(cum: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """cum [B,L,N] (i64 holding the u64 sums of prefixkv_select / prefixkv_rank) -> Gini coefficients [B,L] f64."""
    _need_cuda(cum, out)
    if cum.dtype != torch.int64 or cum.dim() != 3 or not cum.is_contiguous():
        raise ValueError("cum must be contiguous i64 [B,L,N]")
    B, L, N = cum.shape
    if out is None:
        out = torch.empty((B, L), dtype=torch.float64, device=cum.device)
    rc = load().prefixkv_gini(B, L, N, _ptr(cum), _ptr(out), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_gini")
    return out


def prefixkv_decode_attn(cache: CompactResult, q: torch.Tensor, k_new: Optional[torch.Tensor],
                         v_new: Optional[torch.Tensor], scale: torch.Tensor, N: int,
                         l0: int = 0, l1: Optional[int] = None,
                         out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One decode step over layers [l0,l1): q [B,L,H,D], k_new/v_new [B,L,Hkv,D] or None
    -> out [B,L,H,D].  Appends in place and advances cache.lens on the device."""
    _need_cuda(q, k_new, v_new, scale, out)
    B, L, H, D = q.shape
    l1 = L if l1 is None else l1
    dt = q.dtype
    if not q.is_contiguous() or dt != cache.kc.dtype or D != cache.D:
        raise ValueError("q must be contiguous [B,L,H,D] in the cache dtype")
    for t in (k_new, v_new):
        if t is not None and (t.shape != (B, L, cache.Hkv, D) or not t.is_contiguous() or t.dtype != dt):
            raise ValueError("k_new/v_new must be contiguous [B,L,Hkv,D] in the cache dtype")
    if scale.dtype != torch.float32 or scale.shape != (L,) or not scale.is_contiguous():
        raise ValueError("scale must be contiguous f32 [L]")
    if out is None:
        out = torch.empty((B, L, H, D), dtype=dt, device=q.device)
    s, need = _decode_shape_of(B, L, H, index(cache.Hkv), index(N), D, _dtype_code(q))
    w = _ws(need, q.device, ws)
    rc = load().prefixkv_decode_attn(s, int(l0), int(l1), q.data_ptr(), _ptr(k_new), _ptr(v_new), scale.data_ptr(),
                                     cache.kc.data_ptr(), _ptr(cache.vc), _ptr(cache.seg_off), _ptr(cache.caps),
                                     _ptr(cache.lens), out.data_ptr(), w.data_ptr(), w.numel() * w.element_size(),
                                     _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_decode_attn")
    return out


_own_decode_attn = prefixkv_decode_attn


def decode_attn_steps(cache: CompactResult, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, scale: torch.Tensor,
                      N: int, T: int, out: torch.Tensor, ws: Optional[torch.Tensor]) -> bool:
    """prefixkv_decode_attn over all layers for steps 0 .. T-1 of contiguous q, out [>=T,B,L,H,D] and k_new, v_new
    [>=T,B,L,Hkv,D]: the same calls, whose arguments are looked at once.  False, and nothing is done, where a step by itself
    has to see to it (other layouts, other types, errors) or a program has put a function of its own in the step's place."""
    xs = (q, k_new, v_new, out)
    if prefixkv_decode_attn is not _own_decode_attn or ws is None:
        return False
    if T < 1 or any(type(x) is not torch.Tensor or not x.is_cuda or x.dim() != 5 or not x.is_contiguous() or x.shape[0] < T for x in xs):
        return False
    _, B, L, H, D = q.shape
    dt, new = q.dtype, (B, L, cache.Hkv, D)
    if (dt != cache.kc.dtype or dt not in (torch.float32, torch.bfloat16) or D != cache.D or any(x.dtype != dt for x in xs)
            or out.shape[1:] != q.shape[1:] or k_new.shape[1:] != new or v_new.shape[1:] != new
            or any(x.requires_grad or x.is_conj() or x.is_neg() for x in xs) or any(x.device != q.device for x in xs)
            or not scale.is_cuda or scale.dtype != torch.float32 or scale.shape != (L,) or not scale.is_contiguous()):
        return False
    s, need = _decode_shape_of(B, L, H, index(cache.Hkv), index(N), D, _dtype_code(q))
    nbytes = ws.numel() * ws.element_size()
    if nbytes < need:
        return False
    step = load().prefixkv_decode_attn
    qs, ns = B * L * H * D * q.element_size(), B * L * cache.Hkv * D * q.element_size()
    qp, kp, vp, op = (x.data_ptr() for x in xs)
    args = (scale.data_ptr(), cache.kc.data_ptr(), _ptr(cache.vc), _ptr(cache.seg_off), _ptr(cache.caps), _ptr(cache.lens))
    wp, st = ws.data_ptr(), _stream()
    for t in range(T):
        rc = step(s, 0, L, qp + t * qs, kp + t * ns, vp + t * ns, *args, op + t * qs, wp, nbytes, st)
        if rc != 0:
            raise PrefixKVError(rc, "prefixkv_decode_attn")
    return True


def prefixkv_decode_attn_evict(cache: CompactResult, base_lens: torch.Tensor, q: torch.Tensor,
                               k_new: torch.Tensor, v_new: torch.Tensor, scale: torch.Tensor, N: int, t: int,
                               distance: int, l0: int = 0, l1: Optional[int] = None,
                               track_positions: bool = True, out: Optional[torch.Tensor] = None,
                               ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Decode step t (1-based) with pruning at `distance` from the newest token; cache.lens counts the
    permanent entries.  base_lens [B,L] i32 = the lengths the cache was compacted with."""
    _need_cuda(q, k_new, v_new, scale, base_lens, out)
    B, L, H, D = q.shape
    l1 = L if l1 is None else l1
    if not q.is_contiguous() or q.dtype != cache.kc.dtype or D != cache.D:
        raise ValueError("q must be contiguous [B,L,H,D] in the cache dtype")
    for x in (k_new, v_new):
        if x.shape != (B, L, cache.Hkv, D) or not x.is_contiguous() or x.dtype != q.dtype:
            raise ValueError("k_new/v_new must be contiguous [B,L,Hkv,D] in the cache dtype")
    if scale.dtype != torch.float32 or scale.shape != (L,) or not scale.is_contiguous():
        raise ValueError("scale must be contiguous f32 [L]")
    if base_lens.dtype != torch.int32 or base_lens.shape != (B, L) or not base_lens.is_contiguous():
        raise ValueError("base_lens must be contiguous i32 [B,L]")
    if out is None:
        out = torch.empty((B, L, H, D), dtype=q.dtype, device=q.device)
    s, need = _decode_shape_of(B, L, H, index(cache.Hkv), index(N), D, _dtype_code(q))
    w = _ws(need, q.device, ws)
    rc = load().prefixkv_decode_attn_evict(
        s, int(l0), int(l1), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(scale), _ptr(cache.kc),
        _ptr(cache.vc), _ptr(cache.seg_off), _ptr(cache.caps), _ptr(base_lens), _ptr(cache.lens),
        _ptr(cache.kept_pos) if track_positions else None, int(t), int(distance), _ptr(out), _ptr(w),
        w.numel() * w.element_size(), _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_decode_attn_evict")
    return out


# ---- packed prompts and paged caches -----------------------------------------------------------------------
# These calls come once per layer and step, and the small ones take the GPU less time than a look at ten tensors takes here:
# what follows from shapes, strides and types alone (the checks and the argument structs) is worked out once per combination.
# (Addresses are asked for in every call.  A cache whose tensors get another shape is another PagedCache.)
@dataclass(frozen=True, eq=False)
class PagedCache:
    kp: torch.Tensor      # [num_pages,Hkv,page_size,D] storage dtype
    vp: torch.Tensor
    table: torch.Tensor   # [S,layers,max_pages] i32
    lens: torch.Tensor    # [S,layers] i32
    ring: torch.Tensor    # [num_pages] i32: the free pages, from head on
    state: torch.Tensor   # [2] i32: head, count

    def __post_init__(self):
        for t in (self.table, self.lens, self.ring, self.state):
            if t.dtype != torch.int32 or not t.is_contiguous():
                raise ValueError("table, lens, ring and state must be contiguous i32")
        if self.kp.dim() != 4 or self.vp.shape != self.kp.shape or self.vp.dtype != self.kp.dtype:
            raise ValueError("kp, vp must be [num_pages,Hkv,page_size,D] of one dtype")
        if (self.table.dim() != 3 or self.lens.shape != self.table.shape[:2] or self.ring.shape != self.kp.shape[:1]
                or self.state.shape != (2,)):
            raise ValueError("table must be [S,layers,max_pages], lens [S,layers], ring [num_pages], state [2]")
        P, Hkv, ps, D = self.kp.shape
        pool = (Hkv, D, self.kp.dtype) if self.kp.is_contiguous() and self.vp.is_contiguous() else None
        device = {t.device for t in (self.kp, self.vp, self.table, self.lens, self.ring, self.state)}
        if len(device) > 1:
            raise ValueError("the parts of a cache must be on one device")
        for name, x in (("_paging", C.byref(_Paging(P, ps, self.table.shape[2], self.table.shape[1]))), ("_pool", pool),
                        ("_S", self.table.shape[0]), ("_layers", self.table.shape[1]), ("_seg", self.lens.shape),
                        ("_offs", (self.table.shape[0] + 1,)), ("_device", self.kp.get_device())):
            object.__setattr__(self, name, x)


def paged_cache(S: int, layers: int, Hkv: int, D: int, page_size: int, num_pages: int, max_pages: int,
                dtype: torch.dtype = torch.bfloat16, device="cuda") -> PagedCache:
    """An empty cache for S sequences: every page is free."""
    pool = (num_pages, Hkv, page_size, D)
    return PagedCache(kp=torch.empty(pool, dtype=dtype, device=device), vp=torch.empty(pool, dtype=dtype, device=device),
                      table=torch.full((S, layers, max_pages), -1, dtype=torch.int32, device=device),
                      lens=torch.zeros((S, layers), dtype=torch.int32, device=device),
                      ring=torch.arange(num_pages, dtype=torch.int32, device=device),
                      state=torch.tensor([0, num_pages], dtype=torch.int32, device=device))


def _here(d: int, *ts) -> int:
    """The current stream's handle; d (a tensor's or a cache's GPU) has to be the current one, and every tensor on it."""
    if d < 0:
        raise ValueError("all tensors must be on the GPU")
    if d != torch.cuda.current_device():
        raise ValueError("all tensors must be on the current GPU")
    for t in ts:
        if t is not None and t.get_device() != d:
            raise ValueError("all tensors must be on the current GPU")
    return _raw_stream(d) if _raw_stream is not None else torch.cuda.current_stream(d).cuda_stream


def _c_int(x: int, what: str) -> int:
    """A number for an int argument: ctypes would take it modulo 2^32."""
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{what} does not fit 32 bits")
    return x


def _i32_like(t: torch.Tensor, shape, what: str) -> torch.Tensor:
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous i32 {list(shape)}")
    return t


@lru_cache(maxsize=256, typed=True)
def page_workspace_bytes(S: int, layers: int) -> int:
    return int(load().prefixkv_page_workspace_bytes(S, layers))


def _page_out(cache: PagedCache, status, lens_out, state_out, ws):
    lens = cache.lens
    status = torch.empty(1, dtype=torch.int32, device=lens.device) if status is None else _i32_like(status, (1,), "status")
    lens_out = lens if lens_out is None else _i32_like(lens_out, cache._seg, "lens_out")
    state_out = cache.state if state_out is None else _i32_like(state_out, (2,), "state_out")
    return status, lens_out, state_out, _ws(page_workspace_bytes(cache._S, cache._layers), lens.device, ws)


def prefixkv_page_resize(cache: PagedCache, target: torch.Tensor, status: Optional[torch.Tensor] = None,
                         lens_out: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gives every segment the length target [S,layers] i32: pages come from the ring or go back to it; the cache's lens and
    state are updated (or lens_out, state_out written in their place).  -> status [1] i32, 0 if it was done."""
    lens, table, ring, state = cache.lens, cache.table, cache.ring, cache.state
    stream = _here(cache._device, target, status, lens_out, state_out, ws)
    _i32_like(target, cache._seg, "target")
    status, lens_out, state_out, w = _page_out(cache, status, lens_out, state_out, ws)
    rc = load().prefixkv_page_resize(cache._S, cache._paging, target.data_ptr(), lens.data_ptr(), table.data_ptr(),
                                     ring.data_ptr(), state.data_ptr(), lens_out.data_ptr(), state_out.data_ptr(),
                                     status.data_ptr(), w.data_ptr(), w.numel() * w.element_size(), stream)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_page_resize")
    return status


def prefixkv_page_append(cache: PagedCache, row_off: torch.Tensor, T: int, slots: Optional[torch.Tensor] = None,
                         status: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
                         state_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Room for the new rows of every sequence, in every layer: row_off [S+1] i32, T packed rows
    -> (slots [layers,T] i64, status [1] i32)."""
    lens, table, ring, state = cache.lens, cache.table, cache.ring, cache.state
    stream = _here(cache._device, row_off, slots, status, lens_out, state_out, ws)
    T = _c_int(index(T), "T")
    _i32_like(row_off, cache._offs, "row_off")
    if slots is None:
        slots = torch.empty((cache._layers, T), dtype=torch.int64, device=lens.device)
    elif slots.dtype is not torch.int64 or slots.shape != (cache._layers, T) or not slots.is_contiguous():
        raise ValueError("slots must be contiguous i64 [layers,T]")
    status, lens_out, state_out, w = _page_out(cache, status, lens_out, state_out, ws)
    rc = load().prefixkv_page_append(cache._S, T, cache._paging, row_off.data_ptr(), lens.data_ptr(), table.data_ptr(),
                                     ring.data_ptr(), state.data_ptr(), lens_out.data_ptr(), state_out.data_ptr(),
                                     slots.data_ptr(), status.data_ptr(), w.data_ptr(), w.numel() * w.element_size(), stream)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_page_append")
    return slots, status


@dataclass(frozen=True, eq=False)
class RopePlan:
    freq: torch.Tensor    # [rot_dim/2] i64 holding the u64 fractions of a turn
    axis: torch.Tensor    # [rot_dim/2] i32
    axes: int
    interleaved: bool

    def __post_init__(self):
        if self.freq.dtype != torch.int64 or self.freq.dim() != 1 or not self.freq.is_contiguous():
            raise ValueError("freq must be contiguous i64 [rot_dim/2]")
        _i32_like(self.axis, self.freq.shape, "axis")
        if self.axis.device != self.freq.device:
            raise ValueError("freq and axis must be on one device")
        at = self.freq.data_ptr(), self.axis.data_ptr()
        for name, x in (("_device", self.freq.get_device()), ("_at", at),
                        ("_struct", C.byref(_Rope(*at, 2 * self.freq.shape[0], self.axes, int(self.interleaved))))):
            object.__setattr__(self, name, x)

    def _args(self):
        """The argument struct, of where the tensors are now: a program may give them other storage."""
        if (self.freq.data_ptr(), self.axis.data_ptr()) != self._at:
            self.__post_init__()
        return self._struct


def rope_plan(rot_dim: int, sections=None, theta: float = 10000.0, interleaved: bool = False, cycled: bool = False,
              device="cuda") -> RopePlan:
    """Frequencies theta^(-2i/rot_dim) and the axis of every pair: the first sections[0] pairs turn with axis 0, the next
    sections[1] with axis 1, ...; cycled: the axes take turns pair by pair until their sections are used up.  Default: one axis."""
    half = rot_dim // 2
    sections = [half] if sections is None else [int(x) for x in sections]
    if sum(sections) != half or any(x < 0 for x in sections):
        raise ValueError(f"the sections must sum to {half} pairs")
    freq = (C.c_uint64 * max(half, 1))()
    rc = load().prefixkv_rope_freq(int(rot_dim), float(theta), freq)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_rope_freq")
    if cycled:
        left, axis = list(sections), []
        while len(axis) < half:
            for a in range(len(left)):
                if left[a] > 0:
                    left[a] -= 1
                    axis.append(a)
    else:
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
    signed = [x - (1 << 64) if x >= 1 << 63 else x for x in freq]
    return RopePlan(freq=torch.tensor(signed, dtype=torch.int64, device=device),
                    axis=torch.tensor(axis, dtype=torch.int32, device=device), axes=len(sections), interleaved=bool(interleaved))


def _row_strides(shape, stride, dtype) -> _Strides:
    """Strides of [L,heads,T,D] rows.  (A dimension of one element may have any stride: its own is not looked at.)"""
    if len(shape) != 4 or stride[3] != 1:
        raise ValueError("row tensors must be [L,heads,T,D] with D contiguous")
    a = 4 if dtype is torch.float32 else 8
    st = [a if n == 1 else x for x, n in zip(stride, shape)]
    return _Strides(0, st[0], st[1], st[2])


_CODES = {torch.float32: PKV_F32, torch.bfloat16: PKV_BF16}


def _packed(S, Hkv, qsh, dtype) -> _Packed:
    if dtype not in _CODES:
        raise TypeError(f"unsupported storage dtype {dtype}")
    return _Packed(S, qsh[0], qsh[1], Hkv, qsh[2], qsh[3], _CODES[dtype])


@lru_cache(maxsize=512)
def _rope_args(qsh, qst, qdt, ksh, kst, kdt, osh, ost, odt, xsh, xst, xdt, psh, pst, pdt, axes, cache):
    """Argument structs of a rotation: x is k_out, or v if the keys go into a cache (its heads, head dimension and dtype)."""
    strides = [_row_strides(*a) for a in ((qsh, qst, qdt), (ksh, kst, kdt), (xsh, xst, xdt), (osh, ost, odt))]
    if not (qdt == kdt == odt == xdt) or (ksh[0], ksh[2], ksh[3]) != (qsh[0], qsh[2], qsh[3]):
        raise ValueError("row tensors must be [L,heads,T,D] of one dtype")
    if osh != qsh or xsh != ksh:
        raise ValueError("q_out must have the shape of q, k_out or v that of k")
    if pdt != torch.int32 or psh != (axes, qsh[2]) or any(x != s for x, s, n in zip(pst, (qsh[2], 1), psh) if n > 1):
        raise ValueError("positions must be contiguous i32 [axes,T]")
    if cache is not None and cache != (ksh[1], ksh[3], kdt):
        raise ValueError("the cache must have k's heads, head dimension and dtype, and contiguous pools")
    return (C.byref(_packed(1, ksh[1], qsh, qdt)), *strides)


def prefixkv_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, plan: RopePlan,
                  q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """q [L,H,T,D], k [L,Hkv,T,D] (bf16 or f32, any strides with D contiguous), positions [axes,T] i32
    -> (q_out, k_out), rotated; q_out = q and k_out = k rotate in place."""
    rope = plan._args()
    stream = _here(plan._device, q, k, positions, q_out, k_out)
    q_out = torch.empty_like(q) if q_out is None else q_out
    k_out = torch.empty_like(k) if k_out is None else k_out
    s, qs, ks, kos, qos = _rope_args(q.shape, q.stride(), q.dtype, k.shape, k.stride(), k.dtype, q_out.shape, q_out.stride(),
                                     q_out.dtype, k_out.shape, k_out.stride(), k_out.dtype, positions.shape, positions.stride(),
                                     positions.dtype, plan.axes, None)
    rc = load().prefixkv_rope(s, rope, positions.data_ptr(), q.data_ptr(), qs, k.data_ptr(), ks, q_out.data_ptr(), qos,
                              k_out.data_ptr(), kos, stream)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_rope")
    return q_out, k_out


def prefixkv_rope_store(cache: PagedCache, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor,
                        plan: RopePlan, slots: torch.Tensor, q_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotates q [L,H,T,D] and k [L,Hkv,T,D] and stores k and v into the cache's pages at slots [L,T] i64 -> q_out."""
    kp, vp = cache.kp, cache.vp
    rope = plan._args()
    stream = _here(plan._device, q, k, v, positions, slots, q_out, kp)
    q_out = torch.empty_like(q) if q_out is None else q_out
    s, qs, ks, vs, qos = _rope_args(q.shape, q.stride(), q.dtype, k.shape, k.stride(), k.dtype, q_out.shape, q_out.stride(),
                                    q_out.dtype, v.shape, v.stride(), v.dtype, positions.shape, positions.stride(),
                                    positions.dtype, plan.axes, cache._pool or ())
    if slots.dtype is not torch.int64 or slots.shape != q.shape[::2] or not slots.is_contiguous():
        raise ValueError("slots must be contiguous i64 [L,T]")
    rc = load().prefixkv_rope_store(s, rope, positions.data_ptr(), q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
                                    q_out.data_ptr(), qos, slots.data_ptr(), cache._paging, kp.data_ptr(), vp.data_ptr(), stream)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_rope_store")
    return q_out


def prefixkv_compact_paged(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, order: torch.Tensor, lengths: torch.Tensor,
                           kept_pos: Optional[torch.Tensor] = None, l0: int = 0) -> PagedCache:
    """prefixkv_compact into the cache's pages: k,v [B,L,Hkv,N,D], order [B,L,N] i32, lengths [B,L] i32; sequence b of the
    batch is sequence b of the cache, layer l its layer l0 + l.  kept_pos [B,L,N] i32, optional output."""
    stream = _here(cache._device, k, v, order, lengths, kept_pos)
    B, L, Hkv, N, D = k.shape
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("v must match k")
    _i32_like(order, (B, L, N), "order")
    _i32_like(lengths, (B, L), "lengths")
    if kept_pos is not None:
        _i32_like(kept_pos, (B, L, N), "kept_pos")
    if cache._pool != (Hkv, D, k.dtype) or cache._S < B:
        raise ValueError("the cache must have k's heads, head dimension and dtype, B sequences and contiguous pools")
    s = _shape_of(B, L, Hkv, Hkv, N, D, _dtype_code(k))
    rc = load().prefixkv_compact_paged(C.byref(s), k.data_ptr(), _strides5(k), v.data_ptr(), _strides5(v), order.data_ptr(),
                                       lengths.data_ptr(), cache._paging, _c_int(int(l0), "l0"), cache.table.data_ptr(), cache.kp.data_ptr(),
                                       cache.vp.data_ptr(), _ptr(kept_pos), stream)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_compact_paged")
    return cache


def attn_workspace_bytes(S: int, L: int, H: int, Hkv: int, T: int, D: int, dtype: torch.dtype, max_rows: int = 0) -> int:
    """Workspace of prefixkv_chunk_attn, or (max_rows = 0) of prefixkv_prefill_attn_packed."""
    return int(load().prefixkv_attn_workspace_bytes(C.byref(_packed(S, Hkv, (L, H, T, D), dtype)), _c_int(int(max_rows), "max_rows")))


@lru_cache(maxsize=512)
def _attn_args(qsh, qst, qdt, osh, ost, odt, S, Hkv, max_rows):
    """Argument structs of rows q and out, and the call's workspace."""
    qs, os_ = _row_strides(qsh, qst, qdt), _row_strides(osh, ost, odt)
    if osh != qsh or odt != qdt:
        raise ValueError("out must have the shape and dtype of q")
    return C.byref(_packed(S, Hkv, qsh, qdt)), qs, os_, attn_workspace_bytes(S, qsh[0], qsh[1], Hkv, qsh[2], qsh[3], qdt, max_rows)


@lru_cache(maxsize=512)
def _key_args(ksh, kst, kdt, vsh, vst, vdt, qsh, qdt):
    if vsh != ksh or not (kdt == vdt == qdt) or len(ksh) != 4 or (ksh[0], ksh[2], ksh[3]) != (qsh[0], qsh[2], qsh[3]):
        raise ValueError("k, v must be [L,Hkv,T,D] with q's dtype")
    return _row_strides(ksh, kst, kdt), _row_strides(vsh, vst, vdt)


def prefixkv_prefill_attn_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, row_off: torch.Tensor, scale: torch.Tensor,
                                 out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                                 ws: Optional[torch.Tensor] = None):
    """Causal attention of packed prompts: q [L,H,T,D], k/v [L,Hkv,T,D] (bf16), row_off [S+1] i32, scale [L] f32
    -> (out [L,H,T,D], lse [L*H*T] f32: [L,H,n] of each sequence one behind the other).  Rows that belong to no sequence are
    left as they are."""
    stream = _here(q.get_device(), k, v, row_off, scale, out, lse, ws)
    out = torch.empty_like(q) if out is None else out
    S = row_off.numel() - 1
    s, qs, os_, need = _attn_args(q.shape, q.stride(), q.dtype, out.shape, out.stride(), out.dtype, S, k.shape[1], 0)
    ks, vs = _key_args(k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype, q.shape, q.dtype)
    L, H, T, _ = q.shape
    _i32_like(row_off, (S + 1,), "row_off")
    if scale.dtype is not torch.float32 or scale.shape != (L,) or not scale.is_contiguous():
        raise ValueError("scale must be contiguous f32 [L]")
    if lse is None:
        lse = torch.empty(L * H * T, dtype=torch.float32, device=q.device)
    elif lse.dtype is not torch.float32 or lse.numel() != L * H * T or not lse.is_contiguous():
        raise ValueError("lse must be contiguous f32 [L*H*T]")
    w = _ws(need, q.device, ws)
    rc = load().prefixkv_prefill_attn_packed(s, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, row_off.data_ptr(),
                                             scale.data_ptr(), out.data_ptr(), os_, lse.data_ptr(), w.data_ptr(),
                                             w.numel() * w.element_size(), stream)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_prefill_attn_packed")
    return out, lse


def prefixkv_chunk_attn(cache: PagedCache, q: torch.Tensor, row_off: torch.Tensor, scale: torch.Tensor, max_rows: int,
                        l0: int = 0, out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of new rows q [L,H,T,D] over the cache's layers l0 ... l0+L-1, which hold their keys and values already:
    row_off [S+1] i32, scale [L] f32, max_rows = the most rows of a sequence -> out [L,H,T,D]."""
    kp, vp, table, lens = cache.kp, cache.vp, cache.table, cache.lens
    stream = _here(cache._device, q, row_off, scale, out, ws)
    out = torch.empty_like(q) if out is None else out
    pool, max_rows = cache._pool, _c_int(index(max_rows), "max_rows")
    qsh = q.shape
    if pool is None or pool[1:] != (qsh[3], q.dtype):
        raise ValueError("the cache must have q's head dimension and dtype, and contiguous pools")
    s, qs, os_, need = _attn_args(qsh, q.stride(), q.dtype, out.shape, out.stride(), out.dtype, cache._S, pool[0], max_rows)
    _i32_like(row_off, cache._offs, "row_off")
    if scale.dtype is not torch.float32 or scale.shape != qsh[:1] or not scale.is_contiguous():
        raise ValueError("scale must be contiguous f32 [L]")
    w = _ws(need, q.device, ws)
    rc = load().prefixkv_chunk_attn(s, q.data_ptr(), qs, row_off.data_ptr(), cache._paging, _c_int(int(l0), "l0"), kp.data_ptr(),
                                    vp.data_ptr(), table.data_ptr(), lens.data_ptr(), scale.data_ptr(), max_rows,
                                    out.data_ptr(), os_, w.data_ptr(), w.numel() * w.element_size(), stream)
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_chunk_attn")
    return out


def prefixkv_calibration_copy(dst: torch.Tensor, src: torch.Tensor) -> None:
    """Plain copy kernel of src's size into dst (byte-counter calibration aid)."""
    _need_cuda(dst, src)
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() < nbytes:
        raise ValueError("dst too small")
    rc = load().prefixkv_calibration_copy(_ptr(dst), _ptr(src), nbytes, _stream())
    if rc != 0:
        raise PrefixKVError(rc, "prefixkv_calibration_copy")
