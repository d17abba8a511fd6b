"""Thin Python binding over libloki.so's C ABI (include/loki.h).

Argument marshalling only: torch supplies device memory and the stream, every
step of the path runs in the HIP kernels.  There is no CPU fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libloki.so")

LOKI_F32, LOKI_BF16 = 0, 1
SELECT_PER_QUERY_HEAD, SELECT_PER_KV_GROUP = 0, 1
PATH_SPLIT, PATH_FUSED, PATH_CLUSTER, PATH_MASK = 0x100, 0x200, 0x300, 0x300
WORKSPACE_ZEROED = 0x400
PROFILE_MAX_KERNELS = 8
ROTARY_NONE, ROTARY_LINEAR, ROTARY_BASE, ROTARY_BANDS, ROTARY_RAMP = 0, 1, 2, 3, 4


class LokiError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Layout(ctypes.Structure):
    """Mirror of ``loki_layout``."""

    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("D", ctypes.c_int32), ("d_split", ctypes.c_int32), ("S_cap", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class RotaryTensor(ctypes.Structure):
    """Mirror of ``loki_rotary_tensor``."""
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("in_batch", "in_token", "in_head", "out_batch", "out_token", "out_head")]


class RotaryArgs(ctypes.Structure):
    """Mirror of ``loki_rotary_args``."""
    _fields_ = [("q", RotaryTensor), ("k", RotaryTensor), ("v", RotaryTensor), ("positions", ctypes.c_void_p),
                ("rows", ctypes.c_void_p), ("frequencies", ctypes.c_void_p), ("n_rows", ctypes.c_int32),
                ("rotary_dims", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("inverse", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class EvictArgs(ctypes.Structure):
    """Mirror of ``loki_evict_args``."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("seq_lens", "weights", "klo", "khi", "v", "klo_out", "khi_out", "v_out",
                                               "weights_out", "lens_out", "out_idx", "page_table")] + [
        (n, ctypes.c_int32) for n in ("S_cap_out", "page_rows", "pages_per_seq", "n_pages")]


class CacheArgs(ctypes.Structure):
    """Mirror of ``loki_cache``."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scales", "v_scales", "page_table")] + [
        (n, ctypes.c_int32) for n in ("page_rows", "pages_per_seq", "n_pages")]


class SpanArgs(ctypes.Structure):
    """Mirror of ``loki_span_args``."""
    _fields_ = [("seq_lens", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("queries_per_seq", "window", "sinks")]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libloki.so (built by ``paper_2406_02542_amd.build``); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2406_02542_amd.build` "
            "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    LP = ctypes.POINTER(Layout)
    L.loki_version.restype = i32
    L.loki_version.argtypes = []
    L.loki_status_string.restype = ctypes.c_char_p
    L.loki_status_string.argtypes = [i32]
    L.loki_cache_bytes.restype = i32
    L.loki_cache_bytes.argtypes = [LP, ctypes.POINTER(sz), ctypes.POINTER(sz), ctypes.POINTER(sz)]
    L.loki_workspace_bytes.restype = i32
    L.loki_workspace_bytes.argtypes = [LP, i32, i32, i32, i32, ctypes.POINTER(sz)]
    L.loki_rotate_keys.restype = i32
    L.loki_rotate_keys.argtypes = [LP, vp, vp, vp, vp, i32, i32, vp]
    L.loki_rotate_keys_paged.restype = i32
    L.loki_rotate_keys_paged.argtypes = [LP, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]
    L.loki_decode_attn.restype = i32
    L.loki_decode_attn.argtypes = [LP, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp, vp, vp]
    L.loki_decode_attn_static.restype = i32
    L.loki_decode_attn_static.argtypes = [LP, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp]
    L.loki_decode_step.restype = i32
    L.loki_decode_step.argtypes = [LP, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, sz, vp, vp, vp]
    L.dense_decode_step.restype = i32
    L.dense_decode_step.argtypes = [LP, vp, vp, vp, i32, vp, vp, sz, vp, vp]
    L.loki_pca_attn.restype = i32
    L.loki_pca_attn.argtypes = [LP, vp, vp, vp, vp, i32, i32, vp, sz, vp, vp]
    L.loki_pca_workspace_bytes.restype = i32
    L.loki_pca_workspace_bytes.argtypes = [LP, ctypes.c_longlong, ctypes.POINTER(sz)]
    L.loki_pca_fit.restype = i32
    L.loki_pca_fit.argtypes = [LP, vp, ctypes.c_longlong, vp, vp, vp, sz, vp]
    L.loki_rank_at.restype = i32
    L.loki_rank_at.argtypes = [vp, i32, i32, ctypes.c_float, vp, vp]
    L.loki_layer_width.restype = i32
    L.loki_layer_width.argtypes = [vp, i32, i32, ctypes.c_float, i32, vp, vp, vp]
    L.loki_index_jaccard.restype = i32
    L.loki_index_jaccard.argtypes = [vp, vp, i32, i32, vp, vp]
    L.loki_rotary.restype = i32
    L.loki_rotary.argtypes = [LP, i32, vp, vp]
    L.loki_rotary_frequencies.restype = i32
    L.loki_rotary_frequencies.argtypes = [i32, ctypes.c_double, i32, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                          vp, ctypes.POINTER(ctypes.c_float)]
    L.dense_weights_workspace_bytes.restype = i32
    L.dense_weights_workspace_bytes.argtypes = [LP, i32, ctypes.POINTER(sz)]
    L.dense_decode_weights.restype = i32
    L.dense_decode_weights.argtypes = [LP, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp, vp]
    L.loki_evict_workspace_bytes.restype = i32
    L.loki_evict_workspace_bytes.argtypes = [LP, i32, i32, ctypes.POINTER(sz)]
    L.loki_evict.restype = i32
    L.loki_evict.argtypes = [LP, vp, i32, i32, i32, i32, vp, sz, vp]
    L.dense_shared_workspace_bytes.restype = i32
    L.dense_shared_workspace_bytes.argtypes = [LP, i32, i32, ctypes.POINTER(sz)]
    L.dense_decode_shared.restype = i32
    L.dense_decode_shared.argtypes = [LP, vp, vp, vp, i32, i32, vp, vp, i32, vp, vp, sz, vp, vp]
    CP, SP = ctypes.POINTER(CacheArgs), ctypes.POINTER(SpanArgs)
    L.loki_append.restype = i32
    L.loki_append.argtypes = [LP, CP, i32, vp, vp]
    L.loki_read_rows.restype = i32
    L.loki_read_rows.argtypes = [LP, CP, i32, vp, vp, vp, vp]
    L.dense_cache_workspace_bytes.restype = i32
    L.dense_cache_workspace_bytes.argtypes = [LP, CP, i32, SP, ctypes.POINTER(sz)]
    L.dense_decode_cache.restype = i32
    L.dense_decode_cache.argtypes = [LP, vp, CP, i32, SP, vp, sz, vp, vp]
    L.dense_decode_attn.restype = i32
    L.dense_decode_attn.argtypes = [LP, vp, vp, vp, i32, vp, sz, vp, vp]
    L.loki_profile_create.restype = i32
    L.loki_profile_create.argtypes = [ctypes.POINTER(vp)]
    L.loki_profile_destroy.restype = i32
    L.loki_profile_destroy.argtypes = [vp]
    L.loki_profile_attach.restype = i32
    L.loki_profile_attach.argtypes = [vp]
    L.loki_debug_cluster_spin_limit.restype = i32
    L.loki_debug_cluster_spin_limit.argtypes = [ctypes.c_uint]
    L.loki_debug_cluster_give_up_at_list.restype = i32
    L.loki_debug_cluster_give_up_at_list.argtypes = [i32]
    L.loki_debug_row_loads.restype = i32
    L.loki_debug_row_loads.argtypes = [LP, i32, i32, i32, i32, vp, ctypes.c_double, ctypes.c_double, ctypes.POINTER(i32)]
    L.loki_cluster_gave_up.restype = i32
    L.loki_cluster_gave_up.argtypes = [vp, ctypes.POINTER(i32), vp]
    L.loki_stream_read.restype = i32
    L.loki_stream_read.argtypes = [vp, sz, vp]
    L.loki_profile_read.restype = i32
    L.loki_profile_read.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_float),
                                    ctypes.POINTER(ctypes.c_char_p)]
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().loki_status_string(int(status)).decode()


def version() -> int:
    return lib().loki_version()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise LokiError(status, where)


def make_layout(B: int, Hq: int, Hkv: int, D: int, d_split: int, S_cap: int,
                dtype: torch.dtype) -> Layout:
    if dtype == torch.float32:
        code = LOKI_F32
    elif dtype == torch.bfloat16:
        code = LOKI_BF16
    else:
        raise ValueError(f"unsupported storage dtype {dtype}")
    return Layout(B, Hq, Hkv, D, d_split, S_cap, code)


def _torch_dtype(layout: Layout) -> torch.dtype:
    return torch.float32 if layout.dtype == LOKI_F32 else torch.bfloat16


def _ptr(t: Optional[torch.Tensor], name: str, dtype: Optional[torch.dtype] = None,
         numel: Optional[int] = None) -> Optional[int]:
    """Device pointer of a tensor after checking it is what the C side assumes."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, the call reads/writes {numel}")
    return t.data_ptr()


# torch.cuda.current_stream().cuda_stream without the Stream object, which took 2.6 of the 8.3 us that
# the host spends on a small loki_rotate_keys (0.2 without it).
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on_current_device(t: torch.Tensor, name: str) -> None:
    """Kernels run on the current device: one of another would read addresses that are not its own."""
    if _current_device is not None and t.get_device() != _current_device():
        raise ValueError(f"{name} must live on the current device ({_current_device()}), got {t.device}")


def _here() -> int:
    """The current device's number; where there is none, one that no tensor has (the host's have -1)."""
    try:
        return torch.cuda.current_device() if _current_device is None else _current_device()
    except RuntimeError:
        return -2


def _ptr_here(here: int, t: Optional[torch.Tensor], name: str, dtype: torch.dtype, numel: int = 0) -> Optional[int]:
    """``_ptr`` of a tensor of the current device."""
    if t is None:
        return None
    if t.get_device() == here and t.dtype is dtype and t.numel() >= numel and t.is_contiguous():
        return t.data_ptr()
    _ptr(t, name, dtype, numel)
    _refuse_device(here, t, name)


def _refuse_device(here: int, t: torch.Tensor, name: str) -> None:
    raise ValueError(f"{name} must live on the current device ({here}), got {t.device}")


def _stream_ptr(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _current_device is None or _current_raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _current_raw_stream(_current_device())


def loki_cache_bytes(layout: Layout):
    a, b, c = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().loki_cache_bytes(ctypes.byref(layout), ctypes.byref(a), ctypes.byref(b),
                                  ctypes.byref(c)), "loki_cache_bytes")
    return a.value, b.value, c.value


def loki_workspace_bytes(layout: Layout, S: int, d: int, k: int, select_mode: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().loki_workspace_bytes(ctypes.byref(layout), S, d, k, select_mode, ctypes.byref(n)),
           "loki_workspace_bytes")
    return n.value


def alloc_cache(layout: Layout, device="cuda"):
    """Allocates (klo, khi, v) tensors of the layout's shape (zero-filled)."""
    dt = _torch_dtype(layout)
    B, H, S, D, d = layout.B, layout.Hkv, layout.S_cap, layout.D, layout.d_split
    klo = torch.zeros((B, H, S, d), dtype=dt, device=device)
    khi = torch.zeros((B, H, S, D - d), dtype=dt, device=device) if d < D else None
    v = torch.zeros((B, H, S, D), dtype=dt, device=device)
    return klo, khi, v


def alloc_workspace(layout: Layout, S: int, d: int, k: int, select_mode: int,
                    device="cuda", zeroed: bool = False) -> torch.Tensor:
    """zeroed: a workspace filled with zeros, which the caller may then pass with WORKSPACE_ZEROED."""
    n = loki_workspace_bytes(layout, S, d, k, select_mode)
    make = torch.zeros if zeroed else torch.empty
    return make(max(n, 256), dtype=torch.uint8, device=device)


def loki_rotate_keys(layout: Layout, k_new: torch.Tensor, P: torch.Tensor, klo: torch.Tensor,
                     khi: Optional[torch.Tensor], pos: int, n_new: int, stream=None) -> None:
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv
    _check(lib().loki_rotate_keys(
        ctypes.byref(layout),
        _ptr(k_new, "k_new", dt, rows * n_new * layout.D),
        _ptr(P, "P", torch.float32, layout.Hkv * layout.D * layout.D),
        _ptr(klo, "klo", dt, rows * layout.S_cap * layout.d_split),
        _ptr(khi, "khi", dt, rows * layout.S_cap * (layout.D - layout.d_split)),
        pos, n_new, _stream_ptr(stream)), "loki_rotate_keys")


def loki_rotate_keys_paged(layout: Layout, k_new: torch.Tensor, P: torch.Tensor, klo: torch.Tensor,
                           khi: Optional[torch.Tensor], page_table: torch.Tensor, page_rows: int,
                           n_pages: int, pos: int, n_new: int, stream=None) -> None:
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv
    pool_rows = n_pages * layout.Hkv * page_rows
    _check(lib().loki_rotate_keys_paged(
        ctypes.byref(layout),
        _ptr(k_new, "k_new", dt, rows * n_new * layout.D),
        _ptr(P, "P", torch.float32, layout.Hkv * layout.D * layout.D),
        _ptr(klo, "klo", dt, pool_rows * layout.d_split),
        _ptr(khi, "khi", dt, pool_rows * (layout.D - layout.d_split)),
        _ptr(page_table, "page_table", torch.int32, layout.B),
        page_rows, page_table.numel() // layout.B, n_pages, pos, n_new,
        _stream_ptr(stream)), "loki_rotate_keys_paged")


def loki_decode_attn(layout: Layout, q: torch.Tensor, P: torch.Tensor, klo: torch.Tensor,
                     khi: Optional[torch.Tensor], v: torch.Tensor, S: int, d: int, k: int,
                     select_mode: int, workspace: torch.Tensor, out: torch.Tensor,
                     out_idx: Optional[torch.Tensor] = None, stream=None) -> None:
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv
    nq = layout.B * layout.Hq * layout.D
    hsel = layout.Hq if (select_mode & ~(PATH_MASK | WORKSPACE_ZEROED)) == SELECT_PER_QUERY_HEAD else layout.Hkv
    _check(lib().loki_decode_attn(
        ctypes.byref(layout),
        _ptr(q, "q", dt, nq),
        _ptr(P, "P", torch.float32, layout.Hkv * layout.D * layout.D),
        _ptr(klo, "klo", dt, rows * layout.S_cap * layout.d_split),
        _ptr(khi, "khi", dt, rows * layout.S_cap * (layout.D - layout.d_split)),
        _ptr(v, "v", dt, rows * layout.S_cap * layout.D),
        S, d, k, select_mode,
        _ptr(workspace, "workspace", torch.uint8), workspace.numel(),
        _ptr(out, "out", dt, nq),
        _ptr(out_idx, "out_idx", torch.int32, layout.B * hsel * k),
        _stream_ptr(stream)), "loki_decode_attn")


STATIC_SCRATCH_BYTES = 64 << 20


def loki_decode_attn_static(layout: Layout, q: torch.Tensor, P: torch.Tensor, klo: torch.Tensor,
                            khi: Optional[torch.Tensor], v: torch.Tensor, S: int, d: int, k: int,
                            select_mode: int, out: torch.Tensor,
                            out_idx: Optional[torch.Tensor] = None, stream=None) -> None:
    """loki_decode_attn on the library's built-in scratch buffer (no workspace argument)."""
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv
    nq = layout.B * layout.Hq * layout.D
    hsel = layout.Hq if (select_mode & ~(PATH_MASK | WORKSPACE_ZEROED)) == SELECT_PER_QUERY_HEAD else layout.Hkv
    _check(lib().loki_decode_attn_static(
        ctypes.byref(layout),
        _ptr(q, "q", dt, nq),
        _ptr(P, "P", torch.float32, layout.Hkv * layout.D * layout.D),
        _ptr(klo, "klo", dt, rows * layout.S_cap * layout.d_split),
        _ptr(khi, "khi", dt, rows * layout.S_cap * (layout.D - layout.d_split)),
        _ptr(v, "v", dt, rows * layout.S_cap * layout.D),
        S, d, k, select_mode,
        _ptr(out, "out", dt, nq),
        _ptr(out_idx, "out_idx", torch.int32, layout.B * hsel * k),
        _stream_ptr(stream)), "loki_decode_attn_static")


class StepArgs(ctypes.Structure):
    """Mirror of ``loki_step_args``."""
    _fields_ = [("seq_lens", ctypes.c_void_p), ("ks", ctypes.c_void_p),
                ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p),
                ("queries_per_seq", ctypes.c_int32), ("page_rows", ctypes.c_int32),
                ("page_table", ctypes.c_void_p), ("pages_per_seq", ctypes.c_int32),
                ("n_pages", ctypes.c_int32)]


def loki_decode_step(layout: Layout, q: torch.Tensor, P: torch.Tensor, klo: torch.Tensor,
                     khi: Optional[torch.Tensor], v: torch.Tensor, S_max: int, d: int, k_max: int,
                     select_mode: int, workspace: torch.Tensor, out: torch.Tensor,
                     out_idx: Optional[torch.Tensor] = None, seq_lens: Optional[torch.Tensor] = None,
                     ks: Optional[torch.Tensor] = None, k_new: Optional[torch.Tensor] = None,
                     v_new: Optional[torch.Tensor] = None, queries_per_seq: int = 1,
                     page_table: Optional[torch.Tensor] = None, page_rows: int = 0,
                     n_pages: int = 0, stream=None) -> None:
    """With ``page_table`` [B, pages_per_seq] (int32), ``klo``/``khi``/``v`` are the paged
    pools [n_pages, Hkv, page_rows, width]."""
    dt = _torch_dtype(layout)
    m = max(1, queries_per_seq)
    rows = layout.B * layout.Hkv
    nq = layout.B * m * layout.Hq * layout.D
    hsel = layout.Hq if (select_mode & ~(PATH_MASK | WORKSPACE_ZEROED)) == SELECT_PER_QUERY_HEAD else layout.Hkv
    args = StepArgs(
        _ptr(seq_lens, "seq_lens", torch.int32, layout.B * m),
        _ptr(ks, "ks", torch.int32, layout.B * m),
        _ptr(k_new, "k_new", dt, rows * m * layout.D),
        _ptr(v_new, "v_new", dt, rows * m * layout.D),
        queries_per_seq, page_rows,
        _ptr(page_table, "page_table", torch.int32, layout.B),
        (page_table.numel() // layout.B) if page_table is not None else 0, n_pages)
    cache_rows = (n_pages * layout.Hkv * page_rows) if page_table is not None else rows * layout.S_cap
    _check(lib().loki_decode_step(
        ctypes.byref(layout),
        _ptr(q, "q", dt, nq),
        _ptr(P, "P", torch.float32, layout.Hkv * layout.D * layout.D),
        _ptr(klo, "klo", dt, cache_rows * layout.d_split),
        _ptr(khi, "khi", dt, cache_rows * (layout.D - layout.d_split)),
        _ptr(v, "v", dt, cache_rows * layout.D),
        S_max, d, k_max, select_mode, ctypes.byref(args),
        _ptr(workspace, "workspace", torch.uint8), workspace.numel(),
        _ptr(out, "out", dt, nq),
        _ptr(out_idx, "out_idx", torch.int32, layout.B * m * hsel * k_max),
        _stream_ptr(stream)), "loki_decode_step")


def dense_decode_step(layout: Layout, q: torch.Tensor, k_full: torch.Tensor, v: torch.Tensor,
                      S_max: int, seq_lens: Optional[torch.Tensor],
                      workspace: Optional[torch.Tensor], out: torch.Tensor, stream=None) -> None:
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv
    nq = layout.B * layout.Hq * layout.D
    _check(lib().dense_decode_step(
        ctypes.byref(layout),
        _ptr(q, "q", dt, nq),
        _ptr(k_full, "k_full", dt, rows * layout.S_cap * layout.D),
        _ptr(v, "v", dt, rows * layout.S_cap * layout.D),
        S_max,
        _ptr(seq_lens, "seq_lens", torch.int32, layout.B),
        _ptr(workspace, "workspace", torch.uint8),
        workspace.numel() if workspace is not None else 0,
        _ptr(out, "out", dt, nq),
        _stream_ptr(stream)), "dense_decode_step")


def dense_decode_attn(layout: Layout, q: torch.Tensor, k_full: torch.Tensor, v: torch.Tensor,
                      S: int, workspace: Optional[torch.Tensor], out: torch.Tensor,
                      stream=None) -> None:
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv
    nq = layout.B * layout.Hq * layout.D
    _check(lib().dense_decode_attn(
        ctypes.byref(layout),
        _ptr(q, "q", dt, nq),
        _ptr(k_full, "k_full", dt, rows * layout.S_cap * layout.D),
        _ptr(v, "v", dt, rows * layout.S_cap * layout.D),
        S,
        _ptr(workspace, "workspace", torch.uint8),
        workspace.numel() if workspace is not None else 0,
        _ptr(out, "out", dt, nq),
        _stream_ptr(stream)), "dense_decode_attn")


def loki_rotary_frequencies(rotary_dims: int, base: float = 10000.0, scaling: int = ROTARY_NONE, factor: float = 1.0,
                            original_context: float = 0.0, low: float = 0.0, high: float = 0.0, device="cuda"):
    """(frequencies, scale): the fp64 tensor [rotary_dims / 2] that ``loki_rotary`` takes, and its scale."""
    f = torch.empty(max(int(rotary_dims), 2) // 2, dtype=torch.float64)
    scale = ctypes.c_float(1.0)
    _check(lib().loki_rotary_frequencies(rotary_dims, base, scaling, factor, original_context, low, high, f.data_ptr(),
                                         ctypes.byref(scale)), "loki_rotary_frequencies")
    return f.to(device), scale.value


def _refuse_rotary(name: str, x: torch.Tensor, y: Optional[torch.Tensor], shape, out_shape, dt: torch.dtype) -> None:
    if y is None:
        raise ValueError(f"{name} needs its output")
    if not (x.is_cuda and y.is_cuda):
        raise ValueError(f"{name} must live on the GPU")
    if x.dtype != dt or y.dtype != dt:
        raise ValueError(f"{name} must have dtype {dt}, got {x.dtype} and {y.dtype}")
    if x.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {tuple(x.shape)}")
    if y.shape != out_shape:
        raise ValueError(f"{name}'s output must be {list(out_shape)}, got {tuple(y.shape)}")
    raise ValueError(f"{name}: the columns of a row must be next to each other")


_NOT_THERE = (0,) * 8


def _rotary_tensor(name: str, x: Optional[torch.Tensor], y: Optional[torch.Tensor], shape, out_shape, dt: torch.dtype, head_major: bool):
    """The members of a ``loki_rotary_tensor``: x [B, n, heads, D] to y, of the same shape or head-major
    [B, heads, rows, D], both with any strides of whole rows."""
    if x is None:
        if y is not None:
            raise ValueError(f"{name}_out without {name}")
        return _NOT_THERE
    if y is not None and x.is_cuda and y.is_cuda and x.dtype is dt and y.dtype is dt and x.shape == shape and y.shape == out_shape:
        ib, it, ih, ic = x.stride()
        ob, ot, oh, oc = y.stride()
        if ic == 1 and oc == 1:
            return (x.data_ptr(), y.data_ptr(), ib, it, ih, ob, oh, ot) if head_major else (x.data_ptr(), y.data_ptr(), ib, it, ih, ob, ot, oh)
    _refuse_rotary(name, x, y, shape, out_shape, dt)


_rotary_pack = struct.Struct("PPqqqqqq" * 3 + "PPPiiiif4x").pack  # RotaryArgs, filled in one go


def loki_rotary(layout: Layout, positions: torch.Tensor, frequencies: torch.Tensor, q: Optional[torch.Tensor] = None,
                q_out: Optional[torch.Tensor] = None, k: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                v: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
                interleaved: bool = False, inverse: bool = False, scale: float = 1.0, token_major: bool = False,
                stream=None) -> None:
    """Rotary positions: ``q``, ``k``, ``v`` [B, n, heads, D] with any strides of whole rows (slices of one
    projection's output, for instance), ``q_out`` the same shape, ``k_out`` and ``v_out`` [B, Hkv, n, D] as
    ``loki_rotate_keys`` takes them, or with ``rows`` [B, n] the caches [B, Hkv, S_cap, D]; token_major:
    [B, n, Hkv, D], as ``loki_decode_step`` takes its new tokens (and in place, given the inputs)."""
    B, n = positions.shape
    if B != layout.B:
        raise ValueError(f"positions must be [{layout.B}, n], got {tuple(positions.shape)}")
    dt = _torch_dtype(layout)
    Hq, H = layout.Hq, layout.Hkv
    n_rows = n
    if rows is not None:
        out = k_out if k_out is not None else v_out
        if out is None or token_major:
            raise ValueError("rows are those of a head-major key or value output")
        n_rows = out.shape[2]
    q_shape, shape = (B, n, Hq, 128), (B, n, H, 128)
    out_shape = shape if token_major else (B, H, n_rows, 128)
    args = _rotary_pack(
        *_rotary_tensor("q", q, q_out, q_shape, q_shape, dt, False),
        *_rotary_tensor("k", k, k_out, shape, out_shape, dt, not token_major),
        *_rotary_tensor("v", v, v_out, shape, out_shape, dt, not token_major),
        _ptr(positions, "positions", torch.int32, 1),
        0 if rows is None else _ptr(rows, "rows", torch.int32, B * n),
        _ptr(frequencies, "frequencies", torch.float64, 1),
        n_rows, 2 * frequencies.numel(), interleaved, inverse, scale)
    _on_current_device(positions, "positions")
    _check(lib().loki_rotary(ctypes.byref(layout), n, args, _stream_ptr(stream)), "loki_rotary")


def dense_weights_workspace_bytes(layout: Layout, S_max: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().dense_weights_workspace_bytes(ctypes.byref(layout), S_max, ctypes.byref(n)), "dense_weights_workspace_bytes")
    return n.value


def dense_decode_weights(layout: Layout, q: torch.Tensor, k_full: torch.Tensor, v: torch.Tensor, S_max: int,
                         seq_lens: Optional[torch.Tensor], weights_in: Optional[torch.Tensor], weights_out: torch.Tensor,
                         workspace: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """``dense_decode_step`` that adds every row's softmax weight to its running total [B, Hkv, S_cap].  A new row's total
    begins with what ``weights_in`` holds there: set it to zero with the append, for instance
    ``weights.scatter_(2, rows.long()[:, None, None].expand(-1, Hkv, 1), 0.0)`` for the rows [B] that are written."""
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv * layout.S_cap
    nq = layout.B * layout.Hq * layout.D
    q_ptr = _ptr(q, "q", dt, nq)
    _on_current_device(q, "q")
    _check(lib().dense_decode_weights(
        ctypes.byref(layout),
        q_ptr,
        _ptr(k_full, "k_full", dt, rows * layout.D),
        _ptr(v, "v", dt, rows * layout.D),
        S_max,
        _ptr(seq_lens, "seq_lens", torch.int32, layout.B),
        _ptr(weights_in, "weights_in", torch.float32, rows),
        _ptr(weights_out, "weights_out", torch.float32, rows),
        _ptr(workspace, "workspace", torch.uint8), workspace.numel(),
        _ptr(out, "out", dt, nq),
        _stream_ptr(stream)), "dense_decode_weights")


def loki_evict_workspace_bytes(layout: Layout, S_max: int, budget: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().loki_evict_workspace_bytes(ctypes.byref(layout), S_max, budget, ctypes.byref(n)), "loki_evict_workspace_bytes")
    return n.value


def _refuse_rows(units: int, rows: int, *parts) -> None:
    """Every part (name, tensor or None, width) of a cache has to hold exactly `rows` rows for each unit: one stride goes for all."""
    for name, t, width in parts:
        if t is not None and t.numel() != units * rows * width:
            raise ValueError(f"{name} holds {t.numel()} elements, {rows} rows of {width} for {units} heads have {units * rows * width}")


_evict_pack = struct.Struct("P" * 12 + "iiii").pack  # EvictArgs


def loki_evict(layout: Layout, weights: torch.Tensor, klo: torch.Tensor, khi: Optional[torch.Tensor], v: torch.Tensor,
               S_max: int, budget: int, sinks: int, recent: int, workspace: torch.Tensor,
               seq_lens: Optional[torch.Tensor] = None, klo_out: Optional[torch.Tensor] = None,
               khi_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None,
               weights_out: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
               out_idx: Optional[torch.Tensor] = None, page_table: Optional[torch.Tensor] = None, page_rows: int = 0,
               n_pages: int = 0, stream=None) -> None:
    """Without ``klo_out`` in place; else the kept rows go to [B, Hkv, S_cap_out, width] caches.  An unsplit cache
    (layout.d_split == D): ``klo`` holds the keys, ``khi`` is None.  With ``page_table`` the cache is paged."""
    dt = _torch_dtype(layout)
    units, D, d = layout.B * layout.Hkv, layout.D, layout.d_split
    cache_rows = (n_pages * layout.Hkv * page_rows) if page_table is not None else units * layout.S_cap
    cap_out = klo_out.numel() // (units * d) if klo_out is not None else 0
    if klo_out is not None:
        rows = units * cap_out
        if (klo_out.numel() != rows * d or (v_out is not None and v_out.numel() != rows * D) or
                (weights_out is not None and weights_out.numel() != rows) or
                (khi_out is not None and d < D and khi_out.numel() != rows * (D - d))):
            _refuse_rows(units, cap_out, ("klo_out", klo_out, d), ("khi_out", khi_out if d < D else None, D - d), ("v_out", v_out, D),
                         ("weights_out", weights_out, 1))
    args = _evict_pack(
        _ptr(seq_lens, "seq_lens", torch.int32, layout.B) or 0,
        _ptr(weights, "weights", torch.float32, units * layout.S_cap),
        _ptr(klo, "klo", dt, cache_rows * d),
        _ptr(khi, "khi", dt, cache_rows * (D - d)) or 0,
        _ptr(v, "v", dt, cache_rows * D),
        _ptr(klo_out, "klo_out", dt, units * cap_out * d) or 0,
        _ptr(khi_out, "khi_out", dt, units * cap_out * (D - d)) or 0,
        _ptr(v_out, "v_out", dt, units * cap_out * D) or 0,
        _ptr(weights_out, "weights_out", torch.float32, units * cap_out) or 0,
        _ptr(lens_out, "lens_out", torch.int32, layout.B) or 0,
        _ptr(out_idx, "out_idx", torch.int32, units * budget) or 0,
        _ptr(page_table, "page_table", torch.int32, layout.B) or 0,
        cap_out, page_rows, (page_table.numel() // layout.B) if page_table is not None else 0, n_pages)
    _on_current_device(weights, "weights")
    _check(lib().loki_evict(ctypes.byref(layout), args, S_max, budget, sinks, recent,
                            _ptr(workspace, "workspace", torch.uint8), workspace.numel(), _stream_ptr(stream)), "loki_evict")


def dense_shared_workspace_bytes(layout: Layout, prefix_rows: int, S_max: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().dense_shared_workspace_bytes(ctypes.byref(layout), prefix_rows, S_max, ctypes.byref(n)),
           "dense_shared_workspace_bytes")
    return n.value


def dense_decode_shared(layout: Layout, q: torch.Tensor, k_prefix: Optional[torch.Tensor], v_prefix: Optional[torch.Tensor],
                        prefix_rows: int, k_full: Optional[torch.Tensor], v: Optional[torch.Tensor], S_max: int,
                        seq_lens: Optional[torch.Tensor], workspace: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """``dense_decode_step`` behind a prefix [Hkv, prefix_cap, D] that all sequences share."""
    dt = _torch_dtype(layout)
    H, D = layout.Hkv, layout.D
    rows = layout.B * H * layout.S_cap if S_max > 0 else 0
    nq = layout.B * layout.Hq * D
    if (k_prefix is None) != (v_prefix is None):
        raise ValueError("k_prefix and v_prefix go together")
    cap = k_prefix.numel() // (H * D) if k_prefix is not None else 0
    if k_prefix is not None and (k_prefix.numel() != H * cap * D or v_prefix.numel() != H * cap * D):
        _refuse_rows(H, cap, ("k_prefix", k_prefix, D), ("v_prefix", v_prefix, D))
    q_ptr = _ptr(q, "q", dt, nq)
    _on_current_device(q, "q")
    _check(lib().dense_decode_shared(
        ctypes.byref(layout),
        q_ptr,
        _ptr(k_prefix, "k_prefix", dt, H * cap * D),
        _ptr(v_prefix, "v_prefix", dt, H * cap * D),
        prefix_rows, cap,
        _ptr(k_full, "k_full", dt, rows * D),
        _ptr(v, "v", dt, rows * D),
        S_max,
        _ptr(seq_lens, "seq_lens", torch.int32, layout.B),
        _ptr(workspace, "workspace", torch.uint8), workspace.numel(),
        _ptr(out, "out", dt, nq),
        _stream_ptr(stream)), "dense_decode_shared")


def loki_pca_attn(layout: Layout, q: torch.Tensor, P: torch.Tensor, klo: torch.Tensor,
                  v: torch.Tensor, S: int, d: int, workspace: torch.Tensor, out: torch.Tensor,
                  stream=None) -> None:
    dt = _torch_dtype(layout)
    rows = layout.B * layout.Hkv
    nq = layout.B * layout.Hq * layout.D
    _check(lib().loki_pca_attn(
        ctypes.byref(layout),
        _ptr(q, "q", dt, nq),
        _ptr(P, "P", torch.float32, layout.Hkv * layout.D * layout.D),
        _ptr(klo, "klo", dt, rows * layout.S_cap * layout.d_split),
        _ptr(v, "v", dt, rows * layout.S_cap * layout.D),
        S, d,
        _ptr(workspace, "workspace", torch.uint8), workspace.numel(),
        _ptr(out, "out", dt, nq),
        _stream_ptr(stream)), "loki_pca_attn")


def loki_pca_workspace_bytes(layout: Layout, n_rows: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().loki_pca_workspace_bytes(ctypes.byref(layout), n_rows, ctypes.byref(n)),
           "loki_pca_workspace_bytes")
    return n.value


def loki_pca_fit(layout: Layout, keys: torch.Tensor, n_rows: int, P: torch.Tensor,
                 eigenvalues: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    dt = _torch_dtype(layout)
    _check(lib().loki_pca_fit(
        ctypes.byref(layout),
        _ptr(keys, "keys", dt, layout.Hkv * n_rows * layout.D), n_rows,
        _ptr(P, "P", torch.float32, layout.Hkv * layout.D * layout.D),
        _ptr(eigenvalues, "eigenvalues", torch.float32, layout.Hkv * layout.D),
        _ptr(workspace, "workspace", torch.uint8), workspace.numel(),
        _stream_ptr(stream)), "loki_pca_fit")


def loki_rank_at(eigenvalues: torch.Tensor, v_percent: float, ranks: torch.Tensor, stream=None) -> None:
    n, D = eigenvalues.shape
    _check(lib().loki_rank_at(_ptr(eigenvalues, "eigenvalues", torch.float32, n * D), n, D, v_percent,
                              _ptr(ranks, "ranks", torch.int32, n), _stream_ptr(stream)), "loki_rank_at")


def loki_layer_width(eigenvalues: torch.Tensor, v_percent: float, multiple: int,
                     mean_rank: Optional[torch.Tensor], d_out: torch.Tensor, stream=None) -> None:
    n, D = eigenvalues.shape
    _check(lib().loki_layer_width(_ptr(eigenvalues, "eigenvalues", torch.float32, n * D), n, D, v_percent,
                                  multiple, _ptr(mean_rank, "mean_rank", torch.float32, 1),
                                  _ptr(d_out, "d_out", torch.int32, 1), _stream_ptr(stream)),
           "loki_layer_width")


def loki_index_jaccard(idx_a: torch.Tensor, idx_b: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    k = idx_a.shape[-1]
    n = idx_a.numel() // k
    _check(lib().loki_index_jaccard(_ptr(idx_a, "idx_a", torch.int32, n * k),
                                    _ptr(idx_b, "idx_b", torch.int32, n * k), n, k,
                                    _ptr(out, "out", torch.float32, n), _stream_ptr(stream)),
           "loki_index_jaccard")


def loki_debug_cluster_spin_limit(polls: int) -> None:
    """Sets how many polls a block of a PATH_CLUSTER launch waits for its unit's other blocks
    (0 restores the default)."""
    _check(lib().loki_debug_cluster_spin_limit(int(polls)), "loki_debug_cluster_spin_limit")


def loki_debug_cluster_give_up_at_list(on: bool) -> None:
    """Makes the blocks of PATH_CLUSTER launches give up at the list of candidates (until switched off)."""
    _check(lib().loki_debug_cluster_give_up_at_list(int(on)), "loki_debug_cluster_give_up_at_list")


def loki_debug_row_loads(layout: Layout, S_max: int, d: int, k_max: int, select_mode: int, args: Optional[StepArgs] = None,
                         rows: float = 0.0, kept: float = 0.0) -> int:
    """How a call loads its rows: 0 through the caches, 1 past them, 2 a group's slab too (see the header)."""
    form = ctypes.c_int32(0)
    _check(lib().loki_debug_row_loads(ctypes.byref(layout), S_max, d, k_max, select_mode,
                                      None if args is None else ctypes.byref(args), float(rows), float(kept),
                                      ctypes.byref(form)), "loki_debug_row_loads")
    return form.value


def loki_cluster_gave_up(workspace: torch.Tensor, stream=None) -> bool:
    """True if a PATH_CLUSTER launch on this workspace gave up waiting since its control words
    were last cleared (synchronises with the stream)."""
    flag = ctypes.c_int32(0)
    _check(lib().loki_cluster_gave_up(ctypes.c_void_p(workspace.data_ptr()), ctypes.byref(flag),
                                      _stream_ptr(stream)), "loki_cluster_gave_up")
    return bool(flag.value)


def loki_stream_read(buf: torch.Tensor, nbytes: int, stream=None) -> None:
    """Enqueues the library's trivial read kernel over the first ``nbytes`` bytes of ``buf``."""
    if not buf.is_cuda or not buf.is_contiguous() or nbytes > buf.numel() * buf.element_size():
        raise ValueError("buf must be a contiguous device tensor of at least nbytes bytes")
    _check(lib().loki_stream_read(ctypes.c_void_p(buf.data_ptr()), nbytes, _stream_ptr(stream)),
           "loki_stream_read")


class Profile:
    """Owns a ``loki_profile``; while attached, every library call made from this
    thread records HIP events around each kernel it launches."""

    def __init__(self):
        h = ctypes.c_void_p()
        _check(lib().loki_profile_create(ctypes.byref(h)), "loki_profile_create")
        self._h = h

    def attach(self):
        _check(lib().loki_profile_attach(self._h), "loki_profile_attach")

    @staticmethod
    def detach():
        _check(lib().loki_profile_attach(None), "loki_profile_attach")

    def read(self):
        """[(kernel name, milliseconds)] of the most recent profiled call."""
        n = ctypes.c_int()
        ms = (ctypes.c_float * PROFILE_MAX_KERNELS)()
        names = (ctypes.c_char_p * PROFILE_MAX_KERNELS)()
        _check(lib().loki_profile_read(self._h, ctypes.byref(n), ms, names), "loki_profile_read")
        return [(names[i].decode(), float(ms[i])) for i in range(n.value)]

    def close(self):
        if self._h is not None:
            lib().loki_profile_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Cache:
    """A cache held whole (``loki_cache``), checked once and kept with its tensors (another page table is another ``Cache``; its
    entries may change): ``k``, ``v`` [B, Hkv, S_cap, 128] of the
    layout's type or, with ``page_table`` [B, pages_per_seq] (int32), pools [n_pages, Hkv, page_rows, 128]; in 4 bits int32
    [.., 16] with ``k_scales``, ``v_scales`` fp16 [.., 4, 2].  See ``alloc_whole_cache``."""

    def __init__(self, layout: Layout, k: torch.Tensor, v: torch.Tensor, k_scales: Optional[torch.Tensor] = None,
                 v_scales: Optional[torch.Tensor] = None, page_table: Optional[torch.Tensor] = None):
        if (k_scales is None) != (v_scales is None):
            raise ValueError("k_scales and v_scales come together")
        dt, tail = (_torch_dtype(layout), (128,)) if k_scales is None else (torch.int32, (16,))
        B, H = layout.B, layout.Hkv
        pages = rows = per_seq = 0
        if page_table is not None:
            if page_table.dim() != 2 or page_table.shape[0] != B:
                raise ValueError(f"page_table must be [{B}, pages_per_seq], got {tuple(page_table.shape)}")
            if k.dim() != 4:
                raise ValueError(f"k must be [n_pages, {H}, page_rows, {tail[0]}], got {tuple(k.shape)}")
            (pages, rows), per_seq = (k.shape[0], k.shape[2]), page_table.shape[1]
        shape = (pages, H, rows) if page_table is not None else (B, H, layout.S_cap)
        parts = [("k", k, dt, shape + tail), ("v", v, dt, shape + tail)]
        if k_scales is not None:
            parts += [(n, t, torch.float16, shape + (4, 2)) for n, t in (("k_scales", k_scales), ("v_scales", v_scales))]
        for name, t, want, size in parts:
            if t.shape != size:
                raise ValueError(f"{name} must be {list(size)}, got {tuple(t.shape)}")
        if page_table is not None:
            parts.append(("page_table", page_table, torch.int32, page_table.shape))
        for name, t, want, _ in parts:
            _ptr(t, name, want)
            if t.get_device() != k.get_device():
                raise ValueError(f"{name} and k must live on the same device")
        self.tensors = (k, v, k_scales, v_scales, page_table)
        self.k = k
        self.args = CacheArgs(*(None if t is None else t.data_ptr() for t in self.tensors), rows, per_seq, pages)
        self.shape = (B, H, layout.S_cap, layout.dtype)
        self.ref = ctypes.byref(self.args)

    def _of(self, layout: Layout):
        if self.shape != (layout.B, layout.Hkv, layout.S_cap, layout.dtype):
            raise ValueError(f"the cache is one of (B, Hkv, S_cap, dtype) = {self.shape}")
        _on_current_device(self.k, "cache")
        return self.ref


def alloc_whole_cache(layout: Layout, four_bits: bool = False, page_table: Optional[torch.Tensor] = None, page_rows: int = 0,
                      n_pages: int = 0, device="cuda") -> Cache:
    """A ``Cache`` of the layout (zero-filled), contiguous or as pools of ``n_pages`` pages."""
    lead = (layout.B, layout.Hkv, layout.S_cap) if page_table is None else (n_pages, layout.Hkv, page_rows)
    make = lambda tail, dt: torch.zeros(lead + tail, dtype=dt, device=device)
    if not four_bits:
        return Cache(layout, make((128,), _torch_dtype(layout)), make((128,), _torch_dtype(layout)), page_table=page_table)
    return Cache(layout, make((16,), torch.int32), make((16,), torch.int32), make((4, 2), torch.float16),
                 make((4, 2), torch.float16), page_table=page_table)


def _refuse_strided(here: int, name: str, x: torch.Tensor, shape, dt: torch.dtype):
    if not x.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if x.get_device() != here:
        _refuse_device(here, x, name)
    if x.dtype is not dt or x.shape != shape:
        raise ValueError(f"{name} must be {list(shape)} of {dt}, got {tuple(x.shape)} of {x.dtype}")
    raise ValueError(f"{name}: the columns of a row must be next to each other")


def _strided(here: int, names, x: torch.Tensor, y: torch.Tensor, shape, dt: torch.dtype):
    """(pointer, strides of a batch, a token and a head) of x, and of y, [B, n, heads, D], rows of whole columns, of the current device."""
    if x.get_device() == here and y.get_device() == here and x.dtype is dt and y.dtype is dt and x.shape == shape and y.shape == shape:
        xb, xt, xh, xc = x.stride()
        yb, yt, yh, yc = y.stride()
        if xc == 1 and yc == 1:
            return x.data_ptr(), xb, xt, xh, y.data_ptr(), yb, yt, yh
    x_right = x.get_device() == here and x.dtype is dt and x.shape == shape and x.stride(3) == 1
    _refuse_strided(here, names[x_right], (x, y)[x_right], shape, dt)


def loki_append(layout: Layout, cache: Cache, rows: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                positions: Optional[torch.Tensor] = None, frequencies: Optional[torch.Tensor] = None,
                q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, interleaved: bool = False,
                inverse: bool = False, scale: float = 1.0, stream=None) -> None:
    """Tokens' ``k``, ``v`` [B, n, Hkv, D] (any strides of whole rows) into the rows ``rows`` [B, n] of the cache, ``k`` and ``q``
    [B, n, Hq, D] turned by ``positions`` [B, n] (as ``loki_rotary``; without ``frequencies`` nothing is turned)."""
    if rows.dim() != 2 or rows.shape[0] != layout.B:
        raise ValueError(f"rows must be [{layout.B}, n], got {tuple(rows.shape)}")
    B, n = rows.shape
    dt = _torch_dtype(layout)
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    if (positions is None) != (frequencies is None):
        raise ValueError("positions and frequencies come together")
    here = _here()
    kp, kb, kt, kh, vp, vb, vt, vh = _strided(here, ("k", "v"), k, v, (B, n, layout.Hkv, 128), dt)
    qp = qb = qt = qh = op = ob = ot = oh = pos = freq = R = 0
    if q is not None:
        qp, qb, qt, qh, op, ob, ot, oh = _strided(here, ("q", "q_out"), q, q_out, (B, n, layout.Hq, 128), dt)
    if frequencies is not None:
        pos, freq = _ptr_here(here, positions, "positions", torch.int32, B * n), _ptr_here(here, frequencies, "frequencies", torch.float64, 1)
        R = 2 * frequencies.numel()
    args = _rotary_pack(qp, op, qb, qt, qh, ob, ot, oh, kp, 0, kb, kt, kh, 0, 0, 0, vp, 0, vb, vt, vh, 0, 0, 0, pos,
                        _ptr_here(here, rows, "rows", torch.int32), freq, 0, R, interleaved, inverse, scale)
    cache_args = cache._of(layout)
    _check(lib().loki_append(ctypes.byref(layout), cache_args, n, args, _stream_ptr(stream)), "loki_append")


def loki_read_rows(layout: Layout, cache: Cache, rows: torch.Tensor, k_out: Optional[torch.Tensor] = None,
                   v_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Rows ``rows`` [B, n] of the cache to ``k_out``, ``v_out`` [B, Hkv, n, D]."""
    if rows.dim() != 2 or rows.shape[0] != layout.B:
        raise ValueError(f"rows must be [{layout.B}, n], got {tuple(rows.shape)}")
    n = rows.shape[1]
    dt, need = _torch_dtype(layout), layout.B * layout.Hkv * n * 128
    cache_args, here = cache._of(layout), _here()
    _check(lib().loki_read_rows(ctypes.byref(layout), cache_args, n, _ptr_here(here, rows, "rows", torch.int32),
                                _ptr_here(here, k_out, "k_out", dt, need), _ptr_here(here, v_out, "v_out", dt, need),
                                _stream_ptr(stream)), "loki_read_rows")


def dense_cache_workspace_bytes(layout: Layout, cache: Cache, S_max: int, queries_per_seq: int = 1, window: int = 0, sinks: int = 0) -> int:
    n = ctypes.c_size_t()
    args = SpanArgs(None, queries_per_seq, window, sinks)
    _check(lib().dense_cache_workspace_bytes(ctypes.byref(layout), cache._of(layout), S_max, ctypes.byref(args), ctypes.byref(n)),
           "dense_cache_workspace_bytes")
    return n.value


def dense_decode_cache(layout: Layout, cache: Cache, q: torch.Tensor, S_max: int, workspace: torch.Tensor, out: torch.Tensor,
                       seq_lens: Optional[torch.Tensor] = None, queries_per_seq: int = 1, window: int = 0, sinks: int = 0,
                       stream=None) -> None:
    """Attention of ``q`` [B, m, Hq, D] over the cache's rows, or with ``window`` over the last of them and the first ``sinks``;
    ``seq_lens`` [B, m] (int32): the rows that every token sees, itself the last, 0 for a padded one."""
    dt = _torch_dtype(layout)
    m = max(1, queries_per_seq)
    nq = layout.B * m * layout.Hq * layout.D
    here = _here()
    args = SpanArgs(_ptr_here(here, seq_lens, "seq_lens", torch.int32, layout.B * m), queries_per_seq, window, sinks)
    cache_args = cache._of(layout)
    _check(lib().dense_decode_cache(ctypes.byref(layout), _ptr_here(here, q, "q", dt, nq), cache_args, S_max, ctypes.byref(args),
                                    _ptr_here(here, workspace, "workspace", torch.uint8), workspace.numel(),
                                    _ptr_here(here, out, "out", dt, nq), _stream_ptr(stream)), "dense_decode_cache")
