"""Thin binding of the C-ABI library (`include/eta.h`).

Argument marshalling only: torch tensors provide device memory and the current
CUDA stream; every step of the path runs in the library's kernels.  There is no
CPU fallback: a missing library or a CPU tensor raises.  The library is loaded
with ctypes; the calls of a decode step are marshalled by the compiled module
`_eta_torch` (`csrc/eta_torch.cpp`), because ctypes takes longer over their
arguments than a small step takes on the GPU.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libeta_b200.so")

ETA_FLAG_DENSE = 1
ETA_FLAG_UNGATE_LAST = 2
ETA_FLAG_PACKED_SIGMA = 4
ETA_BUILD_SIGMA_ENVELOPE = 1
ETA_BUILD_PACKED_SIGMA = 2
ETA_DEV_TIMEOUT, ETA_DEV_LEN_CLAMPED, ETA_DEV_EMPTY_ROW = 1, 2, 4
ETA_DEV_BAD_SLOT, ETA_DEV_REFUSED = 8, 16
ETA_TOKENS_INTERLEAVED = 1

EXPORTS = ("eta_workspace_bytes", "eta_build_block_summaries", "eta_append_summary", "eta_build_block_summaries_paged",
           "eta_append_summary_paged", "eta_decode_paged", "eta_stage_query", "eta_predict_threshold",
           "eta_score_dual", "eta_calibration_workspace_bytes", "eta_calibrate_head_const", "eta_decode", "eta_decode_static", "eta_static_scratch_bytes", "eta_decode_kernel_count", "eta_decode_launches", "eta_profile_enable", "eta_profile_read",
           "eta_profile_kernel_name", "eta_set_pdl", "eta_strerror", "eta_last_cuda_error", "eta_plan_pages",
           "eta_append_tokens", "eta_append_tokens_kv4", "eta_kv4_block_bytes", "eta_unpack_kv4",
           "eta_build_block_summaries_kv4", "eta_append_summary_kv4", "eta_decode_kv4", "eta_kv4_workspace_bytes",
           "eta_prefill", "eta_prefill_workspace_bytes", "eta_fork_pages", "eta_fork_summaries", "eta_free_pages", "eta_compact_pages",
           "eta_copy_pages", "eta_pages_workspace_bytes")


class CacheDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32), ("t_cap", ctypes.c_int32),
                ("nb_cap", ctypes.c_int32),
                ("k_stride_b", ctypes.c_int64), ("k_stride_h", ctypes.c_int64), ("k_stride_t", ctypes.c_int64),
                ("v_stride_b", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("v_stride_t", ctypes.c_int64)]


class Params(ctypes.Structure):
    _fields_ = [("z", ctypes.c_float), ("a", ctypes.c_float), ("beta", ctypes.c_float), ("scale", ctypes.c_float),
                ("lwb", ctypes.c_int32), ("rescue_window", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class PageTable(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("table_stride", ctypes.c_int32), ("n_pages", ctypes.c_int32)]


class Kv4Desc(ctypes.Structure):
    _fields_ = [("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_j", ctypes.c_int64),
                ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


class TokensDesc(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int32), ("type", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("q_stride_r", ctypes.c_int64), ("q_stride_h", ctypes.c_int64), ("k_stride_r", ctypes.c_int64),
                ("k_stride_h", ctypes.c_int64), ("v_stride_r", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("eps", ctypes.c_float)]


class PagePool(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("piece_stride", ctypes.c_int64), ("piece_bytes", ctypes.c_int64),
                ("n_pieces", ctypes.c_int32)]


class EtaError(RuntimeError):
    pass


_lib = None
_native = None          # the compiled marshalling module, or what stands for it where it is missing
_STEP_CALLS = ("eta_append_summary", "eta_append_summary_paged", "eta_predict_threshold", "eta_decode", "eta_decode_paged",
               "eta_decode_static", "eta_plan_pages", "eta_append_tokens", "eta_append_tokens_kv4", "eta_unpack_kv4",
               "eta_build_block_summaries_kv4", "eta_append_summary_kv4", "eta_decode_kv4", "eta_prefill", "eta_fork_pages", "eta_fork_summaries", "eta_free_pages",
               "eta_compact_pages", "eta_copy_pages")


class _Missing:
    """Every call through a module that could not be imported raises the reason."""

    def __init__(self, why: Exception):
        self._why = why

    def __getattr__(self, name):
        raise EtaError(f"_eta_torch is missing ({self._why}): build it with `python -m paper_2609_20888_b200.build`") from self._why


def _marshalling():
    try:
        from . import _eta_torch
    except ImportError as e:
        return _Missing(e)
    _eta_torch.set_classes(EtaError, CacheDesc, PageTable, DecodeParams, Params, Kv4Desc)
    return _eta_torch


def load(path: str | None = None) -> ctypes.CDLL:
    """Load the in-tree library; fails loudly when it has not been built.  With a path: another build of the same
    sources (a test variant), loaded beside the product library and not remembered."""
    global _lib, _native
    if _lib is None or path is not None:
        if _native is None:
            _native = _marshalling()           # only the calls of a decode step need it
        lib_path = path or LIB_PATH
        if not os.path.exists(lib_path):
            raise EtaError(f"{lib_path} is missing: build it with `python -m paper_2609_20888_b200.build` "
                           "(there is no fallback path)")
        lib = ctypes.CDLL(lib_path)
        vp, i32p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
        D, P = ctypes.POINTER(CacheDesc), ctypes.POINTER(Params)
        lib.eta_workspace_bytes.argtypes = [D, ctypes.POINTER(ctypes.c_size_t)]
        lib.eta_build_block_summaries.argtypes = [D, vp, i32p, vp, f32p, ctypes.c_uint32, vp]
        lib.eta_append_summary.argtypes = [D, vp, i32p, vp, f32p, ctypes.c_uint32, vp]
        PT = ctypes.POINTER(PageTable)
        lib.eta_build_block_summaries_paged.argtypes = [D, PT, vp, i32p, vp, f32p, ctypes.c_uint32, vp]
        lib.eta_append_summary_paged.argtypes = [D, PT, vp, i32p, vp, f32p, ctypes.c_uint32, vp]
        lib.eta_decode_paged.argtypes = [D, PT, P, vp, vp, vp, i32p, vp, f32p, f32p, f32p, f32p, vp, i32p, vp, vp,
                                         ctypes.c_size_t, vp]
        lib.eta_predict_threshold.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, f32p, f32p, f32p, vp]
        lib.eta_stage_query.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp, vp]
        lib.eta_score_dual.argtypes = [D, P, vp, i32p, vp, f32p, f32p, vp]
        i32 = ctypes.c_int32
        lib.eta_calibration_workspace_bytes.argtypes = [i32, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        lib.eta_calibrate_head_const.argtypes = [i32, i32, i32, i32, i32, vp, vp, f32p, ctypes.c_float, ctypes.c_float,
                                                 i32, ctypes.c_float, ctypes.c_float, f32p, f32p, vp, ctypes.c_size_t, vp]
        lib.eta_decode.argtypes = [D, P, vp, vp, vp, i32p, vp, f32p, f32p, f32p, f32p, vp, i32p, vp, vp,
                                   ctypes.c_size_t, vp]
        lib.eta_plan_pages.argtypes = [i32, i32, i32, i32p, i32p, i32p, i32p, i32p, i32, i32p, i32p, i32p, i32, i32, vp, i32p, i32p,
                                       i32p, vp, vp]
        Q4, TD = ctypes.POINTER(Kv4Desc), ctypes.POINTER(TokensDesc)
        lib.eta_append_tokens.argtypes = [D, TD, vp, vp, vp, f32p, f32p, vp, i32p, vp, i32, vp, vp, vp, vp, vp]
        lib.eta_append_tokens_kv4.argtypes = [D, Q4, TD, vp, vp, vp, f32p, f32p, vp, i32p, vp, i32, vp, vp, vp, vp]
        lib.eta_unpack_kv4.argtypes = [D, Q4, vp, i32, vp, vp, vp]
        lib.eta_build_block_summaries_kv4.argtypes = [D, Q4, PT, vp, i32p, vp, f32p, ctypes.c_uint32, vp]
        lib.eta_append_summary_kv4.argtypes = [D, Q4, PT, vp, i32p, vp, f32p, ctypes.c_uint32, vp]
        lib.eta_decode_kv4.argtypes = [D, Q4, PT, P, vp, vp, i32p, vp, f32p, f32p, f32p, f32p, vp, i32p, vp, vp, ctypes.c_size_t, vp]
        lib.eta_kv4_workspace_bytes.argtypes = [D, ctypes.POINTER(ctypes.c_size_t)]
        lib.eta_kv4_block_bytes.argtypes = [i32, i32]
        lib.eta_kv4_block_bytes.restype = ctypes.c_size_t
        lib.eta_prefill_workspace_bytes.argtypes = [D, ctypes.POINTER(ctypes.c_size_t)]
        lib.eta_prefill.argtypes = [D, PT, P, i32, vp, i32p, i32p, i32p, vp, vp, f32p, f32p, vp, vp, vp, ctypes.c_size_t, vp]
        lib.eta_pages_workspace_bytes.argtypes = [i32, ctypes.POINTER(ctypes.c_size_t)]
        lib.eta_fork_pages.argtypes = [i32, i32, i32, i32p, i32p, i32p, i32p, i32p, i32, i32p, i32p, i32p, i32p, i32p, i32, i32p, i32p, i32p, vp, vp]
        lib.eta_fork_summaries.argtypes = [D, i32p, i32p, vp, f32p, ctypes.c_uint32, vp, vp]
        lib.eta_free_pages.argtypes = [i32, i32, i32, i32p, i32p, i32p, i32p, i32, i32p, i32p, i32p, i32p, i32p, i32, vp, vp, ctypes.c_size_t, vp]
        lib.eta_compact_pages.argtypes = [i32, i32, i32, i32p, i32p, i32p, i32, i32p, i32p, i32p, i32p, i32p, i32p, i32, i32p, i32p, i32p, vp, vp,
                                          ctypes.c_size_t, vp]
        lib.eta_copy_pages.argtypes = [ctypes.POINTER(PagePool), i32, i32, i32p, i32p, i32, i32p, vp, vp]
        lib.eta_decode_static.argtypes = [D, P, vp, vp, vp, i32p, vp, f32p, f32p, f32p, f32p, vp, i32p, vp, vp]
        lib.eta_static_scratch_bytes.restype = ctypes.c_size_t
        lib.eta_decode_kernel_count.restype = ctypes.c_int
        lib.eta_decode_launches.argtypes = [D, P]
        lib.eta_strerror.restype = ctypes.c_char_p
        lib.eta_strerror.argtypes = [ctypes.c_int]
        lib.eta_last_cuda_error.restype = ctypes.c_char_p
        lib.eta_profile_enable.argtypes = [ctypes.c_int]
        lib.eta_set_pdl.argtypes = [ctypes.c_int]
        lib.eta_profile_read.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_int]
        lib.eta_profile_kernel_name.restype = ctypes.c_char_p
        lib.eta_profile_kernel_name.argtypes = [ctypes.c_int]
        for name in EXPORTS:
            if name not in ("eta_strerror", "eta_last_cuda_error", "eta_decode_kernel_count",
                            "eta_profile_kernel_name", "eta_static_scratch_bytes", "eta_kv4_block_bytes"):
                getattr(lib, name).restype = ctypes.c_int
        lib.addresses = {name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _STEP_CALLS}
        if path is not None:
            return lib
        _lib = lib
    return _lib


def _check(rc: int, what: str) -> None:
    if rc != 0:
        lib = load()
        raise EtaError(f"{what}: {lib.eta_strerror(rc).decode()} ({rc}) {lib.eta_last_cuda_error().decode()}")


def _dev(t: torch.Tensor | None, dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise EtaError(f"{name} must be a CUDA tensor (no CPU path exists)")
    if dtype is not None and t.dtype != dtype:
        raise EtaError(f"{name} must be {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


def _dev_musig(t: torch.Tensor):
    """Summary records: fp16 (compact layout) or uint8 (packed layout)."""
    if t is not None and t.dtype not in (torch.float16, torch.uint8):
        raise EtaError(f"musig must be float16 (compact records) or uint8 (packed records), got {t.dtype}")
    return _dev(t, None, "musig")


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


@dataclass
class DecodeParams:
    z: float = 1.0
    a: float = 0.0
    beta: float = 5.0
    scale: float = 0.0
    lwb: int = 0
    rescue_window: int = 128
    flags: int = 0

    def c(self) -> Params:
        return Params(self.z, self.a, self.beta, self.scale, self.lwb, self.rescue_window, self.flags)


def cache_desc(K: torch.Tensor, V: torch.Tensor, n_q_heads: int, block_size: int, nb_cap: int | None = None) -> CacheDesc:
    """Describe a cache K, V of logical shape [batch, n_kv_heads, t_cap, head_dim] (any strides with unit
    stride along head_dim)."""
    B, Hkv, Tcap, d = K.shape
    if K.stride(3) != 1 or V.stride(3) != 1 or V.shape != K.shape:
        raise EtaError("K and V must have the same shape and unit stride along head_dim")
    nb = nb_cap if nb_cap is not None else (Tcap + block_size - 1) // block_size
    return CacheDesc(B, n_q_heads, Hkv, d, block_size, Tcap, nb, K.stride(0), K.stride(1), K.stride(2),
                     V.stride(0), V.stride(1), V.stride(2))


def paged_cache_desc(K_pool: torch.Tensor, V_pool: torch.Tensor, batch: int, n_q_heads: int, t_cap: int,
                     nb_cap: int | None = None) -> CacheDesc:
    """Describe a paged cache: pools of logical shape [n_pages, n_kv_heads, block_size, head_dim] (any strides with
    unit stride along head_dim); the page size is the block size, the stride of the first axis the page stride."""
    n_pages, Hkv, b, d = K_pool.shape
    if K_pool.stride(3) != 1 or V_pool.stride(3) != 1 or V_pool.shape != K_pool.shape:
        raise EtaError("K_pool and V_pool must have the same shape and unit stride along head_dim")
    nb = nb_cap if nb_cap is not None else (t_cap + b - 1) // b
    return CacheDesc(batch, n_q_heads, Hkv, d, b, t_cap, nb, K_pool.stride(0), K_pool.stride(1), K_pool.stride(2),
                     V_pool.stride(0), V_pool.stride(1), V_pool.stride(2))


def page_table(block_table: torch.Tensor, n_pages: int) -> PageTable:
    """block_table: int32 CUDA tensor [batch, table_stride], page of every block of tokens of every sequence."""
    if block_table.dim() != 2 or block_table.stride(1) != 1:
        raise EtaError("block_table must be a 2-D tensor with unit stride along its second axis")
    return PageTable(_dev(block_table, torch.int32, "block_table"), block_table.stride(0), n_pages)


def eta_workspace_bytes(desc: CacheDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(load().eta_workspace_bytes(ctypes.byref(desc), ctypes.byref(n)), "eta_workspace_bytes")
    return n.value


def alloc_summaries(desc: CacheDesc, device, packed: bool = False):
    """musig, mnorm for the compact layout (fp16 [.., 2, d]) or, with `packed`, the packed one (bytes [.., 3 d]: the
    centroid as fp16, then sigma rounded up to e4m3)."""
    if packed:
        musig = torch.zeros((desc.batch, desc.n_kv_heads, desc.nb_cap, 3 * desc.head_dim), dtype=torch.uint8, device=device)
        mnorm = torch.zeros((desc.batch, desc.n_kv_heads, desc.nb_cap), dtype=torch.float32, device=device)
        return musig, mnorm
    musig = torch.zeros((desc.batch, desc.n_kv_heads, desc.nb_cap, 2, desc.head_dim), dtype=torch.float16, device=device)
    mnorm = torch.zeros((desc.batch, desc.n_kv_heads, desc.nb_cap), dtype=torch.float32, device=device)
    return musig, mnorm


def eta_build_block_summaries(desc, K, seq_lens, musig, mnorm, flags: int = 0) -> None:
    _check(load().eta_build_block_summaries(ctypes.byref(desc), _dev(K, torch.bfloat16, "K"),
                                            _dev(seq_lens, torch.int32, "seq_lens"), _dev_musig(musig),
                                            _dev(mnorm, torch.float32, "mnorm"), flags, _stream()),
           "eta_build_block_summaries")


def eta_append_summary(desc, K, seq_lens_after, musig, mnorm, flags: int = 0) -> None:
    lib = _lib or load()
    rc = _native.append(lib.addresses["eta_append_summary"], desc, K, seq_lens_after, musig, mnorm, flags)
    if rc:
        _check(rc, "eta_append_summary")


def eta_build_block_summaries_paged(desc, pages: PageTable, K_pool, seq_lens, musig, mnorm, flags: int = 0) -> None:
    _check(load().eta_build_block_summaries_paged(ctypes.byref(desc), ctypes.byref(pages), _dev(K_pool, torch.bfloat16, "K_pool"),
                                                  _dev(seq_lens, torch.int32, "seq_lens"),
                                                  _dev_musig(musig), _dev(mnorm, torch.float32, "mnorm"),
                                                  flags, _stream()),
           "eta_build_block_summaries_paged")


def eta_append_summary_paged(desc, pages: PageTable, K_pool, seq_lens_after, musig, mnorm, flags: int = 0) -> None:
    lib = _lib or load()
    rc = _native.append_paged(lib.addresses["eta_append_summary_paged"], desc, pages, K_pool, seq_lens_after, musig, mnorm, flags)
    if rc:
        _check(rc, "eta_append_summary_paged")


def eta_stage_query(q_host, q_dev) -> None:
    """Copies a step's queries from a page-locked host tensor into `q_dev` with a kernel on the current stream."""
    if q_host.is_cuda or not q_host.is_pinned():
        raise EtaError("q_host must be a page-locked host tensor")
    if q_host.shape != q_dev.shape or q_host.dtype != torch.bfloat16 or not q_host.is_contiguous() or not q_dev.is_contiguous():
        raise EtaError("q_host and q_dev must be contiguous bf16 tensors of the same shape")
    B, Hq, d = q_host.shape
    _check(load().eta_stage_query(B, Hq, d, ctypes.c_void_p(q_host.data_ptr()), _dev(q_dev, torch.bfloat16, "q_dev"),
                                  _stream()), "eta_stage_query")


def eta_predict_threshold(q, W, bias, tau) -> None:
    lib = _lib or load()
    rc = _native.predict(lib.addresses["eta_predict_threshold"], q, W, bias, tau)
    if rc:
        _check(rc, "eta_predict_threshold")


def eta_score_dual(desc, params: DecodeParams, q, seq_lens, musig, mnorm, bound) -> None:
    p = params.c()
    _check(load().eta_score_dual(ctypes.byref(desc), ctypes.byref(p), _dev(q, torch.bfloat16, "q"),
                                 _dev(seq_lens, torch.int32, "seq_lens"), _dev_musig(musig),
                                 _dev(mnorm, torch.float32, "mnorm"), _dev(bound, torch.float32, "bound"), _stream()),
           "eta_score_dual")


def eta_calibrate_head_const(Q, K, tau, head_const, dbar=None, beta=5.0, scale=0.0, n_bins=2048, s_min=-8.0,
                             s_max=8.0, workspace=None):
    """Q bf16 [n_seq, Hq, T, d], K bf16 [n_seq, Hkv, T, d], tau fp32 [n_seq, Hq, T] -> head_const fp32 [Hq]
    (and dbar fp32 [Hq]).  Allocates the scratch with torch when none is given; returns it for reuse."""
    n_seq, Hq, T, d = Q.shape
    Hkv = K.shape[1]
    need = ctypes.c_size_t(0)
    _check(load().eta_calibration_workspace_bytes(n_seq, T, Hq, n_bins, ctypes.byref(need)),
           "eta_calibration_workspace_bytes")
    if workspace is None:
        workspace = torch.empty(need.value + 256, dtype=torch.uint8, device=Q.device)
        off = (-workspace.data_ptr()) % 256
        workspace = workspace[off:off + need.value]
    _check(load().eta_calibrate_head_const(n_seq, T, Hq, Hkv, d, _dev(Q, torch.bfloat16, "Q"),
                                           _dev(K, torch.bfloat16, "K"), _dev(tau, torch.float32, "tau"), beta, scale,
                                           n_bins, s_min, s_max, _dev(head_const, torch.float32, "head_const"),
                                           _dev(dbar, torch.float32, "dbar"), _dev(workspace, torch.uint8, "workspace"),
                                           workspace.numel(), _stream()),
           "eta_calibrate_head_const")
    return workspace


def eta_decode(desc, params: DecodeParams, q, K, V, seq_lens, musig, mnorm, tau, head_const, out, sel_mask,
               workspace, stats=None, status=None, lib=None) -> None:
    lib = lib or _lib or load()
    rc = _native.decode(lib.addresses["eta_decode"], desc, params, q, K, V, seq_lens, musig, mnorm, tau, head_const, out,
                        sel_mask, stats, status, workspace)
    if rc:
        _check(rc, "eta_decode")


def eta_decode_paged(desc, pages: PageTable, params: DecodeParams, q, K_pool, V_pool, seq_lens, musig, mnorm, tau,
                     head_const, out, sel_mask, workspace, stats=None, status=None) -> None:
    lib = _lib or load()
    rc = _native.decode_paged(lib.addresses["eta_decode_paged"], desc, pages, params, q, K_pool, V_pool, seq_lens, musig, mnorm,
                              tau, head_const, out, sel_mask, stats, status, workspace)
    if rc:
        _check(rc, "eta_decode_paged")


def eta_decode_static(desc, params: DecodeParams, q, K, V, seq_lens, musig, mnorm, tau, head_const, out, sel_mask,
                      stats=None, status=None) -> None:
    """eta_decode without a workspace argument, for callers that have no device memory to give: the scratch is
    an 8 MiB array built into the library (see include/eta.h for its limit and sharing rules)."""
    lib = _lib or load()
    rc = _native.decode_static(lib.addresses["eta_decode_static"], desc, params, q, K, V, seq_lens, musig, mnorm, tau, head_const,
                               out, sel_mask, stats, status)
    if rc:
        _check(rc, "eta_decode_static")


def eta_plan_pages(block_size: int, t_cap: int, new_lens, seq_lens, block_table, free_pages, n_free, slot_map, positions, row_start,
                   granted, seq_lens_out=None, n_free_out=None, release=None, status=None) -> None:
    """Block tables and slot maps from request lengths (see include/eta.h): pages of released sequences go back to the free stack, new
    tokens get pages, `granted`, `row_start`, `slot_map` and `positions` say where they go.  int32 CUDA tensors on the current
    device, slot_map int64; lengths and the free count are updated in place unless outputs are given."""
    lib = _lib or load()
    rc = _native.plan(lib.addresses["eta_plan_pages"], block_size, t_cap, new_lens, release, seq_lens,
                      seq_lens if seq_lens_out is None else seq_lens_out, block_table, free_pages, n_free,
                      n_free if n_free_out is None else n_free_out, slot_map, positions, row_start, granted, status)
    if rc:
        _check(rc, "eta_plan_pages")


def eta_append_tokens(desc: CacheDesc, q, k, v, slot_map, positions, q_out, K, V, inv_freq=None, q_weight=None, k_weight=None,
                      eps: float = 1e-6, interleaved: bool = False, paged: bool = False, status=None) -> None:
    """A step's new tokens (see include/eta.h): q [rows, n_q_heads, head_dim], k and v [rows, n_kv_heads, head_dim] (bf16, fp16 or fp32; parts of one
    projection will do) are normed per head and rotated by their positions; queries go to q_out (bf16), keys and values to the
    places of K and V that slot_map (int64 [rows]) names.  inv_freq: float64 [rotary_dim / 2]."""
    lib = _lib or load()
    rc = _native.tokens(lib.addresses["eta_append_tokens"], desc, None, q, k, v, q_weight, k_weight, inv_freq, positions, slot_map, paged,
                        q_out, K, V, status, eps, ETA_TOKENS_INTERLEAVED if interleaved else 0)
    if rc:
        _check(rc, "eta_append_tokens")


def kv4_block_bytes(block_size: int, head_dim: int) -> int:
    """Bytes of a block of one KV head of a 4-bit cache, K and V together."""
    return load().eta_kv4_block_bytes(block_size, head_dim)


def kv4_cache_desc(pool: torch.Tensor, n_q_heads: int, head_dim: int, block_size: int, batch: int | None = None, t_cap: int | None = None,
                   nb_cap: int | None = None, k_scale: float = 1.0, v_scale: float = 1.0) -> tuple[CacheDesc, Kv4Desc]:
    """Describe a 4-bit cache: pool uint8 [batch, n_kv_heads, blocks, block bytes], or paged [n_pages, n_kv_heads, block bytes] with the batch
    and the capacity of a sequence (any strides of multiples of 16 bytes, unit stride along the bytes)."""
    if pool.dim() not in (3, 4) or pool.stride(-1) != 1 or pool.dtype != torch.uint8 or pool.shape[-1] != kv4_block_bytes(block_size, head_dim):
        raise EtaError("pool must be uint8 [batch, n_kv_heads, blocks, block bytes] or [n_pages, n_kv_heads, block bytes]")
    paged = pool.dim() == 3
    if paged and (batch is None or t_cap is None):
        raise EtaError("a paged cache needs the batch and t_cap")
    if not paged and batch not in (None, pool.shape[0]):
        raise EtaError("batch and pool do not agree")
    batch = pool.shape[0] if batch is None else batch
    t_cap = pool.shape[2] * block_size if t_cap is None else t_cap
    if not paged and pool.shape[2] * block_size < t_cap:
        raise EtaError("pool has too few blocks for t_cap tokens")
    nb = nb_cap if nb_cap is not None else (t_cap + block_size - 1) // block_size
    Hkv, tokens = pool.shape[1], block_size if paged else t_cap
    bf16 = (Hkv * tokens * head_dim, tokens * head_dim, head_dim)          # of the bf16 cache it stands for
    least = pool.shape[-1]                                                 # where an axis has one element its stride says nothing
    strides = [pool.stride(k) if pool.shape[k] > 1 else least for k in range(pool.dim() - 1)]
    return (CacheDesc(batch, n_q_heads, Hkv, head_dim, block_size, t_cap, nb, *bf16, *bf16),
            Kv4Desc(strides[0], strides[1], 0 if paged else strides[2], k_scale, v_scale))


def eta_append_tokens_kv4(desc: CacheDesc, kv4: Kv4Desc, q, k, v, slot_map, positions, q_out, pool, inv_freq=None, q_weight=None,
                          k_weight=None, eps: float = 1e-6, interleaved: bool = False, status=None) -> None:
    """eta_append_tokens into a 4-bit cache."""
    lib = _lib or load()
    if kv4 is None:
        raise EtaError("kv4 must be a Kv4Desc")
    rc = _native.tokens(lib.addresses["eta_append_tokens_kv4"], desc, kv4, q, k, v, q_weight, k_weight, inv_freq, positions, slot_map, None,
                        q_out, pool, None, status, eps, ETA_TOKENS_INTERLEAVED if interleaved else 0)
    if rc:
        _check(rc, "eta_append_tokens_kv4")


def eta_unpack_kv4(desc: CacheDesc, kv4: Kv4Desc, pool, K, V) -> None:
    """What a 4-bit cache stands for, as a bf16 cache K, V [batch, n_kv_heads, t_cap, head_dim] (paged: [n_pages, n_kv_heads, block_size,
    head_dim]), any strides."""
    lib = _lib or load()
    rc = _native.unpack(lib.addresses["eta_unpack_kv4"], desc, kv4, pool, K, V)
    if rc:
        _check(rc, "eta_unpack_kv4")


def eta_build_block_summaries_kv4(desc: CacheDesc, kv4: Kv4Desc, pool, seq_lens, musig, mnorm, flags: int = 0,
                                  pages: PageTable | None = None) -> None:
    """The block index of a 4-bit cache, of all full blocks; paged with a page table."""
    lib = _lib or load()
    rc = _native.index_kv4(lib.addresses["eta_build_block_summaries_kv4"], desc, kv4, pages, pool, seq_lens, musig, mnorm, flags)
    if rc:
        _check(rc, "eta_build_block_summaries_kv4")


def eta_append_summary_kv4(desc: CacheDesc, kv4: Kv4Desc, pool, seq_lens_after, musig, mnorm, flags: int = 0,
                           pages: PageTable | None = None) -> None:
    """The same, of the blocks that the newest tokens completed."""
    lib = _lib or load()
    rc = _native.index_kv4(lib.addresses["eta_append_summary_kv4"], desc, kv4, pages, pool, seq_lens_after, musig, mnorm, flags)
    if rc:
        _check(rc, "eta_append_summary_kv4")


def eta_kv4_workspace_bytes(desc: CacheDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(load().eta_kv4_workspace_bytes(ctypes.byref(desc), ctypes.byref(n)), "eta_kv4_workspace_bytes")
    return n.value


def eta_decode_kv4(desc: CacheDesc, kv4: Kv4Desc, params: DecodeParams, q, pool, seq_lens, musig, mnorm, tau, head_const, out, sel_mask,
                   workspace, stats=None, status=None, pages: PageTable | None = None) -> None:
    """eta_decode over a 4-bit cache; paged with a page table.  musig and mnorm may be None with ETA_FLAG_DENSE."""
    lib = _lib or load()
    rc = _native.decode_kv4(lib.addresses["eta_decode_kv4"], desc, kv4, pages, params, q, pool, seq_lens, musig, mnorm, tau, head_const, out,
                            sel_mask, stats, status, workspace)
    if rc:
        _check(rc, "eta_decode_kv4")


def eta_prefill_workspace_bytes(desc: CacheDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(load().eta_prefill_workspace_bytes(ctypes.byref(desc), ctypes.byref(n)), "eta_prefill_workspace_bytes")
    return n.value


def eta_prefill(desc: CacheDesc, params: DecodeParams, q, K, V, row_start, seq_lens, out, workspace, tau=None, head_const=None,
                granted=None, status=None, pages: PageTable | None = None) -> None:
    """Attention of a step's new tokens over the cache that holds them (see include/eta.h): q and out bf16 [rows, n_q_heads, head_dim],
    packed by row_start (int32 [batch + 1]); tau fp32 [rows, n_q_heads] or head_const fp32 [n_q_heads], neither with ETA_FLAG_DENSE;
    paged with a page table."""
    lib = _lib or load()
    rc = _native.prefill(lib.addresses["eta_prefill"], desc, pages, params, q, row_start, seq_lens, granted, K, V, tau, head_const, out,
                         status, workspace)
    if rc:
        _check(rc, "eta_prefill")


def eta_pages_workspace_bytes(n_pages: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().eta_pages_workspace_bytes(n_pages, ctypes.byref(n)), "eta_pages_workspace_bytes")
    return n.value


def eta_fork_pages(block_size: int, t_cap: int, parent, seq_lens, block_table, shared, free_pages, n_free, copy_src, copy_dst, granted, take=None,
                   seq_lens_out=None, shared_out=None, n_free_out=None, status=None) -> None:
    """Sequences that begin as copies of others (see include/eta.h): full pages are shared, copy_src and copy_dst name the last, partly
    filled ones for eta_copy_pages.  int32 CUDA tensors on the current device; lengths, counts and the free count are updated in place unless
    outputs are given."""
    lib = _lib or load()
    rc = _native.fork_pages(lib.addresses["eta_fork_pages"], block_size, t_cap, parent, take, seq_lens,
                            seq_lens if seq_lens_out is None else seq_lens_out, block_table, shared, shared if shared_out is None else shared_out,
                            free_pages, n_free, n_free if n_free_out is None else n_free_out, copy_src, copy_dst, granted, status)
    if rc:
        _check(rc, "eta_fork_pages")


def eta_fork_summaries(desc: CacheDesc, parent, granted, musig, mnorm, status=None) -> None:
    """The forks' block summaries, from their parents' rows to theirs; the layout of the records goes by musig's type."""
    lib = _lib or load()
    rc = _native.fork_summaries(lib.addresses["eta_fork_summaries"], desc, parent, granted, musig, mnorm, status)
    if rc:
        _check(rc, "eta_fork_summaries")


def eta_free_pages(block_size: int, t_cap: int, release, seq_lens, block_table, shared, free_pages, n_free, workspace, seq_lens_out=None,
                   shared_out=None, n_free_out=None, status=None) -> None:
    """Finished sequences let go of their pages; those that nobody else holds go back to the free stack."""
    lib = _lib or load()
    rc = _native.free_pages(lib.addresses["eta_free_pages"], block_size, t_cap, release, seq_lens, seq_lens if seq_lens_out is None else seq_lens_out,
                            block_table, shared, shared if shared_out is None else shared_out, free_pages, n_free,
                            n_free if n_free_out is None else n_free_out, status, workspace)
    if rc:
        _check(rc, "eta_free_pages")


def eta_compact_pages(block_size: int, t_cap: int, seq_lens, block_table, shared, free_pages, n_free, move_src, move_dst, n_moves, workspace,
                      block_table_out=None, shared_out=None, free_pages_out=None, n_free_out=None, status=None) -> None:
    """Pages in use move to the low end of the pool: tables, counts and stack after the move, and the list of copies for eta_copy_pages."""
    lib = _lib or load()
    rc = _native.compact_pages(lib.addresses["eta_compact_pages"], block_size, t_cap, seq_lens, block_table,
                               block_table if block_table_out is None else block_table_out, shared, shared if shared_out is None else shared_out,
                               free_pages, free_pages if free_pages_out is None else free_pages_out, n_free,
                               n_free if n_free_out is None else n_free_out, move_src, move_dst, n_moves, status, workspace)
    if rc:
        _check(rc, "eta_compact_pages")


def eta_copy_pages(pools, src, dst, n_moves=None, status=None) -> None:
    """Page src[k] of every pool (a tensor [pages, ...] of any type whose pages are contiguous but for one axis) to page dst[k]; n_moves: an int32 CUDA
    tensor that says how many pairs count (None: all).  Negative numbers are skipped."""
    lib = _lib or load()
    rc = _native.copy_pages(lib.addresses["eta_copy_pages"], pools, src, dst, n_moves, status)
    if rc:
        _check(rc, "eta_copy_pages")


def eta_static_scratch_bytes() -> int:
    return int(load().eta_static_scratch_bytes())


def eta_decode_kernel_count() -> int:
    return load().eta_decode_kernel_count()


def eta_decode_launches(desc: CacheDesc, params: DecodeParams) -> int:
    """Kernels that eta_decode launches for this cache and these parameters on the current device."""
    n = load().eta_decode_launches(ctypes.byref(desc), ctypes.byref(params.c()))
    if n < 0:
        _check(n, "eta_decode_launches")
    return n


def eta_set_pdl(on: bool) -> None:
    _check(load().eta_set_pdl(1 if on else 0), "eta_set_pdl")


def eta_profile_enable(on: bool) -> None:
    _check(load().eta_profile_enable(1 if on else 0), "eta_profile_enable")


def eta_profile_read() -> dict:
    """Device time (ms) of each kernel of the most recent profiled eta_decode call, by kernel name."""
    lib = load()
    ms = (ctypes.c_float * 8)()
    n = lib.eta_profile_read(ms, 8)
    if n < 0:
        _check(n, "eta_profile_read")
    return {lib.eta_profile_kernel_name(k).decode(): float(ms[k]) for k in range(n)}


class DecodeState:
    """Device buffers one decode loop needs (allocated once with torch; the library allocates nothing)."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor, n_q_heads: int, block_size: int):
        dev = K.device
        self.desc = cache_desc(K, V, n_q_heads, block_size)
        self.K, self.V = K, V
        self.musig, self.mnorm = alloc_summaries(self.desc, dev)
        self.workspace = torch.zeros(eta_workspace_bytes(self.desc) + 256, dtype=torch.uint8, device=dev)
        off = (-self.workspace.data_ptr()) % 256
        self.workspace = self.workspace[off:off + eta_workspace_bytes(self.desc)]
        B, Hkv, d = self.desc.batch, self.desc.n_kv_heads, self.desc.head_dim
        self.out = torch.empty((B, n_q_heads, d), dtype=torch.float32, device=dev)
        self.sel_mask = torch.zeros((B, Hkv, self.desc.nb_cap), dtype=torch.uint8, device=dev)
        self.tau = torch.empty((B, n_q_heads), dtype=torch.float32, device=dev)
        self.stats = torch.zeros((B, Hkv), dtype=torch.int32, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
