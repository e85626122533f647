"""Thin ctypes binding of libzc's C ABI.

Argument marshalling only: every step of the codec runs in the library's CUDA kernels (or, for
the codebook and the statistics, in its host code).  The functions have the names of the C entry
points without the ``zc_`` prefix.  PyTorch supplies device memory and streams.

The library must be present (``paper_2508_19263_b200/libzc.so``, built by ``build.build_library``);
importing this module fails loudly when it is not — there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from typing import Optional

import numpy as np
import torch

from . import build as _build

FMT_BF16, FMT_FP8_E4M3, FMT_FP4_E2M1, FMT_SCALE_U8, FMT_FP8_E5M2 = 1, 2, 3, 4, 5
POLICY_AUTO, POLICY_HUFF_ALL, POLICY_RAW_ALL, POLICY_STATIC = 0, 1, 2, 3
MODE_RAW, MODE_HUFF = 0, 1
(OK, E_INVALID_ARG, E_UNSUPPORTED, E_BUFFER_TOO_SMALL, E_CORRUPT, E_CUDA, E_NOMEM, E_DEVICE_TIMEOUT, E_NO_CODE,
 E_TOO_LARGE) = range(10)
NOALLOC_MAX_CHUNKS = 65536
REAL_F32, REAL_BF16, REAL_F16 = 0, 1, 2
_REAL = {torch.float32: REAL_F32, torch.bfloat16: REAL_BF16, torch.float16: REAL_F16}


class ZcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_lib.zc_strerror(status).decode()} (status {status})")


class PlanInfo(C.Structure):
    _fields_ = [("format", C.c_uint32), ("group", C.c_uint32), ("chunk_bytes", C.c_uint32), ("n_chunks", C.c_uint32),
                ("n_elems", C.c_uint64), ("n_syms", C.c_uint64), ("input_bytes", C.c_uint64),
                ("syms_per_chunk", C.c_uint32), ("syms_per_subchunk", C.c_uint32)]


class StreamStats(C.Structure):
    _fields_ = [("n_syms", C.c_uint64), ("raw_bits", C.c_uint64), ("payload_bits", C.c_uint64),
                ("container_bytes", C.c_uint64), ("mode", C.c_uint32), ("n_active_symbols", C.c_uint32),
                ("max_len", C.c_uint32), ("reserved", C.c_uint32), ("avg_len", C.c_double),
                ("entropy_bits", C.c_double)]


class Stats(C.Structure):
    _fields_ = [("stream", StreamStats * 2), ("in_bytes", C.c_uint64), ("out_bytes", C.c_uint64),
                ("ratio_payload", C.c_double), ("ratio_container", C.c_double)]


class DictInfo(C.Structure):
    _fields_ = [("tolerance", C.c_double), ("baseline_ratio", C.c_double), ("last_ratio", C.c_double),
                ("n_observed", C.c_uint64), ("n_rebuilds", C.c_uint64), ("has_baseline", C.c_uint32), ("reserved", C.c_uint32)]


class Fp8MatrixDesc(C.Structure):
    _fields_ = [("d_elems", C.c_void_p), ("d_scales", C.c_void_p), ("rows", C.c_uint64), ("cols", C.c_uint64),
                ("ld_elems", C.c_uint64), ("ld_scales", C.c_uint64), ("format", C.c_uint32), ("block_rows", C.c_uint32)]


class Fp8MoeLayerDesc(C.Structure):
    _fields_ = [("d_router", C.c_void_p), ("d_gate_up", C.c_void_p), ("d_gate_up_scales", C.c_void_p), ("d_down", C.c_void_p),
                ("d_down_scales", C.c_void_p), ("ld_router", C.c_uint64), ("ld_gate_up", C.c_uint64), ("ld_down", C.c_uint64),
                ("n_experts", C.c_uint32), ("top_k", C.c_uint32), ("hidden", C.c_uint32), ("inter", C.c_uint32),
                ("format", C.c_uint32), ("real_type", C.c_uint32)]


class KvCacheDesc(C.Structure):
    _fields_ = [("d_k_elems", C.c_void_p), ("d_k_scales", C.c_void_p), ("d_v_elems", C.c_void_p), ("d_v_scales", C.c_void_p),
                ("n_pages", C.c_uint64), ("page_tokens", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("format", C.c_uint32)]


class KvBatchDesc(C.Structure):
    _fields_ = [("d_page_table", C.c_void_p), ("d_lens", C.c_void_p), ("d_first", C.c_void_p), ("ld_page_table", C.c_uint64),
                ("n_rows", C.c_uint64), ("max_pages", C.c_uint32), ("n_seqs", C.c_uint32), ("max_new", C.c_uint32)]


class KvTensorDesc(C.Structure):
    _fields_ = [("d", C.c_void_p), ("ld_row", C.c_uint64), ("ld_head", C.c_uint64)]


class KvAttentionArgs(C.Structure):
    _fields_ = [("q", KvTensorDesc), ("out", KvTensorDesc), ("d_lse", C.c_void_p), ("type", C.c_uint32), ("q_heads", C.c_uint32),
                ("scale", C.c_float), ("causal", C.c_uint32), ("window", C.c_uint32)]


def _load():
    # ZC_LIBRARY: another build of the same library (the development build with in-kernel checks), for tests
    path = os.environ.get("ZC_LIBRARY") or _build.LIB
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: run paper_2508_19263_b200.build.build_library() "
                          "(or __graft_entry__.build()) first; there is no fallback implementation")
    L = C.CDLL(path)
    vp, u64p = C.c_void_p, C.POINTER(C.c_uint64)
    L.zc_plan.restype = C.c_int
    L.zc_plan.argtypes = [C.c_int, C.c_uint64, C.c_uint32, C.POINTER(vp)]
    L.zc_plan_destroy.restype = None
    L.zc_plan_destroy.argtypes = [vp]
    L.zc_plan_get_info.restype = C.c_int
    L.zc_plan_get_info.argtypes = [vp, C.POINTER(PlanInfo)]
    L.zc_max_compressed_bytes.restype = C.c_size_t
    L.zc_max_compressed_bytes.argtypes = [vp]
    L.zc_workspace_bytes.restype = C.c_size_t
    L.zc_workspace_bytes.argtypes = [vp]
    L.zc_histogram.restype = C.c_int
    L.zc_histogram.argtypes = [vp, vp, vp, vp]
    L.zc_histogram_batch.restype = C.c_int
    L.zc_histogram_batch.argtypes = [C.c_uint32, C.POINTER(vp), C.POINTER(vp), vp, vp]
    L.zc_build_codebook.restype = C.c_int
    L.zc_build_codebook.argtypes = [vp, u64p, C.c_int, C.POINTER(vp)]
    L.zc_build_codebooks.restype = C.c_int
    L.zc_build_codebooks.argtypes = [C.c_uint32, C.POINTER(vp), u64p, C.c_int, C.c_uint32, C.POINTER(vp)]
    L.zc_codebook_destroy.restype = None
    L.zc_codebook_destroy.argtypes = [vp]
    L.zc_codebook_get.restype = C.c_int
    L.zc_codebook_get.argtypes = [vp, C.c_uint32, C.POINTER(C.c_uint32), C.POINTER(C.c_uint8), C.POINTER(C.c_uint32)]
    L.zc_compress.restype = C.c_int
    L.zc_compress.argtypes = [vp, vp, vp, vp, C.c_size_t, vp, u64p, vp]
    L.zc_compress_noalloc.restype = C.c_int
    L.zc_compress_noalloc.argtypes = [vp, vp, vp, vp, C.c_size_t, u64p, vp]
    L.zc_decompress.restype = C.c_int
    L.zc_decompress.argtypes = [vp, vp, C.c_size_t, vp, vp, vp]
    L.zc_compress_batch_workspace_bytes.restype = C.c_size_t
    L.zc_compress_batch_workspace_bytes.argtypes = [C.c_uint32, C.POINTER(vp)]
    L.zc_compress_batch.restype = C.c_int
    L.zc_compress_batch.argtypes = [C.c_uint32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(C.c_size_t),
                                    vp, C.c_size_t, u64p, vp]
    L.zc_decompress_batch.restype = C.c_int
    L.zc_decompress_batch.argtypes = [C.c_uint32, C.POINTER(vp), C.POINTER(vp), C.POINTER(C.c_size_t), C.POINTER(vp), vp, vp]
    L.zc_batch_status.restype = C.c_int
    L.zc_batch_status.argtypes = [vp, C.POINTER(C.c_uint32), vp]
    L.zc_histogram_xor.restype = C.c_int
    L.zc_histogram_xor.argtypes = [vp, vp, vp, vp, vp]
    L.zc_histogram_batch_xor.restype = C.c_int
    L.zc_histogram_batch_xor.argtypes = [C.c_uint32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), vp, vp]
    L.zc_compress_xor.restype = C.c_int
    L.zc_compress_xor.argtypes = [vp, vp, vp, vp, vp, C.c_size_t, vp, u64p, vp]
    L.zc_compress_batch_xor.restype = C.c_int
    L.zc_compress_batch_xor.argtypes = [C.c_uint32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                        C.POINTER(C.c_size_t), vp, C.c_size_t, u64p, vp]
    L.zc_decompress_xor.restype = C.c_int
    L.zc_decompress_xor.argtypes = [vp, vp, C.c_size_t, vp, vp, vp, vp]
    L.zc_decompress_batch_xor.restype = C.c_int
    L.zc_decompress_batch_xor.argtypes = [C.c_uint32, C.POINTER(vp), C.POINTER(vp), C.POINTER(C.c_size_t), C.POINTER(vp), C.POINTER(vp),
                                          vp, vp]
    L.zc_decompress_chunks.restype = C.c_int
    L.zc_decompress_chunks.argtypes = [vp, vp, C.c_size_t, C.c_uint32, C.c_uint32, vp, vp, vp]
    L.zc_device_status.restype = C.c_int
    L.zc_device_status.argtypes = [vp, vp, vp]
    L.zc_validate_container.restype = C.c_int
    L.zc_validate_container.argtypes = [vp, vp, C.c_size_t]
    L.zc_stats.restype = C.c_int
    L.zc_stats.argtypes = [vp, vp, u64p, vp, C.POINTER(Stats)]
    L.zc_dict_create.restype = C.c_int
    L.zc_dict_create.argtypes = [vp, u64p, C.c_double, C.POINTER(vp)]
    L.zc_dict_destroy.restype = None
    L.zc_dict_destroy.argtypes = [vp]
    L.zc_dict_codebook.restype = vp
    L.zc_dict_codebook.argtypes = [vp]
    L.zc_dict_observe.restype = C.c_int
    L.zc_dict_observe.argtypes = [vp, C.c_uint64, C.c_uint64, C.POINTER(C.c_int)]
    L.zc_dict_rebuild.restype = C.c_int
    L.zc_dict_rebuild.argtypes = [vp, vp, u64p]
    L.zc_dict_get_info.restype = C.c_int
    L.zc_dict_get_info.argtypes = [vp, C.POINTER(DictInfo)]
    L.zc_strerror.restype = C.c_char_p
    L.zc_strerror.argtypes = [C.c_int]
    L.zc_test_split16.restype = C.c_int
    L.zc_test_split16.argtypes = [C.c_int, vp, vp, vp]
    L.zc_test_merge16.restype = C.c_int
    L.zc_test_merge16.argtypes = [C.c_int, vp, vp, vp]
    L.zc_noalloc_status.restype = C.c_int
    L.zc_noalloc_status.argtypes = [vp]
    L.zc_test_encoder_workers.restype = C.c_uint32
    L.zc_test_encoder_workers.argtypes = [vp, C.c_uint32, C.c_uint32, C.c_uint64]
    L.zc_test_decoder_warps.restype = C.c_uint32
    L.zc_test_decoder_warps.argtypes = [vp, C.c_uint32]
    L.zc_test_decoder_pieces.restype = C.c_uint32
    L.zc_test_decoder_pieces.argtypes = [vp, C.c_uint32, C.c_uint64, C.POINTER(C.c_uint32)]
    L.zc_test_debug_counts.restype = C.c_int
    L.zc_test_debug_counts.argtypes = [C.POINTER(C.c_uint32)]
    L.zc_test_fp8_marks.restype = C.c_uint32
    L.zc_test_fp8_marks.argtypes = []
    L.zc_fp8_quantize.restype = C.c_int
    L.zc_fp8_quantize.argtypes = [C.c_int, vp, C.c_uint64, vp, vp, vp]
    L.zc_fp8_matmul.restype = C.c_int
    L.zc_fp8_matmul.argtypes = [vp, vp, C.c_int, vp, C.c_uint64, C.c_uint32, vp]
    L.zc_fp8_moe_workspace_bytes.restype = C.c_size_t
    L.zc_fp8_moe_workspace_bytes.argtypes = [vp, C.c_uint32]
    L.zc_fp8_moe.restype = C.c_int
    L.zc_fp8_moe.argtypes = [vp, C.c_uint32, vp, C.c_uint64, vp, C.c_uint64, vp, vp, vp, C.c_size_t, vp]
    for name in ("zc_kv_append", "zc_kv_read"):
        getattr(L, name).restype = C.c_int
        getattr(L, name).argtypes = [vp, vp, C.c_int, vp, vp, vp]
    L.zc_kv_attention_workspace_bytes.restype = C.c_size_t
    L.zc_kv_attention_workspace_bytes.argtypes = [vp, vp, C.c_uint32]
    L.zc_kv_attention.restype = C.c_int
    L.zc_kv_attention.argtypes = [vp, vp, vp, vp, C.c_size_t, vp]
    L.zc_kv_status.restype = C.c_int
    L.zc_kv_status.argtypes = [vp]
    L.zc_fp8_status.restype = C.c_int
    L.zc_fp8_status.argtypes = [vp]
    for name in ("zc_test_set_wait_limit", "zc_test_stall_encoder", "zc_test_stall_decoder", "zc_test_stall_math"):
        getattr(L, name).restype = None
        getattr(L, name).argtypes = [C.c_uint32]
    return L


_lib = _load()


def _check(status: int, where: str):
    if status != OK:
        raise ZcError(status, where)


def _stream_ptr(stream, _raw=getattr(torch._C, "_cuda_getCurrentRawStream", None)) -> int:
    if stream is None:
        # the handle alone: torch.cuda.current_stream() builds a stream object for it, 3 us of every call
        return _raw(torch.cuda.current_device()) if _raw is not None else torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def strerror(status: int) -> str:
    return _lib.zc_strerror(status).decode()


class Plan:
    """zc_plan: the problem statement of one tensor (format, element count, chunk size)."""

    def __init__(self, fmt: int, n_elems: int, chunk_bytes: int):
        h = C.c_void_p()
        _check(_lib.zc_plan(fmt, n_elems, chunk_bytes, C.byref(h)), "zc_plan")
        self._h = h
        info = PlanInfo()
        _check(_lib.zc_plan_get_info(h, C.byref(info)), "zc_plan_get_info")
        self.info = info
        self.format, self.n_elems, self.chunk_bytes = fmt, n_elems, chunk_bytes
        self.n_syms, self.n_chunks, self.input_bytes = info.n_syms, info.n_chunks, info.input_bytes
        self.max_compressed_bytes = _lib.zc_max_compressed_bytes(h)
        self.workspace_bytes = _lib.zc_workspace_bytes(h)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h and _lib is not None:
            _lib.zc_plan_destroy(h)
            self._h = None


def plan(fmt: int, n_elems: int, chunk_bytes: int) -> Plan:
    return Plan(fmt, n_elems, chunk_bytes)


def _quick_function(name, restype, argtypes=None):
    """A function of the library that takes nanoseconds, called without letting go of the GIL; without argtypes the arguments
    have to be ctypes objects already."""
    f = getattr(C.PyDLL(_lib._name, handle=_lib._handle), name)
    f.restype, f.argtypes = restype, argtypes
    return f


class Codebook:
    """zc_build_codebook result: per stream a mode, 256 code lengths and 256 canonical code values."""

    def __init__(self, handle: int, owned: bool = True):
        self._h = handle
        self._owned = owned                      # a dictionary's codebook belongs to the dictionary

    def __reduce_ex__(self, protocol):
        # the handle is an address in this process with one owner: a copy would destroy it a second time
        raise ValueError("a codebook cannot be copied or pickled")

    def get(self, stream_idx: int):
        mode = C.c_uint32()
        lens = np.zeros(256, np.uint8)
        codes = np.zeros(256, np.uint32)
        _check(_lib.zc_codebook_get(self._h, stream_idx, C.byref(mode), lens.ctypes.data_as(C.POINTER(C.c_uint8)),
                                    codes.ctypes.data_as(C.POINTER(C.c_uint32))), "zc_codebook_get")
        return mode.value, lens, codes

    @property
    def modes(self):
        return [self.get(0)[0], self.get(1)[0]]

    # Codebooks come and go by the tensor: the handle is a plain number and destroying one keeps the GIL (FP4 scales of 36
    # tensors, encoded and decoded: 356 us with an object around every handle, 348 us so).
    def __del__(self, _destroy=_quick_function("zc_codebook_destroy", None, [C.c_void_p])):
        if self._owned and self._h:
            _destroy(self._h)
            self._h = None


def histogram(p: Plan, d_in: torch.Tensor, d_hist: Optional[torch.Tensor] = None, stream=None,
              d_base: Optional[torch.Tensor] = None) -> torch.Tensor:
    """zc_histogram (zc_histogram_xor when d_base is given): returns a device tensor uint64-as-int64 [2, 256]."""
    assert d_in.is_cuda and d_in.is_contiguous()
    if d_hist is None:
        d_hist = torch.empty((2, 256), dtype=torch.int64, device=d_in.device)
    if d_base is None:
        _check(_lib.zc_histogram(p._h, d_in.data_ptr(), d_hist.data_ptr(), _stream_ptr(stream)), "zc_histogram")
    else:
        _check(_lib.zc_histogram_xor(p._h, d_in.data_ptr(), d_base.data_ptr(), d_hist.data_ptr(), _stream_ptr(stream)),
               "zc_histogram_xor")
    return d_hist


def _base_array(d_bases, n):
    """Host array of base-tensor pointers for the XOR-delta forms (None: no base at all, a None entry: none for that tensor)."""
    if d_bases is None:
        return None
    return (C.c_void_p * max(n, 1))(*[(t.data_ptr() if t is not None else None) for t in d_bases])


class HistogramBatch:
    """Argument arrays of zc_histogram_batch, marshalled once."""

    def __init__(self, plans, d_ins, d_bases=None):
        n = len(plans)
        assert len(d_ins) == n and (d_bases is None or len(d_bases) == n)
        self.n = n
        self._keep = (list(plans), list(d_ins), list(d_bases) if d_bases is not None else None)
        self.plans = (C.c_void_p * max(n, 1))(*[p._h.value for p in plans])
        self.ins = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in d_ins])
        self.bases = _base_array(d_bases, n)     # XOR-delta form when given


def histogram_batch(batch: HistogramBatch, d_hists: torch.Tensor, stream=None) -> torch.Tensor:
    """zc_histogram_batch: d_hists is a device tensor int64 [n, 2, 256] (uint64 counts)."""
    assert d_hists.is_cuda and d_hists.is_contiguous() and d_hists.numel() == 512 * batch.n and d_hists.element_size() == 8
    _check(_lib.zc_histogram_batch_xor(batch.n, batch.plans, batch.ins, batch.bases, d_hists.data_ptr(), _stream_ptr(stream)),
           "zc_histogram_batch")
    return d_hists


def build_codebook(p: Plan, h_hist, policy: int = POLICY_AUTO) -> Codebook:
    """zc_build_codebook: host only.  h_hist: array-like [2, 256] of counts."""
    h = np.asarray(h_hist)
    if h.dtype == np.int64 and h.flags.c_contiguous:
        h = h.view(np.uint64)                    # counts as produced by histogram(): no copy
    elif h.dtype != np.uint64 or not h.flags.c_contiguous:
        h = np.ascontiguousarray(h.astype(np.uint64))
    assert h.size == 512
    out = C.c_void_p()
    _check(_lib.zc_build_codebook(p._h, C.cast(h.ctypes.data, C.POINTER(C.c_uint64)), policy, C.byref(out)),
           "zc_build_codebook")
    return Codebook(out.value)


def _hist_ptr(h_hist):
    h = np.asarray(h_hist)
    if h.dtype == np.int64 and h.flags.c_contiguous:
        h = h.view(np.uint64)
    elif h.dtype != np.uint64 or not h.flags.c_contiguous:
        h = np.ascontiguousarray(h.astype(np.uint64))
    assert h.size == 512
    return h, C.cast(h.ctypes.data, C.POINTER(C.c_uint64))


class Dictionary:
    """zc_dict_*: a static codebook for K/V cache tensors plus the rule that says when to replace it."""

    def __init__(self, p: Plan, h_hist, tolerance: float):
        _keep, ptr = _hist_ptr(h_hist)
        self._h = C.c_void_p()
        _check(_lib.zc_dict_create(p._h, ptr, tolerance, C.byref(self._h)), "zc_dict_create")
        # a dictionary is used from one thread at a time
        self._in, self._out, self._flag = C.c_uint64(0), C.c_uint64(0), C.c_int(0)
        self._flag_ref = C.byref(self._flag)

    @property
    def codebook(self) -> Codebook:
        """The current codebook (not owned: valid until rebuild())."""
        return Codebook(_lib.zc_dict_codebook(self._h), owned=False)

    # made for every page of a step: checking and converting the arguments and letting go of the GIL took 0.9 us, this 0.5 us
    def observe(self, input_bytes: int, container_bytes: int, _observe=_quick_function("zc_dict_observe", C.c_int)) -> bool:
        try:
            self._in.value = input_bytes
            self._out.value = container_bytes
        except TypeError:                        # not a plain number: converted, or refused, argument by argument
            status = _lib.zc_dict_observe(self._h, input_bytes, container_bytes, self._flag_ref)
        else:
            status = _observe(self._h, self._in, self._out, self._flag_ref)
        if status != OK:
            raise ZcError(status, "zc_dict_observe")
        return self._flag.value != 0

    def rebuild(self, p: Plan, h_hist) -> None:
        _keep, ptr = _hist_ptr(h_hist)
        _check(_lib.zc_dict_rebuild(self._h, p._h, ptr), "zc_dict_rebuild")

    @property
    def info(self) -> DictInfo:
        out = DictInfo()
        _check(_lib.zc_dict_get_info(self._h, C.byref(out)), "zc_dict_get_info")
        return out

    def __del__(self):
        h = getattr(self, "_h", None)
        if h and _lib is not None:
            _lib.zc_dict_destroy(h)
            self._h = None


def build_codebooks(plans, h_hists, policy: int = POLICY_AUTO, n_threads: int = 0):
    """zc_build_codebooks: the codebooks of many tensors, built on several host threads.
    h_hists: array-like [n, 2, 256] of counts."""
    n = len(plans)
    h = np.asarray(h_hists)
    if h.dtype == np.int64 and h.flags.c_contiguous:
        h = h.view(np.uint64)
    elif h.dtype != np.uint64 or not h.flags.c_contiguous:
        h = np.ascontiguousarray(h.astype(np.uint64))
    assert h.size == 512 * n
    handles = (C.c_void_p * max(n, 1))()
    plan_arr = (C.c_void_p * max(n, 1))(*[p._h.value for p in plans])
    _check(_lib.zc_build_codebooks(n, plan_arr, C.cast(h.ctypes.data, C.POINTER(C.c_uint64)), policy, n_threads, handles),
           "zc_build_codebooks")
    return [Codebook(h) for h in handles[:n]]


def compress(p: Plan, cb: Codebook, d_in: torch.Tensor, d_out: torch.Tensor, d_workspace: torch.Tensor,
             sync: bool = True, stream=None, d_base: Optional[torch.Tensor] = None) -> Optional[int]:
    """zc_compress (zc_compress_xor when d_base is given).  With sync=True returns the container size in bytes
    (and raises on a device-side error); with sync=False the call is asynchronous and returns None."""
    assert d_in.is_cuda and d_out.is_cuda and d_workspace.is_cuda
    assert d_workspace.numel() * d_workspace.element_size() >= p.workspace_bytes
    n = C.c_uint64(0)
    if d_base is None:
        st = _lib.zc_compress(p._h, cb._h, d_in.data_ptr(), d_out.data_ptr(), d_out.numel() * d_out.element_size(),
                              d_workspace.data_ptr(), C.byref(n) if sync else None, _stream_ptr(stream))
    else:
        st = _lib.zc_compress_xor(p._h, cb._h, d_in.data_ptr(), d_base.data_ptr(), d_out.data_ptr(),
                                  d_out.numel() * d_out.element_size(), d_workspace.data_ptr(), C.byref(n) if sync else None,
                                  _stream_ptr(stream))
    _check(st, "zc_compress")
    return n.value if sync else None


def compress_noalloc(p: Plan, cb: Codebook, d_in: torch.Tensor, d_out: torch.Tensor, sync: bool = True,
                     stream=None) -> Optional[int]:
    """zc_compress_noalloc: like compress() but without a workspace argument.  The scratch is a fixed array
    inside the library (at most NOALLOC_MAX_CHUNKS chunks; larger plans raise E_TOO_LARGE).  For callers that
    may not allocate device memory.  Calls that overlap on the GPU must not be issued: they share the scratch."""
    assert d_in.is_cuda and d_out.is_cuda
    n = C.c_uint64(0)
    st = _lib.zc_compress_noalloc(p._h, cb._h, d_in.data_ptr(), d_out.data_ptr(), d_out.numel() * d_out.element_size(),
                                  C.byref(n) if sync else None, _stream_ptr(stream))
    _check(st, "zc_compress_noalloc")
    return n.value if sync else None


def noalloc_status(stream=None) -> int:
    """zc_noalloc_status: device status of the last compress_noalloc call on the current device."""
    return int(_lib.zc_noalloc_status(_stream_ptr(stream)))


def decompress(p: Plan, d_comp: torch.Tensor, comp_bytes: int, d_out: torch.Tensor, d_workspace: torch.Tensor,
               stream=None, d_base: Optional[torch.Tensor] = None) -> None:
    """zc_decompress, or zc_decompress_xor when d_base is given (asynchronous; call device_status() to learn the
    outcome)."""
    assert d_comp.is_cuda and d_out.is_cuda and d_workspace.is_cuda
    assert d_out.numel() * d_out.element_size() >= p.input_bytes
    if d_base is None:
        _check(_lib.zc_decompress(p._h, d_comp.data_ptr(), comp_bytes, d_out.data_ptr(), d_workspace.data_ptr(),
                                  _stream_ptr(stream)), "zc_decompress")
    else:
        _check(_lib.zc_decompress_xor(p._h, d_comp.data_ptr(), comp_bytes, d_base.data_ptr(), d_out.data_ptr(),
                                      d_workspace.data_ptr(), _stream_ptr(stream)), "zc_decompress_xor")


def decompress_chunks(p: Plan, d_comp: torch.Tensor, comp_bytes: int, first_chunk: int, n_chunks: int, d_out: torch.Tensor,
                      d_workspace: torch.Tensor, stream=None) -> None:
    """zc_decompress_chunks: d_out receives the element bytes of chunks first_chunk .. first_chunk + n_chunks - 1."""
    assert d_comp.is_cuda and d_out.is_cuda and d_workspace.is_cuda
    _check(_lib.zc_decompress_chunks(p._h, d_comp.data_ptr(), comp_bytes, first_chunk, n_chunks, d_out.data_ptr(),
                                     d_workspace.data_ptr(), _stream_ptr(stream)), "zc_decompress_chunks")


def device_status(p: Plan, d_workspace: torch.Tensor, stream=None) -> int:
    return _lib.zc_device_status(p._h, d_workspace.data_ptr(), _stream_ptr(stream))


class CompressBatch:
    """Argument arrays of zc_compress_batch, marshalled once; set_codebooks() swaps in new codebooks."""

    def __init__(self, plans, d_ins, d_outs, d_bases=None):
        n = len(plans)
        assert len(d_ins) == n and len(d_outs) == n and (d_bases is None or len(d_bases) == n)
        self.n = n
        self._keep = (list(plans), list(d_ins), list(d_outs), list(d_bases) if d_bases is not None else None)
        self.bases = _base_array(d_bases, n)     # XOR-delta form when given
        self.plans = (C.c_void_p * n)(*[p._h.value for p in plans])
        self.ins = (C.c_void_p * n)(*[t.data_ptr() for t in d_ins])
        self.outs = (C.c_void_p * n)(*[t.data_ptr() for t in d_outs])
        self.caps = (C.c_size_t * n)(*[t.numel() for t in d_outs])
        self.cbs = (C.c_void_p * n)()
        self._cbs = None
        self.workspace_bytes = _lib.zc_compress_batch_workspace_bytes(n, self.plans)

    def set_codebooks(self, codebooks):
        assert len(codebooks) == self.n
        self._cbs = list(codebooks)
        for i, cb in enumerate(codebooks):
            self.cbs[i] = cb._h


def compress_batch(batch: CompressBatch, d_workspace: torch.Tensor, sync: bool = True, stream=None):
    """zc_compress_batch.  Returns the list of container sizes (sync=True) or None (asynchronous)."""
    sizes = (C.c_uint64 * max(batch.n, 1))()
    _check(_lib.zc_compress_batch_xor(batch.n, batch.plans, batch.cbs, batch.ins, batch.bases, batch.outs, batch.caps,
                                      d_workspace.data_ptr(), d_workspace.numel(), sizes if sync else None, _stream_ptr(stream)),
           "zc_compress_batch")
    return sizes[: batch.n] if sync else None


class DecompressBatch:
    """Argument arrays of zc_decompress_batch, marshalled once and reusable for repeated calls."""

    def __init__(self, plans, d_comps, comp_bytes, d_outs, d_bases=None):
        n = len(plans)
        assert len(d_comps) == n and len(comp_bytes) == n and len(d_outs) == n and (d_bases is None or len(d_bases) == n)
        self.n = n
        self._keep = (list(plans), list(d_comps), list(d_outs), list(d_bases) if d_bases is not None else None)
        self.bases = _base_array(d_bases, n)     # XOR-delta form when given
        self.plans = (C.c_void_p * n)(*[p._h.value for p in plans])
        self.comps = (C.c_void_p * n)(*[t.data_ptr() for t in d_comps])
        self.sizes = (C.c_size_t * n)(*[int(b) for b in comp_bytes])
        self.outs = (C.c_void_p * n)(*[t.data_ptr() for t in d_outs])


def decompress_batch(batch: DecompressBatch, d_workspace: torch.Tensor, stream=None) -> None:
    """zc_decompress_batch (asynchronous; read the outcome with batch_status)."""
    _check(_lib.zc_decompress_batch_xor(batch.n, batch.plans, batch.comps, batch.sizes, batch.bases, batch.outs,
                                        d_workspace.data_ptr(), _stream_ptr(stream)), "zc_decompress_batch")


def batch_status(d_workspace: torch.Tensor, stream=None):
    """zc_batch_status: (status, index of the failing tensor or None)."""
    failed = C.c_uint32(0xFFFFFFFF)
    st = _lib.zc_batch_status(d_workspace.data_ptr(), C.byref(failed), _stream_ptr(stream))
    return st, (None if failed.value == 0xFFFFFFFF else failed.value)


# ---- operators on FP8 matrices with block scales ----

def _real_matrix(t: torch.Tensor, what: str):
    """(type code, address, row pitch in elements) of a 2-D tensor of real numbers with contiguous rows."""
    real = _REAL.get(t.dtype)
    if real is None:
        raise TypeError(f"{what}: float32, bfloat16 or float16 is wanted, got {t.dtype}")
    stride, shape = t.stride(), t.shape
    if len(stride) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{what}: a matrix with contiguous rows is wanted, got shape {tuple(shape)}, strides {stride}")
    return real, t.data_ptr(), (stride[0] if shape[0] > 1 else max(stride[0], shape[1]))


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _same_device(*indices) -> int:
    """The library launches on the current device: tensors of another one (or of the host, -1) are refused instead of read from
    there.  Returns the device's index."""
    if -1 in indices:
        raise ValueError("a tensor is in host memory")
    dev = _current_device()
    for i in indices:
        if i != dev:
            raise ValueError(f"a tensor is on cuda:{i}, the current device is cuda:{dev}")
    return dev


def _stream_of(stream, dev: int, _raw=getattr(torch._C, "_cuda_getCurrentRawStream", None)) -> int:
    return _raw(dev) if stream is None and _raw is not None else _stream_ptr(stream)


class Fp8Matrix:
    """zc_fp8_matrix: FP8 elements [rows, cols] and E8M0 scale bytes [ceil(rows / block_rows), ceil(cols / 128)], both
    uint8 with contiguous rows; the elements' rows have a pitch that is a multiple of 16 bytes.  Marshalled once; keeps
    its tensors alive."""

    def __init__(self, elems: torch.Tensor, scales: torch.Tensor, fmt: int = FMT_FP8_E4M3, block_rows: int = 1):
        for t, what in ((elems, "elems"), (scales, "scales")):
            if t.dtype != torch.uint8 or t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
                raise ValueError(f"{what}: a uint8 matrix with contiguous rows is wanted")
        rows, cols = elems.shape
        if block_rows in (1, 128) and tuple(scales.shape) != (-(-rows // block_rows), -(-cols // 128)):
            raise ValueError(f"scales: shape {tuple(scales.shape)} does not fit {rows} x {cols} elements in blocks of {block_rows} x 128")
        self.elems, self.scales, self.format, self.block_rows = elems, scales, fmt, block_rows
        pitch = lambda t: t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])  # noqa: E731
        self.desc = Fp8MatrixDesc(elems.data_ptr(), scales.data_ptr(), rows, cols, -(-pitch(elems) // 16) * 16 if rows <= 1 else pitch(elems),
                                  pitch(scales), fmt, block_rows)
        self._ref = C.addressof(self.desc)
        self.shape = (rows, cols)
        if elems.get_device() != scales.get_device():
            raise ValueError(f"elems are on {elems.device}, scales on {scales.device}")
        self._dev = elems.get_device()           # -1: host memory


def fp8_empty(rows: int, cols: int, fmt: int = FMT_FP8_E4M3, block_rows: int = 1, device="cuda") -> Fp8Matrix:
    """An Fp8Matrix of new buffers, contents undefined."""
    pitch = -(-cols // 16) * 16
    elems = torch.empty((rows, pitch), dtype=torch.uint8, device=device)[:, :cols]
    return Fp8Matrix(elems, torch.empty((-(-rows // block_rows), -(-cols // 128)), dtype=torch.uint8, device=device), fmt, block_rows)


def fp8_quantize(d_in: torch.Tensor, q: Optional[Fp8Matrix], qt: Optional[Fp8Matrix] = None, stream=None) -> Optional[Fp8Matrix]:
    """zc_fp8_quantize: the matrix d_in into q and / or its transposed form into qt (asynchronous)."""
    real, ptr, ld = _real_matrix(d_in, "d_in")
    rows, cols = d_in.shape
    dev = d_in.get_device()
    if q is not None and q.shape != (rows, cols):
        raise ValueError(f"q is {q.shape}, the matrix to quantise asks for {(rows, cols)}")
    if qt is not None and qt.shape != (cols, rows):
        raise ValueError(f"qt is {qt.shape}, the matrix to quantise asks for {(cols, rows)}")
    dev = _same_device(dev, q._dev if q is not None else dev, qt._dev if qt is not None else dev)
    status = _lib.zc_fp8_quantize(real, ptr, ld, q._ref if q is not None else None, qt._ref if qt is not None else None, _stream_of(stream, dev))
    if status != OK:
        raise ZcError(status, "zc_fp8_quantize")
    return q


def fp8_matmul(a: Fp8Matrix, b: Fp8Matrix, d_out: torch.Tensor, accumulate: bool = False, stream=None) -> torch.Tensor:
    """zc_fp8_matmul: d_out = a b^T, or d_out += a b^T (asynchronous)."""
    real, ptr, ld = _real_matrix(d_out, "d_out")
    if d_out.shape != (a.shape[0], b.shape[0]):
        raise ValueError(f"d_out is {tuple(d_out.shape)}, the product is {(a.shape[0], b.shape[0])}")
    dev = _same_device(a._dev, b._dev, d_out.get_device())
    status = _lib.zc_fp8_matmul(a._ref, b._ref, real, ptr, ld, accumulate, _stream_of(stream, dev))
    if status != OK:
        raise ZcError(status, "zc_fp8_matmul")
    return d_out


def fp8_status(stream=None) -> int:
    """zc_fp8_status: device status of the fp8_matmul and fp8_moe calls on the current device since the last query."""
    return int(_lib.zc_fp8_status(_stream_ptr(stream)))


class Fp8MoeLayer:
    """zc_fp8_moe_layer: router [experts, hidden] in BF16 or FP16 (row pitch a multiple of 8), gate_up uint8
    [experts, 2, inter, hidden] and down uint8 [experts, hidden, inter] (row pitches multiples of 16, no gaps between
    matrices), scale bytes [experts, 2, ceil(inter / 128), ceil(hidden / 128)] and [experts, ceil(hidden / 128),
    ceil(inter / 128)], contiguous.  Marshalled once; keeps its tensors alive."""

    def __init__(self, router: torch.Tensor, gate_up: torch.Tensor, gate_up_scales: torch.Tensor, down: torch.Tensor,
                 down_scales: torch.Tensor, top_k: int, fmt: int = FMT_FP8_E4M3):
        experts, two, inter, hidden = gate_up.shape
        blocks = lambda n: -(-n // 128)  # noqa: E731
        if two != 2 or tuple(down.shape) != (experts, hidden, inter) or tuple(router.shape) != (experts, hidden):
            raise ValueError(f"gate_up {tuple(gate_up.shape)}, down {tuple(down.shape)} and router {tuple(router.shape)} do not belong together")
        if tuple(gate_up_scales.shape) != (experts, 2, blocks(inter), blocks(hidden)) or tuple(down_scales.shape) != (experts, blocks(hidden), blocks(inter)):
            raise ValueError("the scale bytes do not fit the matrices in blocks of 128 x 128")
        if any(t.dtype != torch.uint8 for t in (gate_up, gate_up_scales, down, down_scales)):
            raise ValueError("weights and scale bytes are uint8")
        if not gate_up_scales.is_contiguous() or not down_scales.is_contiguous():
            raise ValueError("scale bytes are contiguous")
        for t in (gate_up, down):
            pitch = t.stride(-2)
            want = tuple(pitch * math.prod(t.shape[i + 1: -1]) for i in range(t.dim() - 1)) + (1,)
            if any(s != w for s, w, n in zip(t.stride(), want, t.shape) if n > 1):
                raise ValueError(f"matrices follow one another with one row pitch: strides {t.stride()}")
        real, ptr, ld = _real_matrix(router, "router")
        ld = ld if experts > 1 else -(-ld // 8) * 8              # a single row has no pitch of its own
        self.experts, self.hidden, self.inter, self.top_k, self.dtype = experts, hidden, inter, top_k, router.dtype
        self.tensors = (router, gate_up, gate_up_scales, down, down_scales)
        self.desc = Fp8MoeLayerDesc(ptr, gate_up.data_ptr(), gate_up_scales.data_ptr(), down.data_ptr(), down_scales.data_ptr(), ld,
                                    gate_up.stride(-2), down.stride(-2), experts, top_k, hidden, inter, fmt, real)
        self._ref = C.addressof(self.desc)
        self._dev = router.get_device()
        if any(t.get_device() != self._dev for t in self.tensors):
            raise ValueError("the layer's tensors are on several devices")

    def workspace_bytes(self, n_tokens: int) -> int:
        return int(_lib.zc_fp8_moe_workspace_bytes(self._ref, n_tokens))


def fp8_moe(layer: Fp8MoeLayer, d_x: torch.Tensor, d_out: torch.Tensor, d_workspace: torch.Tensor, d_ids: Optional[torch.Tensor] = None,
            d_weights: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """zc_fp8_moe: d_out = the layer applied to the tokens d_x (asynchronous).  d_ids (int32) and d_weights (float32),
    [tokens, top_k] and contiguous, receive the experts chosen and their weights."""
    _, x_ptr, ld_x = _real_matrix(d_x, "d_x")
    _, y_ptr, ld_y = _real_matrix(d_out, "d_out")
    tokens = d_x.shape[0]
    if d_x.dtype != layer.dtype or d_out.dtype != layer.dtype:
        raise TypeError(f"the layer works in {layer.dtype}, d_x is {d_x.dtype}, d_out {d_out.dtype}")
    if d_x.shape[1] != layer.hidden or d_out.shape != d_x.shape:
        raise ValueError(f"d_x is {tuple(d_x.shape)}, d_out {tuple(d_out.shape)}, the layer's width {layer.hidden}")
    for t, dtype in ((d_ids, torch.int32), (d_weights, torch.float32)):
        if t is not None and (t.dtype != dtype or tuple(t.shape) != (tokens, layer.top_k) or not t.is_contiguous()):
            raise ValueError(f"d_ids and d_weights are contiguous int32 and float32 of shape {(tokens, layer.top_k)}")
    devices = [t.get_device() for t in (d_x, d_out, d_workspace, d_ids, d_weights) if t is not None]
    dev = _same_device(layer._dev, *devices)
    status = _lib.zc_fp8_moe(layer._ref, tokens, x_ptr, ld_x if tokens > 1 else -(-ld_x // 8) * 8, y_ptr, ld_y, d_ids.data_ptr() if d_ids is not None else None,
                             d_weights.data_ptr() if d_weights is not None else None, d_workspace.data_ptr(),
                             d_workspace.numel() * d_workspace.element_size(), _stream_of(stream, dev))
    if status != OK:
        raise ZcError(status, "zc_fp8_moe")
    return d_out


# ---- a quantised cache of keys and values ----

class KvCache:
    """zc_kv_cache: the keys and values of one layer in pages.  Elements uint8 [pages, kv_heads, page_tokens, head_dim / 2]
    (FMT_FP4_E2M1) or [..., head_dim] (FMT_FP8_E4M3) and scale bytes uint8 [pages, kv_heads, page_tokens, head_dim / 32], all
    contiguous.  Marshalled once; keeps its tensors alive."""

    def __init__(self, k_elems: torch.Tensor, k_scales: torch.Tensor, v_elems: torch.Tensor, v_scales: torch.Tensor, fmt: int = FMT_FP4_E2M1):
        if fmt not in (FMT_FP4_E2M1, FMT_FP8_E4M3):
            raise ValueError("a cache is FMT_FP4_E2M1 or FMT_FP8_E4M3")
        if any(t.dtype != torch.uint8 or t.dim() != 4 or not t.is_contiguous() for t in (k_elems, k_scales, v_elems, v_scales)):
            raise ValueError("elements and scale bytes are contiguous uint8 tensors [pages, kv_heads, page_tokens, bytes]")
        pages, heads, tokens, width = k_elems.shape
        dim = width * (2 if fmt == FMT_FP4_E2M1 else 1)
        if v_elems.shape != k_elems.shape or any(tuple(t.shape) != (pages, heads, tokens, dim // 32) for t in (k_scales, v_scales)):
            raise ValueError(f"elements {tuple(k_elems.shape)}, {tuple(v_elems.shape)} and scales {tuple(k_scales.shape)}, {tuple(v_scales.shape)} do not belong together")
        self.k_elems, self.k_scales, self.v_elems, self.v_scales, self.format = k_elems, k_scales, v_elems, v_scales, fmt
        self.n_pages, self.kv_heads, self.page_tokens, self.head_dim = pages, heads, tokens, dim
        self.desc = KvCacheDesc(k_elems.data_ptr(), k_scales.data_ptr(), v_elems.data_ptr(), v_scales.data_ptr(), pages, tokens, heads, dim, fmt)
        self._ref = C.addressof(self.desc)
        self._dev = k_elems.get_device()
        if any(t.get_device() != self._dev for t in (k_scales, v_elems, v_scales)):
            raise ValueError("the cache's tensors are on several devices")


def kv_empty(n_pages: int, kv_heads: int, page_tokens: int, head_dim: int, fmt: int = FMT_FP4_E2M1, device="cuda") -> KvCache:
    """A KvCache of new buffers, contents undefined."""
    make = lambda width: torch.empty((n_pages, kv_heads, page_tokens, width), dtype=torch.uint8, device=device)  # noqa: E731
    width = head_dim // 2 if fmt == FMT_FP4_E2M1 else head_dim
    return KvCache(make(width), make(head_dim // 32), make(width), make(head_dim // 32), fmt)


class KvBatch:
    """zc_kv_batch: page_table int32 [sequences, pages] with contiguous rows, lens int32 [sequences], first int32 [sequences + 1], all read
    on the device; max_new: rows that a sequence is expected to have at most (it decides which kernels run, not what they
    compute).  Marshalled once; keeps its tensors alive."""

    def __init__(self, page_table: torch.Tensor, lens: torch.Tensor, first: torch.Tensor, max_new: int = 1):
        if any(t.dtype != torch.int32 for t in (page_table, lens, first)):
            raise ValueError("page_table, lens and first are int32")
        if page_table.dim() != 2 or (page_table.stride(1) != 1 and page_table.shape[1] > 1):
            raise ValueError("page_table is a matrix with contiguous rows")
        seqs, pages = page_table.shape
        if tuple(lens.shape) != (seqs,) or tuple(first.shape) != (seqs + 1,) or not lens.is_contiguous() or not first.is_contiguous():
            raise ValueError(f"lens and first are contiguous, of {seqs} and {seqs + 1} elements")
        if not 0 <= max_new < 1 << 32:
            raise ValueError("max_new is out of range")
        self.page_table, self.lens, self.first, self.max_new, self.n_seqs = page_table, lens, first, max_new, seqs
        pitch = page_table.stride(0) if seqs > 1 else max(page_table.stride(0), pages)
        self._front, self._back = (page_table.data_ptr(), lens.data_ptr(), first.data_ptr(), pitch), (pages, seqs, max_new)
        self._dev = lens.get_device()
        if any(t.get_device() != self._dev for t in (page_table, first)):
            raise ValueError("the batch's tensors are on several devices")

    def _ref(self, n_rows: int) -> bytes:
        """The descriptor for tensors of n_rows rows."""
        return _pack_batch(*self._front, n_rows, *self._back)


# the C structures as packed bytes: made in one go, and nobody else's while a call is under way
_pack_tensor = struct.Struct("<QQQ").pack                    # zc_kv_tensor
_pack_batch = struct.Struct("<QQQQQIII4x").pack              # zc_kv_batch
_pack_attention = struct.Struct("<QQQQQQQIIfII4x").pack      # zc_kv_attention_args: q, out, lse, type, heads, scale, causal, window
assert len(_pack_tensor(0, 0, 0)) == C.sizeof(KvTensorDesc) and len(_pack_batch(*[0] * 8)) == C.sizeof(KvBatchDesc) and len(_pack_attention(*[0] * 12)) == C.sizeof(KvAttentionArgs)


def _kv_strides(t: torch.Tensor, what: str, heads: int, dim: int):
    """(pitch of rows, of heads) of a tensor [rows, heads, dim]."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim or stride[2] != 1:
        raise ValueError(f"{what}: [rows, {heads}, {dim}] with contiguous heads is wanted, got shape {tuple(shape)}, strides {stride}")
    return stride[0], stride[1]


def _kv_rows(call, where: str, cache: KvCache, batch: KvBatch, d_k: Optional[torch.Tensor], d_v: Optional[torch.Tensor], stream):
    one = d_k if d_k is not None else d_v
    if one is None:
        raise ValueError("neither keys nor values")
    dtype, rows, dev = one.dtype, one.shape[0], one.get_device()
    real = _REAL.get(dtype)
    if real is None:
        raise TypeError(f"float32, bfloat16 or float16 is wanted, got {dtype}")
    heads, dim = cache.kv_heads, cache.head_dim
    k = v = None
    if d_k is not None:
        k = _pack_tensor(d_k.data_ptr(), *_kv_strides(d_k, "d_k", heads, dim))
    if d_v is not None:
        v = _pack_tensor(d_v.data_ptr(), *_kv_strides(d_v, "d_v", heads, dim))
        if d_v is not one and (d_v.dtype != dtype or d_v.shape[0] != rows):
            raise ValueError("d_k and d_v are of one type and have the same rows")
    dev = _same_device(cache._dev, batch._dev, dev, d_v.get_device() if d_v is not None else dev)
    status = call(cache._ref, batch._ref(rows), real, k, v, _stream_of(stream, dev))
    if status != OK:
        raise ZcError(status, where)


def kv_append(cache: KvCache, batch: KvBatch, d_k: torch.Tensor, d_v: torch.Tensor, stream=None) -> None:
    """zc_kv_append: keys and values [rows, kv_heads, head_dim] of the batch's rows into the cache (asynchronous)."""
    if d_k is None or d_v is None:
        raise ValueError("keys and values are written together")
    _kv_rows(_lib.zc_kv_append, "zc_kv_append", cache, batch, d_k, d_v, stream)


def kv_read(cache: KvCache, batch: KvBatch, d_k: Optional[torch.Tensor], d_v: Optional[torch.Tensor], stream=None):
    """zc_kv_read: the batch's rows out of the cache into d_k and / or d_v (asynchronous)."""
    _kv_rows(_lib.zc_kv_read, "zc_kv_read", cache, batch, d_k, d_v, stream)
    return d_k, d_v


def kv_attention_workspace_bytes(cache: KvCache, batch: KvBatch, q_heads: int) -> int:
    """zc_kv_attention_workspace_bytes."""
    return int(_lib.zc_kv_attention_workspace_bytes(cache._ref, batch._ref(1), q_heads))


def kv_attention(cache: KvCache, batch: KvBatch, d_q: torch.Tensor, d_out: torch.Tensor, d_workspace: torch.Tensor, scale: Optional[float] = None,
                 causal: bool = True, window: int = 0, d_lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """zc_kv_attention: d_out[rows, q_heads, head_dim] = attention of d_q over the cache (asynchronous).  scale: 1 / sqrt(head_dim) where it is not
    given; d_lse: float32 [rows, q_heads], contiguous, receives the logarithms of the sums."""
    real = _REAL.get(d_q.dtype)
    if real is None or d_out.dtype != d_q.dtype:
        raise TypeError(f"d_q and d_out are bfloat16 or float16, got {d_q.dtype} and {d_out.dtype}")
    shape, dim = d_q.shape, cache.head_dim
    if d_out.shape != shape or len(shape) != 3:
        raise ValueError(f"d_q is {tuple(shape)}, d_out {tuple(d_out.shape)}")
    if not 0 <= window < 1 << 32:
        raise ValueError("window is out of range")
    if not d_workspace.is_contiguous():                         # its bytes are counted as if they followed one another
        raise ValueError("d_workspace is contiguous")
    rows, heads = shape[0], shape[1]
    dev, lse = d_q.get_device(), 0
    dev = _same_device(cache._dev, batch._dev, dev, d_out.get_device(), d_workspace.get_device(), d_lse.get_device() if d_lse is not None else dev)
    if d_lse is not None:
        if d_lse.dtype != torch.float32 or d_lse.shape != (rows, heads) or not d_lse.is_contiguous():
            raise ValueError(f"d_lse is contiguous float32 of shape {(rows, heads)}")
        lse = d_lse.data_ptr()
    args = _pack_attention(d_q.data_ptr(), *_kv_strides(d_q, "d_q", heads, dim), d_out.data_ptr(), *_kv_strides(d_out, "d_out", heads, dim), lse, real, heads,
                           dim ** -0.5 if scale is None else scale, causal, window)
    status = _lib.zc_kv_attention(cache._ref, batch._ref(rows), args, d_workspace.data_ptr(), d_workspace.nbytes, _stream_of(stream, dev))
    if status != OK:
        raise ZcError(status, "zc_kv_attention")
    return d_out


def kv_status(stream=None) -> int:
    """zc_kv_status: device status of the kv_* calls on the current device since the last query."""
    return int(_lib.zc_kv_status(_stream_ptr(stream)))


def validate_container(p: Plan, h_container) -> int:
    c = np.ascontiguousarray(h_container, np.uint8)
    return _lib.zc_validate_container(p._h, c.ctypes.data, c.size)


def stats(p: Plan, cb: Codebook, h_hist, h_header=None) -> Stats:
    h = np.ascontiguousarray(np.asarray(h_hist).astype(np.uint64)).reshape(512)
    hd = None
    if h_header is not None:
        hd = np.ascontiguousarray(h_header, np.uint8)
        assert hd.size >= 128
    out = Stats()
    _check(_lib.zc_stats(p._h, cb._h, h.ctypes.data_as(C.POINTER(C.c_uint64)), hd.ctypes.data if hd is not None else None,
                         C.byref(out)), "zc_stats")
    return out


def test_split16(fmt: int, in16: np.ndarray):
    a = np.ascontiguousarray(in16, np.uint8)
    e, sm = np.zeros(8, np.uint8), np.zeros(8, np.uint8)
    _check(_lib.zc_test_split16(fmt, a.ctypes.data, e.ctypes.data, sm.ctypes.data), "zc_test_split16")
    return e, sm


def test_merge16(fmt: int, e8: np.ndarray, sm8: np.ndarray):
    e, sm = np.ascontiguousarray(e8, np.uint8), np.ascontiguousarray(sm8, np.uint8)
    out = np.zeros(16, np.uint8)
    _check(_lib.zc_test_merge16(fmt, e.ctypes.data, sm.ctypes.data, out.ctypes.data), "zc_test_merge16")
    return out


test_split16.__test__ = False
test_merge16.__test__ = False


def test_set_wait_limit(polls: int) -> None:
    """zc_test_set_wait_limit (0 restores the default)."""
    _lib.zc_test_set_wait_limit(polls)


def test_stall_encoder(first_ticket: int) -> None:
    """zc_test_stall_encoder (0 turns the stall off)."""
    _lib.zc_test_stall_encoder(first_ticket)


def test_stall_decoder(on: bool) -> None:
    """zc_test_stall_decoder."""
    _lib.zc_test_stall_decoder(1 if on else 0)


def test_stall_math(on: bool) -> None:
    """zc_test_stall_math."""
    _lib.zc_test_stall_math(1 if on else 0)


def test_fp8_marks() -> int:
    """zc_test_fp8_marks."""
    return int(_lib.zc_test_fp8_marks())


def test_debug_counts():
    """zc_test_debug_counts: (refused shared accesses, refused global accesses) of a development build, else None."""
    out = (C.c_uint32 * 2)()
    return (int(out[0]), int(out[1])) if _lib.zc_test_debug_counts(out) else None


def test_encoder_workers(p: Plan, n_coded: int, any_base: bool, total_chunks: int) -> int:
    """zc_test_encoder_workers."""
    return int(_lib.zc_test_encoder_workers(p._h, n_coded, int(any_base), total_chunks))


def test_decoder_warps(p: Plan, both_coded: bool) -> int:
    return int(_lib.zc_test_decoder_warps(p._h, 1 if both_coded else 0))


def test_decoder_pieces(p: Plan, any_base: bool, total_chunks: int):
    """zc_test_decoder_pieces: where the pieces of a slice end, in 65536ths of it."""
    end = (C.c_uint32 * 5)()
    return [int(end[i]) for i in range(_lib.zc_test_decoder_pieces(p._h, int(any_base), total_chunks, end))]
