"""Thin ctypes binding of ``libmage.so``: argument marshalling only.

Function names and arguments mirror ``include/mage.h``.  Tensors are torch CUDA
tensors (torch is used for device memory and streams, nothing else); every
step of the path runs inside the library's kernels.  There is no fallback: if
the library has not been built, the first call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmage.so")
_lib = None

MAGE_OK = 0
FLAG_SIMT_KERNELS = 1
FLAG_TEST_STALL = 2
DEV_BAD_INDEX, DEV_BAD_PAGE, DEV_TIMEOUT, DEV_CACHE_FULL, DEV_BAD_CHUNK = 1, 2, 4, 8, 16


class MageError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


class mage_k8_t(ctypes.Structure):
    _fields_ = [("k8_cache", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("scratch", ctypes.c_void_p)]


class mage_kv_t(ctypes.Structure):
    _fields_ = [
        ("P", ctypes.c_int32), ("H_q", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("d", ctypes.c_int32),
        ("B", ctypes.c_int32), ("page_size", ctypes.c_int32),
        ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
        ("stride_p", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64),
        ("block_table", ctypes.c_void_p), ("max_pages", ctypes.c_int32), ("num_pages", ctypes.c_int32),
        ("seq_lens", ctypes.c_void_p), ("N_max", ctypes.c_int32), ("flags", ctypes.c_int32),
    ]


class mage_chunk_t(ctypes.Structure):
    _fields_ = [("q_start", ctypes.c_void_p), ("n_tokens", ctypes.c_int32), ("max_len", ctypes.c_int32)]


class mage_kv8_t(ctypes.Structure):
    _fields_ = [("k8", ctypes.c_void_p), ("v8", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class mage_kv4_t(ctypes.Structure):
    _fields_ = [("k4", ctypes.c_void_p), ("v4", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class mage_rope_t(ctypes.Structure):
    _fields_ = [
        ("d", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("halves", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("mult", ctypes.c_float),
        ("inv_freq", ctypes.c_void_p), ("axis_of_pair", ctypes.c_uint8 * 64),
    ]


EXPORTS = ("mage_pruned_workspace_bytes", "mage_exact_select_pruned", "mage_quest_workspace_bytes", "mage_quest_build", "mage_quest_select", "mage_append_block", "mage_workspace_bytes", "mage_exact_select", "mage_exact_select_events", "mage_exact_select_static", "mage_exact_attn", "mage_select_scores", "mage_topk", "mage_sparse_block_attn",
           "mage_k8_scratch_bytes", "mage_k8_quantize_cache", "mage_exact_select_k8", "mage_exact_select_k8_events", "mage_sparse_block_attn_k8",
           "mage_rope", "mage_append_chunk", "mage_append_chunk_kv8", "mage_kv8_read", "mage_chunk_workspace_bytes", "mage_chunk_attn", "mage_chunk_attn_kv8",
           "mage_append_chunk_kv4", "mage_kv4_read", "mage_chunk_workspace_bytes_kv4", "mage_chunk_attn_kv4", "mage_rope_append_chunk", "mage_rope_append_chunk_kv8", "mage_rope_append_chunk_kv4",
           "mage_status_string", "mage_launch_count")


def load():
    """Load libmage.so (once).  Raises if it is missing: there is no other implementation to fall back to."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is not built; run `python -m paper_2602_14209_b200.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64
    lib.mage_workspace_bytes.restype = ctypes.c_size_t
    lib.mage_workspace_bytes.argtypes = [ctypes.POINTER(mage_kv_t), i32]
    lib.mage_exact_select.restype = ctypes.c_int
    lib.mage_exact_select.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.mage_exact_select_events.restype = ctypes.c_int
    lib.mage_exact_select_events.argtypes = lib.mage_exact_select.argtypes + [ctypes.POINTER(ctypes.c_void_p)]
    lib.mage_exact_select_static.restype = ctypes.c_int
    lib.mage_exact_select_static.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, ctypes.c_float, vp, vp, vp, vp]
    lib.mage_exact_attn.restype = ctypes.c_int
    lib.mage_exact_attn.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, ctypes.c_float, vp, vp, ctypes.c_size_t, vp, vp]
    lib.mage_select_scores.restype = ctypes.c_int
    lib.mage_select_scores.argtypes = [ctypes.POINTER(mage_kv_t), vp, ctypes.c_float, vp, vp, ctypes.c_size_t, vp, vp]
    lib.mage_topk.restype = ctypes.c_int
    lib.mage_topk.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, ctypes.c_size_t, vp]
    lib.mage_sparse_block_attn.restype = ctypes.c_int
    lib.mage_sparse_block_attn.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, vp, vp, i32, ctypes.c_float, vp, vp, ctypes.c_size_t, vp, vp]
    lib.mage_append_block.restype = ctypes.c_int
    lib.mage_append_block.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, vp, vp]
    lib.mage_pruned_workspace_bytes.restype = ctypes.c_size_t
    lib.mage_pruned_workspace_bytes.argtypes = [ctypes.POINTER(mage_kv_t), i32]
    lib.mage_exact_select_pruned.restype = ctypes.c_int
    lib.mage_exact_select_pruned.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, ctypes.c_float, i32, ctypes.c_float, vp, vp, vp, vp, vp, vp,
                                             ctypes.c_size_t, vp, vp]
    lib.mage_quest_workspace_bytes.restype = ctypes.c_size_t
    lib.mage_quest_workspace_bytes.argtypes = [ctypes.POINTER(mage_kv_t), i32]
    lib.mage_quest_build.restype = ctypes.c_int
    lib.mage_quest_build.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, vp]
    lib.mage_quest_select.restype = ctypes.c_int
    lib.mage_quest_select.argtypes = [ctypes.POINTER(mage_kv_t), vp, vp, vp, i32, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.mage_k8_scratch_bytes.restype = ctypes.c_size_t
    lib.mage_k8_scratch_bytes.argtypes = [ctypes.POINTER(mage_kv_t)]
    lib.mage_k8_quantize_cache.restype = ctypes.c_int
    lib.mage_k8_quantize_cache.argtypes = [ctypes.POINTER(mage_kv_t), i32, vp, vp, vp, vp]
    lib.mage_exact_select_k8.restype = ctypes.c_int
    lib.mage_exact_select_k8.argtypes = [ctypes.POINTER(mage_kv_t), ctypes.POINTER(mage_k8_t), vp, vp, vp, ctypes.c_float, vp, vp, vp,
                                         ctypes.c_size_t, vp, vp]
    lib.mage_exact_select_k8_events.restype = ctypes.c_int
    lib.mage_exact_select_k8_events.argtypes = lib.mage_exact_select_k8.argtypes + [ctypes.POINTER(ctypes.c_void_p)]
    lib.mage_sparse_block_attn_k8.restype = ctypes.c_int
    lib.mage_sparse_block_attn_k8.argtypes = [ctypes.POINTER(mage_kv_t), ctypes.POINTER(mage_k8_t), vp, vp, vp, vp, vp, i32, ctypes.c_float,
                                              vp, vp, ctypes.c_size_t, vp, vp]
    # (the calls on packed chunks take their structs by address, kept by the objects: a pointer object per call would cost more)
    i64, vs = ctypes.c_int64, [vp, ctypes.c_int64, ctypes.c_int64]
    lib.mage_rope.restype = ctypes.c_int
    lib.mage_rope.argtypes = [vp, i32, vp, i64, i32] + vs * 2 + [i32] + vs * 2 + [vp]
    lib.mage_append_chunk.restype = ctypes.c_int
    lib.mage_append_chunk.argtypes = [vp, vp, vp, vp, i64, i64, vp, vp]
    lib.mage_append_chunk_kv8.restype = ctypes.c_int
    lib.mage_append_chunk_kv8.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp]
    lib.mage_kv8_read.restype = ctypes.c_int
    lib.mage_kv8_read.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.mage_chunk_workspace_bytes.restype = ctypes.c_size_t
    lib.mage_chunk_workspace_bytes.argtypes = [vp, vp]
    lib.mage_chunk_workspace_bytes_kv4.restype = ctypes.c_size_t
    lib.mage_chunk_workspace_bytes_kv4.argtypes = [vp, vp]
    lib.mage_chunk_attn.restype = ctypes.c_int
    lib.mage_chunk_attn.argtypes = [vp, vp, vp, i64, i64, i32, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp, vp]
    for to, of in (("mage_append_chunk_kv4", lib.mage_append_chunk_kv8), ("mage_kv4_read", lib.mage_kv8_read)):
        getattr(lib, to).restype, getattr(lib, to).argtypes = ctypes.c_int, of.argtypes
    for form, arrays in (("", []), ("_kv8", [vp]), ("_kv4", [vp])):
        f = getattr(lib, "mage_rope_append_chunk" + form)
        f.restype, f.argtypes = ctypes.c_int, [vp] + arrays + [vp, vp, vp, i64] + vs * 2 + [vp, vp, i64, i64, vp, vp]
    lib.mage_chunk_attn_kv4.restype = ctypes.c_int
    lib.mage_chunk_attn_kv4.argtypes = [vp, vp, vp, vp, i64, i64, i32, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.mage_chunk_attn_kv8.restype = ctypes.c_int
    lib.mage_chunk_attn_kv8.argtypes = [vp, vp, vp, vp, i64, i64, i32, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.mage_status_string.restype = ctypes.c_char_p
    lib.mage_status_string.argtypes = [ctypes.c_int]
    lib.mage_launch_count.restype = u64
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load().mage_status_string(int(code)).decode()


def launch_count() -> int:
    return int(load().mage_launch_count())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


class KVCache:
    """Host-side description of the prefix KV cache of a batch of P problems (``mage_kv_t``).

    Contiguous: ``k``, ``v`` are [P, H_kv, N_max, d] bf16 views (any strides with d contiguous).
    Paged: ``k``, ``v`` are pools [num_pages, H_kv, page_size, d] and ``block_table`` is [P, max_pages] int32.
    ``seq_lens`` is a device int32 [P] tensor or None (every problem has N_max keys).
    The object only keeps references; it owns no memory of its own.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, H_q: int, B: int, seq_lens: Optional[torch.Tensor] = None,
                 block_table: Optional[torch.Tensor] = None, N_max: Optional[int] = None, flags: int = 0):
        assert k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16 and k.dim() == 4 and k.shape == v.shape
        assert k.stride() == v.stride() and k.stride(3) == 1
        self.k, self.v, self.seq_lens, self.block_table = k, v, seq_lens, block_table
        c = mage_kv_t()
        if block_table is None:
            P, H_kv, n, d = k.shape
            c.page_size = 0
            c.stride_p, c.stride_h, c.stride_n = k.stride(0), k.stride(1), k.stride(2)
            c.N_max = n if N_max is None else N_max
        else:
            assert k.is_contiguous() and v.is_contiguous() and block_table.dtype == torch.int32 and block_table.is_contiguous()
            num_pages, H_kv, page, d = k.shape
            P = block_table.shape[0]
            c.page_size, c.num_pages, c.max_pages = page, num_pages, block_table.shape[1]
            c.block_table = block_table.data_ptr()
            assert N_max is not None
            c.N_max = N_max
        c.P, c.H_q, c.H_kv, c.d, c.B, c.flags = P, H_q, H_kv, d, B, flags
        c.k_cache, c.v_cache = k.data_ptr(), v.data_ptr()
        if seq_lens is not None:
            assert seq_lens.dtype == torch.int32 and seq_lens.numel() == P and seq_lens.is_cuda
            c.seq_lens = seq_lens.data_ptr()
        self.c = c
        self.at = ctypes.addressof(c)
        self.P, self.H_q, self.H_kv, self.d, self.B, self.N_max = P, H_q, H_kv, d, B, int(c.N_max)
        self.device = k.device

    def workspace_bytes(self, k_max: int = 1) -> int:
        return int(load().mage_workspace_bytes(ctypes.byref(self.c), int(k_max)))

    def new_workspace(self, k_max: int = 1) -> torch.Tensor:
        n = self.workspace_bytes(k_max)
        if n == 0:
            raise MageError(-1, "mage_workspace_bytes")
        return torch.empty(n, dtype=torch.uint8, device=self.device)


def mage_exact_select(kv: KVCache, q, k_blk, v_blk, sm_scale: float, out, scores, workspace, dev_status=None, stream=None,
                      events=None):
    """Step 1 of a block: exact attention into ``out`` and block scores into ``scores`` (see mage.h).

    ``events``: optional list of four recorded-on-demand ``torch.cuda.Event(enable_timing=True)`` objects; when given,
    the call goes through ``mage_exact_select_events`` and the library records them between its kernels.
    """
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    args = (ctypes.byref(kv.c), _ptr(q), _ptr(k_blk), _ptr(v_blk), float(sm_scale), _ptr(out), _ptr(scores), _ptr(workspace),
            ws_bytes, _ptr(dev_status), _stream(stream))
    if events is None:
        rc = load().mage_exact_select(*args)
    else:
        for e in events:                 # torch creates the CUDA event lazily, at its first record
            if not e.cuda_event:
                e.record()
        handles = (ctypes.c_void_p * 4)(*[ctypes.c_void_p(e.cuda_event) for e in events])
        rc = load().mage_exact_select_events(*args, handles)
    if rc != MAGE_OK:
        raise MageError(rc, "mage_exact_select")


def mage_exact_attn(kv: KVCache, q, k_blk, v_blk, sm_scale: float, out, workspace, dev_status=None, stream=None):
    """Exact attention of the block without the score pass (the main stream's half of Step 1; see mage.h)."""
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = load().mage_exact_attn(ctypes.byref(kv.c), _ptr(q), _ptr(k_blk), _ptr(v_blk), float(sm_scale), _ptr(out), _ptr(workspace),
                                ws_bytes, _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_exact_attn")


def mage_select_scores(kv: KVCache, q, sm_scale: float, scores, workspace, dev_status=None, stream=None):
    """Block scores from the queries and the cached keys alone (the select stream's own computation; see mage.h)."""
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = load().mage_select_scores(ctypes.byref(kv.c), _ptr(q), float(sm_scale), _ptr(scores), _ptr(workspace), ws_bytes,
                                   _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_select_scores")


STATIC_SCRATCH_BYTES = 32 << 20


def mage_exact_select_static(kv: KVCache, q, k_blk, v_blk, sm_scale: float, out, scores, dev_status=None, stream=None):
    """Step 1 without a caller workspace: the scratch is a fixed array inside the library (see mage.h).

    For hosts that may not allocate device memory when they call.  Descriptions that need more than
    STATIC_SCRATCH_BYTES are refused with MAGE_ERR_WORKSPACE.  Calls on one device share the scratch, so
    calls that could overlap on the GPU must be ordered by the caller.
    """
    rc = load().mage_exact_select_static(ctypes.byref(kv.c), _ptr(q), _ptr(k_blk), _ptr(v_blk), float(sm_scale), _ptr(out),
                                         _ptr(scores), _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_exact_select_static")


def mage_topk(scores, seq_lens, P: int, H_kv: int, N_max: int, k: int, indices, k_eff, stream=None):
    """Per-KV-head Top-k of ``scores`` into ``indices`` / ``k_eff`` (see mage.h)."""
    rc = load().mage_topk(_ptr(scores), _ptr(seq_lens), P, H_kv, N_max, k, _ptr(indices), _ptr(k_eff), None, 0, _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_topk")


def mage_sparse_block_attn(kv: KVCache, q, k_blk, v_blk, indices, k_eff, k: int, sm_scale: float, out, workspace=None,
                           dev_status=None, stream=None):
    """Reuse step: attention over the selected cache rows plus the block's own keys (see mage.h)."""
    rc = load().mage_sparse_block_attn(ctypes.byref(kv.c), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(indices), _ptr(k_eff), int(k),
                                       float(sm_scale), _ptr(out), _ptr(workspace),
                                       workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                       _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_sparse_block_attn")


class K8Keys:
    """The keys of a cache as e4m3 codes (``mage_k8_t``): ``codes`` is a uint8 tensor shaped and strided like ``kv.k``,
    ``k_scale`` is [P, H_kv] fp32, ``scratch`` the per-call buffer.  ``quantize`` fills codes (and, from row 0, the scales)."""

    def __init__(self, kv: KVCache):
        self.kv = kv
        self.codes = torch.empty_strided(kv.k.shape, kv.k.stride(), dtype=torch.uint8, device=kv.device)
        self.k_scale = torch.empty(kv.P, kv.H_kv, dtype=torch.float32, device=kv.device)
        n = int(load().mage_k8_scratch_bytes(ctypes.byref(kv.c)))
        if n == 0:
            raise MageError(-1, "mage_k8_scratch_bytes")
        self.scratch = torch.empty(n, dtype=torch.uint8, device=kv.device)
        self.c = mage_k8_t(self.codes.data_ptr(), self.k_scale.data_ptr(), self.scratch.data_ptr())

    def quantize(self, row_begin: int = 0, dev_status=None, stream=None):
        rc = load().mage_k8_quantize_cache(ctypes.byref(self.kv.c), int(row_begin), _ptr(self.codes), _ptr(self.k_scale), _ptr(dev_status),
                                           _stream(stream))
        if rc != MAGE_OK:
            raise MageError(rc, "mage_k8_quantize_cache")
        return self


def mage_exact_select_k8(kv: KVCache, k8: K8Keys, q, k_blk, v_blk, sm_scale: float, out, scores, workspace, dev_status=None, stream=None,
                         events=None):
    """mage_exact_select with the keys (and queries) in 8 bits (see mage.h); ``events`` as in ``mage_exact_select``."""
    args = (ctypes.byref(kv.c), ctypes.byref(k8.c), _ptr(q), _ptr(k_blk), _ptr(v_blk), float(sm_scale), _ptr(out), _ptr(scores),
            _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream))
    if events is None:
        rc = load().mage_exact_select_k8(*args)
    else:
        for e in events:
            if not e.cuda_event:
                e.record()
        handles = (ctypes.c_void_p * 4)(*[ctypes.c_void_p(e.cuda_event) for e in events])
        rc = load().mage_exact_select_k8_events(*args, handles)
    if rc != MAGE_OK:
        raise MageError(rc, "mage_exact_select_k8")


def mage_sparse_block_attn_k8(kv: KVCache, k8: K8Keys, q, k_blk, v_blk, indices, k_eff, k: int, sm_scale: float, out, workspace=None,
                              dev_status=None, stream=None):
    """mage_sparse_block_attn with the keys (and queries) in 8 bits (see mage.h)."""
    rc = load().mage_sparse_block_attn_k8(ctypes.byref(kv.c), ctypes.byref(k8.c), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(indices),
                                          _ptr(k_eff), int(k), float(sm_scale), _ptr(out), _ptr(workspace),
                                          workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                          _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_sparse_block_attn_k8")


def mage_append_block(kv: KVCache, k_blk, v_blk, seq_lens, dev_status=None, stream=None):
    """End of a block: append the block's final K/V to the cache and add B to ``seq_lens`` (see mage.h)."""
    rc = load().mage_append_block(ctypes.byref(kv.c), _ptr(k_blk), _ptr(v_blk), _ptr(seq_lens), _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_append_block")


QUEST_PAGE = 16


def mage_quest_build(kv: KVCache, page_min, page_max, dev_status=None, stream=None):
    """Quest-style page summaries (per-channel min / max of each whole 16-token page of the prefix; see mage.h)."""
    rc = load().mage_quest_build(ctypes.byref(kv.c), _ptr(page_min), _ptr(page_max), _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_quest_build")


def mage_quest_select(kv: KVCache, q, page_min, page_max, k: int, page_scores, indices, k_eff, workspace, stream=None):
    """Per-block Quest-style selection: page scores, the k/16 best pages, their tokens as an index set (see mage.h)."""
    rc = load().mage_quest_select(ctypes.byref(kv.c), _ptr(q), _ptr(page_min), _ptr(page_max), int(k), _ptr(page_scores), _ptr(indices),
                                  _ptr(k_eff), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_quest_select")


def quest_workspace(kv: KVCache, k: int) -> torch.Tensor:
    n = int(load().mage_quest_workspace_bytes(ctypes.byref(kv.c), int(k)))
    if n == 0:
        raise MageError(-1, "mage_quest_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=kv.device)


def pruned_workspace(kv: KVCache, k: int) -> torch.Tensor:
    n = int(load().mage_pruned_workspace_bytes(ctypes.byref(kv.c), int(k)))
    if n == 0:
        raise MageError(-1, "mage_pruned_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=kv.device)


def mage_exact_select_pruned(kv: KVCache, q, k_blk, v_blk, sm_scale: float, k: int, out, scores, indices, k_eff, workspace,
                             tiles_scored=None, dense_above: float = 0.5, dev_status=None, stream=None):
    """Step 1 + selection with the score pass restricted to the key tiles that can hold a selected key (see mage.h)."""
    rc = load().mage_exact_select_pruned(ctypes.byref(kv.c), _ptr(q), _ptr(k_blk), _ptr(v_blk), float(sm_scale), int(k), float(dense_above),
                                         _ptr(out), _ptr(scores), _ptr(indices), _ptr(k_eff), _ptr(tiles_scored), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream))
    if rc != MAGE_OK:
        raise MageError(rc, "mage_exact_select_pruned")


# ------------------------------------------------------------------------------------------ packed chunks of new tokens
def _require(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _tokens(t: torch.Tensor, shape, device, name: str):
    """Strides of a packed token tensor [n, heads, 128] bf16 (the head dimension contiguous) on ``device``."""
    st = t.stride()
    if t.dtype is not torch.bfloat16 or t.shape != shape or st[2] != 1 or t.device != device:
        raise ValueError(f"{name}: expected bf16 {shape} with a contiguous head dimension on {device}, got {t.dtype} {tuple(t.shape)} strides {st} on {t.device}")
    return st


def _enqueue(where: str, device, stream, call, *args):
    """Call into the library on ``stream`` (default: the current stream of the tensors' device) with that device current."""
    current = torch.cuda.current_device()
    index = device.index if device.index is not None else current
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(index)
    else:
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if current == index:
        rc = call(*args, handle)
    else:
        with torch.cuda.device(index):
            rc = call(*args, handle)
    if rc != MAGE_OK:
        raise MageError(rc, where)


class _CodedCache:
    """What the caches in 8 and 4 bits have in common: arrays of codes and scales, checked, and the two descriptions of them."""

    def _describe(self, struct, per, codes, scales, H_q, seq_lens, block_table, N_max, B):     # per: elements of a code byte
        k, v = codes
        c, dev = mage_kv_t(), k.device
        if block_table is None:
            P, H_kv, n = k.shape[:3]
            _require(N_max is None or N_max == n, "N_max of a contiguous 8- or 4-bit cache is its row count (the scales' row stride)")
            c.stride_p, c.stride_h, c.stride_n, c.N_max = k.stride(0) * per, k.stride(1) * per, k.stride(2) * per, n
        else:
            _require(k.is_contiguous() and v.is_contiguous() and N_max is not None, "paged: contiguous pools, N_max given")
            _require(block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.is_contiguous() and block_table.device == dev, "block_table: contiguous int32 [P, max_pages]")
            (num_pages, H_kv, page), P = k.shape[:3], block_table.shape[0]
            c.page_size, c.num_pages, c.max_pages, c.block_table, c.N_max = page, num_pages, block_table.shape[1], block_table.data_ptr(), N_max
        c.P, c.H_q, c.H_kv, c.d, c.B = P, H_q, H_kv, k.shape[3] * per, B
        if seq_lens is not None:
            _require(seq_lens.dtype == torch.int32 and seq_lens.numel() == P and seq_lens.is_contiguous() and seq_lens.device == dev, "seq_lens: int32 [P]")
            c.seq_lens = seq_lens.data_ptr()
        self.k_scale, self.v_scale, self.seq_lens, self.block_table = scales[0], scales[1], seq_lens, block_table
        self.c, self.at = c, ctypes.addressof(c)
        self.c_codes = struct(k.data_ptr(), v.data_ptr(), scales[0].data_ptr(), scales[1].data_ptr())
        self.at_codes = ctypes.addressof(self.c_codes)
        self.P, self.H_q, self.H_kv, self.d, self.B, self.N_max, self.device = P, H_q, H_kv, int(c.d), B, int(c.N_max), dev


def _rows_like(kv: KVCache) -> tuple:
    """Pages or problems, heads and rows of a coded cache for what a 16-bit one holds (contiguous tensors may have more rows than are used)."""
    return tuple(kv.k.shape[:2]) + (kv.N_max if kv.block_table is None else kv.k.shape[2],)


class Kv8Cache(_CodedCache):
    """A cache held in 8 bits (``mage_kv8_t`` with its ``mage_kv_t``): e4m3 codes as uint8 and one fp32 scale per row.

    Contiguous: ``k8``, ``v8`` are [P, H_kv, N_max, 128] uint8 views and ``k_scale``, ``v_scale`` [P, H_kv, N_max] fp32, contiguous.
    Paged: pools [num_pages, H_kv, page_size, 128] and [num_pages, H_kv, page_size], ``block_table`` [P, max_pages] int32.
    The object keeps references and owns no memory; ``Kv8Cache.like`` allocates.
    """

    def __init__(self, k8: torch.Tensor, v8: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, H_q: int,
                 seq_lens: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None, N_max: Optional[int] = None, B: int = 1):
        _require(k8.dtype == torch.uint8 and v8.dtype == torch.uint8 and k8.dim() == 4 and k8.shape == v8.shape and k8.stride() == v8.stride() and k8.stride(3) == 1,
                 "k8, v8: uint8, four dimensions, the same shape and strides, the head dimension contiguous")
        for s in (k_scale, v_scale):
            _require(s.dtype == torch.float32 and tuple(s.shape) == tuple(k8.shape[:3]) and s.is_contiguous() and s.device == k8.device,
                     "k_scale, v_scale: contiguous fp32 of the codes' first three dimensions on their device")
        _require(v8.device == k8.device, "k8, v8: one device")
        self.k8, self.v8 = k8, v8
        self._describe(mage_kv8_t, 1, (k8, v8), (k_scale, v_scale), H_q, seq_lens, block_table, N_max, B)
        self.c8, self.at8 = self.c_codes, self.at_codes

    @classmethod
    def like(cls, kv: KVCache) -> "Kv8Cache":
        """An empty 8-bit cache of the shape, page table and lengths of a 16-bit one."""
        rows, dev = _rows_like(kv), kv.device
        codes = rows + (kv.d,)
        return cls(torch.zeros(codes, dtype=torch.uint8, device=dev), torch.zeros(codes, dtype=torch.uint8, device=dev), torch.zeros(rows, device=dev),
                   torch.zeros(rows, device=dev), kv.H_q, seq_lens=kv.seq_lens, block_table=kv.block_table, N_max=kv.N_max if kv.block_table is not None else None, B=kv.B)


class Kv4Cache(_CodedCache):
    """A cache held in 4 bits (``mage_kv4_t`` with its ``mage_kv_t``): two codes a byte and a scale byte for each 16 elements.

    Contiguous: ``k4``, ``v4`` are [P, H_kv, N_max, 64] uint8 views and ``k_scale``, ``v_scale`` [P, H_kv, N_max, 8] uint8, contiguous.
    Paged: pools [num_pages, H_kv, page_size, 64] and [num_pages, H_kv, page_size, 8], ``block_table`` [P, max_pages] int32.
    The object keeps references and owns no memory; ``Kv4Cache.like`` allocates.
    """

    def __init__(self, k4: torch.Tensor, v4: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, H_q: int,
                 seq_lens: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None, N_max: Optional[int] = None, B: int = 1):
        _require(k4.dtype == torch.uint8 and v4.dtype == torch.uint8 and k4.dim() == 4 and k4.shape == v4.shape and k4.stride() == v4.stride() and k4.stride(3) == 1,
                 "k4, v4: uint8, four dimensions, the same shape and strides, the head dimension contiguous")
        for s in (k_scale, v_scale):
            _require(s.dtype == torch.uint8 and tuple(s.shape) == tuple(k4.shape[:3]) + (8,) and s.is_contiguous() and s.device == k4.device,
                     "k_scale, v_scale: contiguous uint8 of the codes' first three dimensions and 8 on their device")
        _require(v4.device == k4.device, "k4, v4: one device")
        self.k4, self.v4 = k4, v4
        self._describe(mage_kv4_t, 2, (k4, v4), (k_scale, v_scale), H_q, seq_lens, block_table, N_max, B)

    @classmethod
    def like(cls, kv: KVCache) -> "Kv4Cache":
        """An empty 4-bit cache of the shape, page table and lengths of a 16-bit one."""
        rows, dev = _rows_like(kv), kv.device
        mk = lambda n: torch.zeros(rows + (n,), dtype=torch.uint8, device=dev)
        return cls(mk(64), mk(64), mk(8), mk(8), kv.H_q, seq_lens=kv.seq_lens, block_table=kv.block_table, N_max=kv.N_max if kv.block_table is not None else None, B=kv.B)


class ChunkBatch:
    """New tokens of a batch, packed (``mage_chunk_t``): problem p owns rows q_start[p] .. q_start[p+1]-1 of the token tensors, and
    the cache's ``seq_lens`` count them already.  ``max_len``: most new tokens of any problem (default: ``n_tokens``)."""

    def __init__(self, kv, q_start: torch.Tensor, n_tokens: int, max_len: Optional[int] = None):
        _require(q_start.dtype == torch.int32 and q_start.dim() == 1 and q_start.numel() == kv.P + 1 and q_start.is_contiguous() and q_start.device == kv.device,
                 f"q_start: contiguous int32 [{kv.P + 1}] on {kv.device}")
        self.kv, self.q_start, self.n_tokens = kv, q_start, int(n_tokens)
        self.max_len = self.n_tokens if max_len is None else int(max_len)
        _require(0 <= self.max_len <= self.n_tokens, "0 <= max_len <= n_tokens")
        self.c = mage_chunk_t(q_start.data_ptr(), self.n_tokens, self.max_len)
        self.at = ctypes.addressof(self.c)
        self.q_shape, self.kv_shape, self.lse_shape = (self.n_tokens, kv.H_q, 128), (self.n_tokens, kv.H_kv, 128), (self.n_tokens, kv.H_q)

    def workspace_bytes(self) -> int:
        """What attention over the cache that the chunk was made for makes use of (over 4 bits up to 1 GiB more for prompts, which may be left out: see mage.h)."""
        lib = load()
        return int((lib.mage_chunk_workspace_bytes_kv4 if isinstance(self.kv, Kv4Cache) else lib.mage_chunk_workspace_bytes)(self.kv.at, self.at))

    def new_workspace(self) -> torch.Tensor:
        n = self.workspace_bytes()
        if n == 0:
            raise MageError(-1, "mage_chunk_workspace_bytes")
        return torch.empty(n, dtype=torch.uint8, device=self.kv.device)


def _same_batch(kv, chunk: ChunkBatch):
    """``chunk`` was made for ``kv``, or for a cache of the same batch (a 16-bit and an 8-bit one, another layer's)."""
    o = chunk.kv
    if o is not kv and (o.P != kv.P or o.H_q != kv.H_q or o.H_kv != kv.H_kv or o.device != kv.device):
        raise ValueError("chunk: made for a cache of another batch, other heads or another device")


def _opt(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _codes(kv, kind) -> tuple:
    """The description of a coded cache's arrays, which have the sizes that a call over ``kind`` addresses only in that class."""
    if not isinstance(kv, kind):
        raise ValueError(f"cache: expected a {kind.__name__}, got a {type(kv).__name__}")
    return (kv.at_codes,)


def _append(where, kv, chunk, codes, call, k_new, v_new, dev_status, stream):
    _same_batch(kv, chunk)
    st = _tokens(k_new, chunk.kv_shape, kv.device, "k_new")
    if _tokens(v_new, chunk.kv_shape, kv.device, "v_new") != st:
        raise ValueError("k_new, v_new: the same strides")
    _enqueue(where, kv.device, stream, call, kv.at, *codes, chunk.at, k_new.data_ptr(), v_new.data_ptr(), st[0], st[1], _opt(dev_status))


def mage_append_chunk(kv: KVCache, chunk: ChunkBatch, k_new, v_new, dev_status=None, stream=None):
    """Write the new tokens' keys and values [n_tokens, H_kv, 128] to the cache (see mage.h)."""
    _append("mage_append_chunk", kv, chunk, (), load().mage_append_chunk, k_new, v_new, dev_status, stream)


def mage_append_chunk_kv8(kv8: Kv8Cache, chunk: ChunkBatch, k_new, v_new, dev_status=None, stream=None):
    """The same into an 8-bit cache, quantised on the way: one scale per row (see mage.h)."""
    _append("mage_append_chunk_kv8", kv8, chunk, _codes(kv8, Kv8Cache), load().mage_append_chunk_kv8, k_new, v_new, dev_status, stream)


def mage_append_chunk_kv4(kv4: Kv4Cache, chunk: ChunkBatch, k_new, v_new, dev_status=None, stream=None):
    """The same into a 4-bit cache: a scale for each 16 elements of a row (see mage.h)."""
    _append("mage_append_chunk_kv4", kv4, chunk, _codes(kv4, Kv4Cache), load().mage_append_chunk_kv4, k_new, v_new, dev_status, stream)


def _read_rows(where, kv, codes, call, k_out, v_out, indices, k_eff, row_begin, dev_status, stream):
    dev, n_rows = kv.device, k_out.shape[2] if k_out.dim() == 4 else -1
    shape = (kv.P, kv.H_kv, n_rows, 128)
    for o in (k_out, v_out):
        if o.dtype is not torch.bfloat16 or o.shape != shape or not o.is_contiguous() or o.device != dev:
            raise ValueError(f"k_out, v_out: contiguous bf16 [{kv.P}, {kv.H_kv}, n_rows, 128] on {dev}")
    if indices is not None:
        if (indices.dtype is not torch.int32 or indices.shape != shape[:3] or not indices.is_contiguous() or indices.device != dev or k_eff is None
                or k_eff.dtype is not torch.int32 or k_eff.numel() != kv.P or not k_eff.is_contiguous() or k_eff.device != dev):
            raise ValueError("indices: contiguous int32 [P, H_kv, n_rows], k_eff: int32 [P]")
    _enqueue(where, dev, stream, call, kv.at, *codes, _opt(indices), _opt(k_eff), row_begin, n_rows, k_out.data_ptr(), v_out.data_ptr(), _opt(dev_status))


def mage_kv8_read(kv8: Kv8Cache, k_out, v_out, indices=None, k_eff=None, row_begin: int = 0, dev_status=None, stream=None):
    """Rows of an 8-bit cache back as bf16 into ``k_out``, ``v_out`` [P, H_kv, n_rows, 128]: rows from ``row_begin`` on, or the
    selected ones (``indices`` [P, H_kv, n_rows], ``k_eff`` [P], as mage_topk writes them; see mage.h)."""
    _read_rows("mage_kv8_read", kv8, _codes(kv8, Kv8Cache), load().mage_kv8_read, k_out, v_out, indices, k_eff, row_begin, dev_status, stream)


def mage_kv4_read(kv4: Kv4Cache, k_out, v_out, indices=None, k_eff=None, row_begin: int = 0, dev_status=None, stream=None):
    """``mage_kv8_read`` of a 4-bit cache; exact (see mage.h)."""
    _read_rows("mage_kv4_read", kv4, _codes(kv4, Kv4Cache), load().mage_kv4_read, k_out, v_out, indices, k_eff, row_begin, dev_status, stream)


def _chunk_attn(where, kv, chunk, codes, call, q, sm_scale, out, workspace, mask_block, lse, dev_status, stream):
    _same_batch(kv, chunk)
    dev = kv.device
    st = _tokens(q, chunk.q_shape, dev, "q")
    _tokens(out, chunk.q_shape, dev, "out")
    if not out.is_contiguous() or workspace.device != dev or not workspace.is_contiguous():
        raise ValueError("out, workspace: contiguous, on the cache's device")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != chunk.lse_shape or not lse.is_contiguous() or lse.device != dev):
        raise ValueError(f"lse: contiguous fp32 {chunk.lse_shape}")
    _enqueue(where, dev, stream, call, kv.at, *codes, chunk.at, q.data_ptr(), st[0], st[1], mask_block, sm_scale, out.data_ptr(), _opt(lse), workspace.data_ptr(),
             workspace.nbytes, _opt(dev_status))


def mage_chunk_attn(kv: KVCache, chunk: ChunkBatch, q, sm_scale: float, out, workspace, mask_block: int = 1, lse=None, dev_status=None, stream=None):
    """Attention of the new tokens ``q`` [n_tokens, H_q, 128] over the cache that holds their keys and values already, into ``out``
    of the same shape; ``mask_block`` 0: open, 1: causal, b: causal between blocks of b tokens (see mage.h)."""
    _chunk_attn("mage_chunk_attn", kv, chunk, (), load().mage_chunk_attn, q, sm_scale, out, workspace, mask_block, lse, dev_status, stream)


def mage_chunk_attn_kv8(kv8: Kv8Cache, chunk: ChunkBatch, q, sm_scale: float, out, workspace, mask_block: int = 1, lse=None, dev_status=None, stream=None):
    """``mage_chunk_attn`` over an 8-bit cache (see mage.h)."""
    _chunk_attn("mage_chunk_attn_kv8", kv8, chunk, _codes(kv8, Kv8Cache), load().mage_chunk_attn_kv8, q, sm_scale, out, workspace, mask_block, lse, dev_status, stream)


def mage_chunk_attn_kv4(kv4: Kv4Cache, chunk: ChunkBatch, q, sm_scale: float, out, workspace, mask_block: int = 1, lse=None, dev_status=None, stream=None):
    """``mage_chunk_attn`` over a 4-bit cache (see mage.h)."""
    _chunk_attn("mage_chunk_attn_kv4", kv4, chunk, _codes(kv4, Kv4Cache), load().mage_chunk_attn_kv4, q, sm_scale, out, workspace, mask_block, lse, dev_status, stream)


class Rope:
    """Rotary positions (``mage_rope_t`` without the tokens): ``inv_freq`` [rot_dim / 2] fp32 on the device, the axis of each pair
    (default: one axis), pairs (i, i + rot_dim/2) with ``halves``, else (2i, 2i+1)."""

    def __init__(self, inv_freq: torch.Tensor, axis_of_pair=None, rot_dim: int = 128, halves: bool = True, mult: float = 1.0):
        pairs = rot_dim // 2
        _require(inv_freq.dtype == torch.float32 and inv_freq.numel() == pairs and inv_freq.is_contiguous(), f"inv_freq: contiguous fp32 [{pairs}]")
        axes = [0] * pairs if axis_of_pair is None else [int(a) for a in axis_of_pair]
        _require(len(axes) == pairs and pairs <= 64 and min(axes, default=0) >= 0 and max(axes, default=0) < 4, "axis_of_pair: one axis below 4 for each pair")
        self.inv_freq, self.n_axes = inv_freq, max(axes, default=0) + 1
        self.c = mage_rope_t(d=128, rot_dim=rot_dim, halves=int(halves), n_axes=self.n_axes, mult=mult, inv_freq=inv_freq.data_ptr())
        self.c.axis_of_pair[:pairs] = axes
        self.at = ctypes.addressof(self.c)


def mage_rope(rope: Rope, positions, q, k=None, q_out=None, k_out=None, stream=None):
    """Rotate packed ``q`` [n, H_q, 128] and ``k`` [n, H_kv, 128] (or None) by ``positions`` [n_axes, n] (or [n]) int32; the outputs
    default to the inputs themselves (see mage.h)."""
    dev, shape = q.device, q.shape
    n = shape[0]
    qs = _tokens(q, shape if len(shape) == 3 and shape[2] == 128 else (n, "H_q", 128), dev, "q")
    qo, qos = (q, qs) if q_out is None else (q_out, _tokens(q_out, shape, dev, "q_out"))
    if k is None:
        keys = (0, None, 0, 0, None, 0, 0)
    else:
        k_shape = (n, k.shape[1], 128)
        ks = _tokens(k, k_shape, dev, "k")
        ko, kos = (k, ks) if k_out is None else (k_out, _tokens(k_out, k_shape, dev, "k_out"))
        keys = (k_shape[1], k.data_ptr(), ks[0], ks[1], ko.data_ptr(), kos[0], kos[1])
    pos_stride = _positions(rope, positions, n, dev)
    _enqueue("mage_rope", dev, stream, load().mage_rope, rope.at, n, positions.data_ptr(), pos_stride, shape[1], q.data_ptr(), qs[0], qs[1],
             qo.data_ptr(), qos[0], qos[1], *keys)


def _positions(rope: Rope, positions, n: int, dev) -> int:
    """Checks ``positions`` [n_axes, n] (or [n]) int32 of ``n`` tokens; the stride of its axes."""
    one = positions.dim() == 1
    if (positions.dtype is not torch.int32 or positions.shape[-1] != n or positions.stride(-1) != 1 and n > 1 or positions.device != dev
            or (rope.n_axes != 1 if one else positions.shape[0] < rope.n_axes)):
        raise ValueError(f"positions: int32 [{rope.n_axes}, {n}], tokens contiguous, on {dev}")
    if rope.inv_freq.device != dev:
        raise ValueError("inv_freq: on the queries' device")
    return n if one else positions.stride(0)


def _rope_append(where, kv, chunk, codes, call, rope, positions, q, k_new, v_new, q_out, dev_status, stream):
    _same_batch(kv, chunk)
    dev = kv.device
    qs, ks = _tokens(q, chunk.q_shape, dev, "q"), _tokens(k_new, chunk.kv_shape, dev, "k_new")
    if _tokens(v_new, chunk.kv_shape, dev, "v_new") != ks:
        raise ValueError("k_new, v_new: the same strides")
    qo, qos = (q, qs) if q_out is None else (q_out, _tokens(q_out, chunk.q_shape, dev, "q_out"))
    pos_stride = _positions(rope, positions, chunk.n_tokens, dev)
    _enqueue(where, dev, stream, call, kv.at, *codes, chunk.at, rope.at, positions.data_ptr(), pos_stride, q.data_ptr(), qs[0], qs[1], qo.data_ptr(), qos[0], qos[1],
             k_new.data_ptr(), v_new.data_ptr(), ks[0], ks[1], _opt(dev_status))


def mage_rope_append_chunk(kv: KVCache, chunk: ChunkBatch, rope: Rope, positions, q, k_new, v_new, q_out=None, dev_status=None, stream=None):
    """Rotate the new tokens' ``q`` [n_tokens, H_q, 128] (into ``q_out``; default: ``q`` itself) and write their rotated keys and their values
    [n_tokens, H_kv, 128] to the cache, in one kernel; ``positions`` as in ``mage_rope`` (see mage.h)."""
    _rope_append("mage_rope_append_chunk", kv, chunk, (), load().mage_rope_append_chunk, rope, positions, q, k_new, v_new, q_out, dev_status, stream)


def mage_rope_append_chunk_kv8(kv8: Kv8Cache, chunk: ChunkBatch, rope: Rope, positions, q, k_new, v_new, q_out=None, dev_status=None, stream=None):
    """The same into an 8-bit cache (see mage.h)."""
    _rope_append("mage_rope_append_chunk_kv8", kv8, chunk, _codes(kv8, Kv8Cache), load().mage_rope_append_chunk_kv8, rope, positions, q, k_new, v_new, q_out, dev_status, stream)


def mage_rope_append_chunk_kv4(kv4: Kv4Cache, chunk: ChunkBatch, rope: Rope, positions, q, k_new, v_new, q_out=None, dev_status=None, stream=None):
    """The same into a 4-bit cache (see mage.h)."""
    _rope_append("mage_rope_append_chunk_kv4", kv4, chunk, _codes(kv4, Kv4Cache), load().mage_rope_append_chunk_kv4, rope, positions, q, k_new, v_new, q_out, dev_status, stream)
