"""Thin ctypes binding of liba3.so: same entry-point names as include/a3.h, argument
marshalling only.  torch is used for device memory and for the current HIP stream; every
step of the path runs in the library's kernels.  There is no fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liba3.so")

A3_OK, A3_ERR_INVALID_ARG, A3_ERR_UNSUPPORTED, A3_ERR_WORKSPACE, A3_ERR_HIP, A3_ERR_IO = 0, -1, -2, -3, -4, -5
A3_F32, A3_BF16 = 0, 1
A3_ROPE_INTERLEAVED, A3_ROPE_HALF = 0, 1
A3_POOL_MAX, A3_POOL_AVG = 0, 1
A3_PAGES_PLAIN, A3_PAGES_Q8 = 0, 1

EXPORTS = ["a3_workspace_bytes", "a3_layout_prepare", "a3_rope_realign", "a3_question_scores", "a3_question_scores_noalloc", "a3_realign_scores", "a3_topk_select", "a3_topk_select_plan",
           "a3_selected_qkv_proj", "a3_selected_qkv_proj_scatter", "a3_kv_scatter", "a3_fused_attention", "a3_attention_plan", "a3_fused_attention_planned", "a3_fused_attention_planned_events", "a3_active_rows",
           "a3_block_tail_ws_bytes", "a3_block_tail", "a3_rms_norm", "a3_question_scores_causal", "a3_window_votes",
           "a3_evict_ws_bytes", "a3_evict_select", "a3_evict_compact", "a3_value_deviation_scores",
           "a3_select_chunk_edges", "a3_chunk_cache_load", "a3_rope_realign_q8", "a3_q8_row_bytes", "a3_quantize_q8",
           "a3_chunk_cache_load_q8", "a3_chunk_file_read", "a3_page_bytes", "a3_pages_prepare", "a3_paged_append",
           "a3_paged_attention_ws_bytes", "a3_paged_attention", "a3_lm_head", "a3_token_logprobs_ws_bytes", "a3_token_logprobs",
           "a3_tree_attention_ws_bytes", "a3_tree_attention", "a3_tree_accept_ws_bytes", "a3_tree_accept", "a3_paged_move",
           "a3_beam_select_ws_bytes", "a3_beam_select",
           "a3_set_tuning", "a3_recompute_count", "a3_chunk_edge_sel_start", "a3_strerror", "a3_last_error", "a3_version"]


class A3Error(RuntimeError):
    def __init__(self, status: int, where: str, text: str):
        super().__init__(f"{where}: status {status}: {text}")
        self.status = status


class a3_layout(C.Structure):
    _fields_ = [
        ("dtype", C.c_int), ("n_q_heads", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int),
        ("hidden", C.c_int), ("rope_layout", C.c_int), ("rope_base", C.c_double), ("sm_scale", C.c_float),
        ("n_req", C.c_int), ("n_chunks", C.c_int), ("total_tokens", C.c_int), ("max_ctx_len", C.c_int),
        ("max_q_len", C.c_int),
        ("seg_start", C.c_void_p), ("ctx_len", C.c_void_p), ("q_len", C.c_void_p),
        ("chunk_start", C.c_void_p), ("chunk_len", C.c_void_p), ("chunk_delta", C.c_void_p),
        ("tok_pos", C.c_void_p), ("tok_req", C.c_void_p), ("tok_chunk", C.c_void_p), ("q_start", C.c_void_p),
        ("rope_chunk_cs", C.c_void_p), ("rope_pos_cs", C.c_void_p),
    ]


class a3_block_weights(C.Structure):
    _fields_ = [("wo", C.c_void_p), ("g_post", C.c_void_p), ("w_gate", C.c_void_p), ("w_up", C.c_void_p),
                ("w_down", C.c_void_p), ("g_next", C.c_void_p), ("ffn", C.c_int), ("eps", C.c_float)]


class a3_pages(C.Structure):
    _fields_ = [
        ("dtype", C.c_int), ("format", C.c_int), ("n_q_heads", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int),
        ("rope_layout", C.c_int), ("rope_base", C.c_double), ("sm_scale", C.c_float), ("page_size", C.c_int),
        ("n_pages", C.c_int), ("n_req", C.c_int), ("max_pages", C.c_int), ("n_pos", C.c_int),
        ("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("page_table", C.c_void_p), ("rope_cs", C.c_void_p),
    ]


_lib = None


def lib() -> C.CDLL:
    """Loads liba3.so (built beforehand by ``python -m paper_2511_17560_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2511_17560_amd.build` "
                           "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    P, I, V = C.POINTER(a3_layout), C.c_int, C.c_void_p
    L.a3_workspace_bytes.restype = C.c_size_t
    L.a3_workspace_bytes.argtypes = [P, I]
    L.a3_layout_prepare.argtypes = [P, V]
    L.a3_rope_realign.argtypes = [P, V, V, V]
    L.a3_question_scores.argtypes = [P, V, V, V, V, C.c_size_t, V]
    L.a3_realign_scores.argtypes = [P, V, V, V, V, V, C.c_size_t, V]
    L.a3_question_scores_noalloc.argtypes = [P, V, V, V, V]
    L.a3_question_scores_noalloc.restype = I
    L.a3_topk_select.argtypes = [P, V, V, I, V, V, C.c_size_t, V]
    L.a3_selected_qkv_proj.argtypes = [P, V, V, I, V, V, V, V, V, V, V, V, V, V]
    L.a3_selected_qkv_proj_scatter.argtypes = [P, V, V, I, V, V, V, V, V, V, V, V, V, V]
    L.a3_kv_scatter.argtypes = [P, V, V, V, I, V, V, V]
    L.a3_fused_attention.argtypes = [P, V, V, I, V, V, V, V, C.c_size_t, V]
    L.a3_active_rows.argtypes = [P, V, V, I, V, V]
    L.a3_attention_plan.argtypes = [P, V, I, V, C.c_size_t, V]
    L.a3_fused_attention_planned.argtypes = [P, V, V, I, V, V, V, V, C.c_size_t, V]
    L.a3_fused_attention_planned_events.argtypes = [P, V, V, I, V, V, V, V, C.c_size_t, V, V, V]
    L.a3_fused_attention_planned_events.restype = I
    L.a3_attention_plan.restype = I
    L.a3_fused_attention_planned.restype = I
    L.a3_block_tail_ws_bytes.restype = C.c_size_t
    L.a3_block_tail_ws_bytes.argtypes = [P, I, I]
    L.a3_block_tail.argtypes = [P, V, V, I, C.POINTER(a3_block_weights), V, V, V, C.c_size_t, V]
    L.a3_rms_norm.argtypes = [P, V, V, I, V, C.c_float, V, V]
    L.a3_block_tail.restype = I
    L.a3_question_scores_causal.argtypes = [P, V, V, V, V, C.c_size_t, V]
    L.a3_window_votes.argtypes = [P, V, V, V, V, C.c_size_t, V]
    L.a3_evict_ws_bytes.restype = C.c_size_t
    L.a3_evict_ws_bytes.argtypes = [P]
    L.a3_evict_select.argtypes = [P, V, V, V, I, I, I, V, V, C.c_size_t, V]
    L.a3_evict_compact.argtypes = [P, V, V, V, I, V, V, V]
    L.a3_value_deviation_scores.argtypes = [P, V, V, V, V]
    L.a3_select_chunk_edges.argtypes = [P, I, I, V, I, V, V]
    L.a3_value_deviation_scores.restype = I
    L.a3_chunk_cache_load.argtypes = [P, C.POINTER(C.c_int), C.POINTER(C.c_int), I, C.POINTER(C.c_void_p),
                                      C.POINTER(C.c_void_p), V, V, V]
    L.a3_chunk_cache_load.restype = I
    L.a3_chunk_file_read.argtypes = [I, C.POINTER(C.c_int), C.POINTER(C.c_longlong), C.POINTER(C.c_size_t),
                                     C.POINTER(C.c_void_p), I]
    L.a3_chunk_file_read.restype = I
    L.a3_q8_row_bytes.argtypes = [P]
    L.a3_q8_row_bytes.restype = C.c_size_t
    L.a3_quantize_q8.argtypes = [P, V, V, V, V]
    L.a3_rope_realign_q8.argtypes = [P, V, V, V, V]
    L.a3_chunk_cache_load_q8.argtypes = [P, C.POINTER(C.c_int), C.POINTER(C.c_int), I, C.POINTER(C.c_void_p), V, V]
    for name in ("a3_quantize_q8", "a3_rope_realign_q8", "a3_chunk_cache_load_q8"):
        getattr(L, name).restype = I
    L.a3_select_chunk_edges.restype = I
    for name in ("a3_question_scores_causal", "a3_window_votes", "a3_evict_select", "a3_evict_compact"):
        getattr(L, name).restype = I
    L.a3_rms_norm.restype = I
    for name in ("a3_realign_scores", "a3_selected_qkv_proj_scatter", "a3_active_rows", "a3_layout_prepare", "a3_rope_realign", "a3_question_scores", "a3_topk_select",
                 "a3_selected_qkv_proj", "a3_selected_qkv_proj_scatter", "a3_kv_scatter", "a3_fused_attention"):
        getattr(L, name).restype = I
    L.a3_topk_select_plan.argtypes = [P, V, V, I, V, I, V, V, C.c_size_t, V]
    L.a3_topk_select_plan.restype = I
    L.a3_recompute_count.argtypes = [I, I, I]
    L.a3_recompute_count.restype = I
    L.a3_chunk_edge_sel_start.argtypes = [I, C.POINTER(C.c_int), C.POINTER(C.c_int), I, C.POINTER(C.c_int),
                                          C.POINTER(C.c_int), I, I, C.POINTER(C.c_int)]
    L.a3_chunk_edge_sel_start.restype = I
    G = C.POINTER(a3_pages)
    L.a3_page_bytes.argtypes = [G]
    L.a3_page_bytes.restype = C.c_size_t
    L.a3_pages_prepare.argtypes = [G, V]
    L.a3_paged_append.argtypes = [G, V, V, V, V, V, I, V, V, V]
    L.a3_paged_attention_ws_bytes.argtypes = [G, I]
    L.a3_paged_attention_ws_bytes.restype = C.c_size_t
    L.a3_paged_attention.argtypes = [G, V, V, V, I, V, V, C.c_size_t, V]
    L.a3_lm_head.argtypes = [P, V, V, I, V, I, V, C.c_longlong, V]
    L.a3_token_logprobs_ws_bytes.argtypes = [I, I, I]
    L.a3_token_logprobs_ws_bytes.restype = C.c_size_t
    L.a3_token_logprobs.argtypes = [I, V, I, I, C.c_longlong, V, I, I, V, V, V, V, V, C.c_size_t, V]
    L.a3_tree_attention_ws_bytes.argtypes = [G, I, I]
    L.a3_tree_attention_ws_bytes.restype = C.c_size_t
    L.a3_tree_attention.argtypes = [G, V, I, V, V, V, V, I, I, I, V, V, C.c_size_t, V]
    L.a3_tree_accept_ws_bytes.argtypes = [I, I]
    L.a3_tree_accept_ws_bytes.restype = C.c_size_t
    L.a3_tree_accept.argtypes = [I, V, I, C.c_longlong, V, V, V, I, V, V, I, I, I, V, V, V, V, V, V, C.c_size_t, V]
    L.a3_paged_move.argtypes = [G, I, V, V, V, V, V, I, I, I, V]
    L.a3_beam_select_ws_bytes.argtypes = [I, I, I, I]
    L.a3_beam_select_ws_bytes.restype = C.c_size_t
    L.a3_beam_select.argtypes = [I, V, I, I, I, C.c_longlong, V, V, I, I, V, V, V, V, C.c_size_t, V]
    for name in ("a3_pages_prepare", "a3_paged_append", "a3_paged_attention", "a3_lm_head", "a3_token_logprobs", "a3_tree_attention",
                 "a3_tree_accept", "a3_paged_move", "a3_beam_select"):
        getattr(L, name).restype = I
    L.a3_set_tuning.argtypes = [C.c_char_p, I]
    L.a3_set_tuning.restype = I
    L.a3_strerror.restype = C.c_char_p
    L.a3_strerror.argtypes = [I]
    L.a3_last_error.restype = C.c_char_p
    L.a3_version.restype = I
    _lib = L
    return L


def _check(status: int, where: str):
    if status != A3_OK:
        L = lib()
        raise A3Error(status, where, f"{L.a3_strerror(status).decode()}: {L.a3_last_error().decode()}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors must be contiguous"
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:           # the current stream's handle (what torch.cuda.current_stream().cuda_stream is, 2.5 us sooner)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def torch_stream(stream) -> torch.cuda.Stream:
    """The same argument as a torch stream (None: the current one; a raw handle: that stream, 0 the device's default one)."""
    if stream is None:
        return torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = _stream(stream)
    return torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()


def torch_dtype(dtype: str) -> torch.dtype:
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


class Layout:
    """Owns the device index arrays and derived tables of one batch and the a3_layout struct
    that points at them."""

    def __init__(self, *, dtype: str, n_q_heads: int, n_kv_heads: int, head_dim: int, hidden: int,
                 rope_base: float, rope_layout: int, seg_start, ctx_len, q_len, chunk_start, chunk_len,
                 chunk_delta, sm_scale: float = 0.0, device="cuda", prepare: bool = True, stream=None):
        dev = torch.device(device)
        i32 = lambda a: torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=dev)
        self.dtype = dtype
        self.device = dev
        self.seg_start, self.ctx_len, self.q_len = i32(seg_start), i32(ctx_len), i32(q_len)
        self.chunk_start, self.chunk_len, self.chunk_delta = i32(chunk_start), i32(chunk_len), i32(chunk_delta)
        n_req, n_chunks = len(ctx_len), len(chunk_start)
        T = int(np.asarray(seg_start)[-1])
        # what the kernels take for granted about the index arrays (they cannot check device memory): every
        # request is [context | question], the chunks tile the context rows exactly, in ascending order
        seg_h, ctx_h, q_h = (np.asarray(a, dtype=np.int64) for a in (seg_start, ctx_len, q_len))
        if not (len(seg_h) == n_req + 1 and np.array_equal(np.diff(seg_h), ctx_h + q_h) and np.all(ctx_h >= 0)
                and np.all(q_h >= 0)):
            raise ValueError("Layout: seg_start, ctx_len and q_len do not describe [context | question] segments")
        cs_h, cl_h = np.asarray(chunk_start, dtype=np.int64), np.asarray(chunk_len, dtype=np.int64)
        covered = np.zeros(max(T, 1), dtype=np.int32)
        for s0, n in zip(cs_h, cl_h):
            covered[s0:s0 + n] += 1
        want = np.zeros(max(T, 1), dtype=np.int32)
        for r in range(n_req):
            want[seg_h[r]:seg_h[r] + ctx_h[r]] = 1
        if n_chunks and not (np.all(np.diff(cs_h) > 0) and np.array_equal(covered, want)):
            raise ValueError("Layout: the chunks do not tile the context rows exactly")
        max_ctx = int(np.max(ctx_len)) if n_req else 0
        max_q = int(np.max(q_len)) if n_req else 0
        self.total_tokens, self.n_req, self.n_chunks = T, n_req, n_chunks
        self.max_len = int(np.max(ctx_h + q_h)) if n_req else 0     # of one request: context and question
        self.tok_pos = torch.empty(max(T, 1), dtype=torch.int32, device=dev)
        self.tok_req = torch.empty(max(T, 1), dtype=torch.int32, device=dev)
        self.tok_chunk = torch.empty(max(T, 1), dtype=torch.int32, device=dev)
        self.q_start = torch.empty(n_req + 1, dtype=torch.int32, device=dev)
        self.rope_chunk_cs = torch.empty((max(n_chunks, 1), head_dim // 2, 2), dtype=torch.float32, device=dev)
        self.rope_pos_cs = torch.empty((max(max_ctx + max_q, 1), head_dim // 2, 2), dtype=torch.float32, device=dev)
        s = a3_layout()
        s.dtype = {"f32": A3_F32, "bf16": A3_BF16}[dtype]
        s.n_q_heads, s.n_kv_heads, s.head_dim, s.hidden = n_q_heads, n_kv_heads, head_dim, hidden
        s.rope_layout, s.rope_base, s.sm_scale = rope_layout, rope_base, sm_scale
        s.n_req, s.n_chunks, s.total_tokens, s.max_ctx_len, s.max_q_len = n_req, n_chunks, T, max_ctx, max_q
        s.seg_start, s.ctx_len, s.q_len = self.seg_start.data_ptr(), self.ctx_len.data_ptr(), self.q_len.data_ptr()
        if n_chunks:
            s.chunk_start, s.chunk_len = self.chunk_start.data_ptr(), self.chunk_len.data_ptr()
            s.chunk_delta = self.chunk_delta.data_ptr()
        s.tok_pos, s.tok_req, s.tok_chunk = self.tok_pos.data_ptr(), self.tok_req.data_ptr(), self.tok_chunk.data_ptr()
        s.q_start = self.q_start.data_ptr()
        s.rope_chunk_cs, s.rope_pos_cs = self.rope_chunk_cs.data_ptr(), self.rope_pos_cs.data_ptr()
        self.struct = s
        if prepare:
            a3_layout_prepare(self, stream)

    @classmethod
    def from_workload(cls, w, device="cuda", **kw) -> "Layout":
        s = w.shape
        return cls(dtype=s.dtype, n_q_heads=s.n_q_heads, n_kv_heads=s.n_kv_heads, head_dim=s.head_dim,
                   hidden=s.hidden, rope_base=s.rope_base, rope_layout=s.rope_layout, seg_start=w.seg_start,
                   ctx_len=w.ctx_len, q_len=w.q_lens, chunk_start=w.chunk_start, chunk_len=w.chunk_len,
                   chunk_delta=w.chunk_delta, device=device, **kw)

    @classmethod
    def decode(cls, *, n_req: int, **kw) -> "Layout":
        """The layout of one decoding step: one row per request, nothing else.  Every row's position in it is 0, so
        a3_selected_qkv_proj leaves Q and K as projected; a3_paged_append turns them to their positions."""
        return cls(seg_start=np.arange(n_req + 1), ctx_len=np.zeros(n_req), q_len=np.ones(n_req), chunk_start=[], chunk_len=[],
                   chunk_delta=[], rope_layout=kw.pop("rope_layout", A3_ROPE_INTERLEAVED), **kw)

    @property
    def ref(self):
        return C.byref(self.struct)

    def workspace(self, max_active_rows: int) -> torch.Tensor:
        n = a3_workspace_bytes(self, max_active_rows)
        return torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)


class Pages:
    """One layer's paged K/V cache: two pools, the page table and the position table, and the a3_pages struct that points
    at them.  ``page_table`` [n_req, max_pages] int32 is the caller's (written as requests grow); pools are allocated unless
    given.  Pool shapes: [n_pages, Hkv, page_size, d] in the rows' type; 8-bit pages (``q8``): int8 [n_pages, Hkv,
    page_size * (d + 4)], codes and then float scales."""

    def __init__(self, *, dtype: str, n_q_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int,
                 page_table: torch.Tensor, rope_base: float, n_pos: int, rope_layout: int = A3_ROPE_INTERLEAVED, q8: bool = False,
                 sm_scale: float = 0.0, k_pool: Optional[torch.Tensor] = None, v_pool: Optional[torch.Tensor] = None,
                 rope_cs: Optional[torch.Tensor] = None, stream=None):
        dev = page_table.device
        if page_table.dtype != torch.int32 or page_table.dim() != 2:
            raise ValueError("Pages: page_table is an int32 tensor [n_req, max_pages]")
        shape = (n_pages, n_kv_heads, page_size * (head_dim + 4)) if q8 else (n_pages, n_kv_heads, page_size, head_dim)
        dt = torch.int8 if q8 else torch_dtype(dtype)
        self.dtype, self.q8, self.device, self.page_table = dtype, q8, dev, page_table
        self.k_pool, self.v_pool = (torch.empty(shape, dtype=dt, device=dev) if p is None else p for p in (k_pool, v_pool))
        for p in (self.k_pool, self.v_pool):
            if tuple(p.shape) != shape or p.dtype != dt or p.device != dev:
                raise ValueError(f"Pages: a pool is {shape} of {dt} on {dev}, got {tuple(p.shape)} of {p.dtype} on {p.device}")
        fresh = rope_cs is None
        self.own_rope = fresh            # whether rope_cs is what rope_base says, and not a table of the caller's
        self.rope_cs = torch.empty((n_pos, head_dim // 2, 2), dtype=torch.float32, device=dev) if fresh else rope_cs
        if tuple(self.rope_cs.shape) != (n_pos, head_dim // 2, 2) or self.rope_cs.dtype != torch.float32 or self.rope_cs.device != dev:
            raise ValueError(f"Pages: rope_cs is float32 {(n_pos, head_dim // 2, 2)} on {dev}")
        s = a3_pages()
        s.dtype, s.format = {"f32": A3_F32, "bf16": A3_BF16}[dtype], A3_PAGES_Q8 if q8 else A3_PAGES_PLAIN
        s.n_q_heads, s.n_kv_heads, s.head_dim = n_q_heads, n_kv_heads, head_dim
        s.rope_layout, s.rope_base, s.sm_scale = rope_layout, rope_base, sm_scale
        s.page_size, s.n_pages, s.n_pos = page_size, n_pages, n_pos
        s.n_req, s.max_pages = page_table.shape
        s.k_pool, s.v_pool, s.page_table, s.rope_cs = _ptr(self.k_pool), _ptr(self.v_pool), _ptr(page_table), _ptr(self.rope_cs)
        self.struct = s
        self.ref = C.byref(s)
        self.torch_dtype, self.kv_elems, self.q_elems = torch_dtype(dtype), n_kv_heads * head_dim, n_q_heads * head_dim
        if fresh:
            a3_pages_prepare(self, stream)

    def sibling(self) -> "Pages":
        """Another layer's cache: pools of its own, the same page table and position table."""
        s = self.struct
        p = Pages(dtype=self.dtype, n_q_heads=s.n_q_heads, n_kv_heads=s.n_kv_heads, head_dim=s.head_dim, page_size=s.page_size,
                  n_pages=s.n_pages, page_table=self.page_table, rope_base=s.rope_base, n_pos=s.n_pos, rope_layout=s.rope_layout,
                  q8=self.q8, sm_scale=s.sm_scale, rope_cs=self.rope_cs)
        p.own_rope = self.own_rope
        return p

    def workspace(self, n_rows: int) -> torch.Tensor:
        return torch.empty(max(a3_paged_attention_ws_bytes(self, n_rows), 256), dtype=torch.uint8, device=self.device)

    def tree_workspace(self, n_groups: int, max_rows: int) -> torch.Tensor:
        return torch.empty(max(a3_tree_attention_ws_bytes(self, n_groups, max_rows), 256), dtype=torch.uint8, device=self.device)


class PageLayers:
    """The pages of a stack's layers as one, for calls that work on all of them: they share the page table and its shape (as
    ``Pages.sibling`` makes them)."""

    def __init__(self, pages):
        self.pages = list(pages)
        if not self.pages:
            raise ValueError("PageLayers: no pages")
        self.device, self.page_table = self.pages[0].device, self.pages[0].page_table
        if any(p.device != self.device or p.page_table.data_ptr() != self.page_table.data_ptr() for p in self.pages):
            raise ValueError("PageLayers: the layers share one page table")
        names = ("format", "dtype", "n_q_heads", "n_kv_heads", "head_dim", "page_size", "n_pages", "n_req", "max_pages")
        like = [tuple(getattr(p.struct, name) for name in names) for p in self.pages]
        for l, mine in enumerate(like):
            if mine != like[0]:
                raise ValueError(f"PageLayers: layer {l} has ({', '.join(names)}) {mine}, layer 0 {like[0]}")
        self.structs = (a3_pages * len(self.pages))(*[p.struct for p in self.pages])


class TokenLogprobs:
    """What a3_token_logprobs writes, and its workspace, allocated once for up to ``n_rows`` rows."""

    def __init__(self, n_rows: int, vocab: int, n_given: int, n_top: int, device="cuda"):
        new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device=device)
        self.n_given, self.n_top = n_given, n_top
        self.logprob, self.entropy = new(n_rows, n_given), new(n_rows)
        self.top_idx, self.top_logprob = new(n_rows, n_top, dtype=torch.int32), new(n_rows, n_top)
        self.ws = new(max(int(lib().a3_token_logprobs_ws_bytes(n_rows, vocab, n_top)), 256), dtype=torch.uint8)

    def rows(self, first: int, end: int) -> "TokenLogprobs":
        """Rows first .. end - 1 as outputs of their own, with the same workspace."""
        part = object.__new__(TokenLogprobs)
        part.n_given, part.n_top, part.ws = self.n_given, self.n_top, self.ws
        part.logprob, part.entropy = self.logprob[first:end], self.entropy[first:end]
        part.top_idx, part.top_logprob = self.top_idx[first:end], self.top_logprob[first:end]
        return part


class TreeAccepted:
    """What a3_tree_accept writes, and its workspace, allocated once for up to ``n_groups`` trees of ``n_rows`` rows together.
    ``vocab`` 0: the picked tokens are given."""

    def __init__(self, n_groups: int, n_rows: int, max_path: int, vocab: int = 0, device="cuda"):
        new = lambda *s: torch.empty(s, dtype=torch.int32, device=device)
        self.max_path = max_path
        self.picked, self.count, self.next_token = new(n_rows), new(n_groups), new(n_groups)
        self.path, self.src_slot, self.dst_slot = (new(n_groups, max_path) for _ in range(3))
        n = int(lib().a3_tree_accept_ws_bytes(n_rows, vocab)) if vocab else 0
        self.ws = torch.empty(max(n, 256), dtype=torch.uint8, device=device)


class BeamChoice:
    """What a3_beam_select writes, and its workspace, allocated once for up to ``n_groups`` groups of ``n_beams`` beams."""

    def __init__(self, n_groups: int, n_beams: int, vocab: int, n_best: int, device="cuda"):
        new = lambda dtype: torch.empty((n_groups, n_best), dtype=dtype, device=device)
        self.n_beams, self.n_best = n_beams, n_best
        self.score, self.row, self.token = new(torch.float32), new(torch.int32), new(torch.int32)
        n = int(lib().a3_beam_select_ws_bytes(n_groups, n_beams, vocab, n_best))
        self.ws = torch.empty(max(n, 256), dtype=torch.uint8, device=device)


# ---- entry points (same names as the C ABI) -----------------------------------------------------

def a3_version() -> int:
    return lib().a3_version()


def a3_set_tuning(name: str, value: int) -> None:
    _check(lib().a3_set_tuning(name.encode(), int(value)), "a3_set_tuning")


def a3_workspace_bytes(layout: Layout, max_active_rows: int) -> int:
    return int(lib().a3_workspace_bytes(layout.ref, int(max_active_rows)))


def a3_layout_prepare(layout: Layout, stream=None) -> None:
    _check(lib().a3_layout_prepare(layout.ref, _stream(stream)), "a3_layout_prepare")


def a3_rope_realign(layout: Layout, k_cat: torch.Tensor, k_fused: torch.Tensor, stream=None) -> None:
    _check(lib().a3_rope_realign(layout.ref, _ptr(k_cat), _ptr(k_fused), _stream(stream)), "a3_rope_realign")


def a3_question_scores(layout: Layout, q_question: torch.Tensor, k_fused: torch.Tensor, scores: torch.Tensor,
                       ws: torch.Tensor, stream=None) -> None:
    _check(lib().a3_question_scores(layout.ref, _ptr(q_question), _ptr(k_fused), _ptr(scores), _ptr(ws),
                                    ws.numel() if ws is not None else 0, _stream(stream)), "a3_question_scores")


def a3_question_scores_noalloc(layout: Layout, q_question: torch.Tensor, k_fused: torch.Tensor, scores: torch.Tensor,
                               stream=None) -> None:
    _check(lib().a3_question_scores_noalloc(layout.ref, _ptr(q_question), _ptr(k_fused), _ptr(scores),
                                            _stream(stream)), "a3_question_scores_noalloc")


def a3_realign_scores(layout: Layout, q_question: torch.Tensor, k_cat: torch.Tensor, k_fused: torch.Tensor,
                      scores: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(lib().a3_realign_scores(layout.ref, _ptr(q_question), _ptr(k_cat), _ptr(k_fused), _ptr(scores), _ptr(ws),
                                   ws.numel() if ws is not None else 0, _stream(stream)), "a3_realign_scores")


def a3_topk_select(layout: Layout, scores: torch.Tensor, sel_start: torch.Tensor, total_k: int,
                   sel_idx: torch.Tensor, ws: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().a3_topk_select(layout.ref, _ptr(scores), _ptr(sel_start), int(total_k), _ptr(sel_idx), _ptr(ws),
                                ws.numel() if ws is not None else 0, _stream(stream)), "a3_topk_select")


def a3_topk_select_plan(layout: Layout, scores: torch.Tensor, sel_start: torch.Tensor, total_k: int,
                        sel_idx: torch.Tensor, n_act: int, act_idx: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(lib().a3_topk_select_plan(layout.ref, _ptr(scores), _ptr(sel_start), int(total_k), _ptr(sel_idx), int(n_act),
                                     _ptr(act_idx), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)),
           "a3_topk_select_plan")


def a3_selected_qkv_proj(layout: Layout, hidden: torch.Tensor, row_idx: Optional[torch.Tensor], n_rows: int,
                         wq, wk, wv, bq=None, bk=None, bv=None, q_out=None, k_out=None, v_out=None,
                         stream=None) -> None:
    _check(lib().a3_selected_qkv_proj(layout.ref, _ptr(hidden), _ptr(row_idx), int(n_rows), _ptr(wq), _ptr(wk),
                                      _ptr(wv), _ptr(bq), _ptr(bk), _ptr(bv), _ptr(q_out), _ptr(k_out), _ptr(v_out),
                                      _stream(stream)), "a3_selected_qkv_proj")


def a3_selected_qkv_proj_scatter(layout: Layout, hidden: torch.Tensor, row_idx: Optional[torch.Tensor], n_rows: int,
                                 wq, wk, wv, bq=None, bk=None, bv=None, q_out=None, k_fused=None, v_fused=None,
                                 stream=None) -> None:
    _check(lib().a3_selected_qkv_proj_scatter(layout.ref, _ptr(hidden), _ptr(row_idx), int(n_rows), _ptr(wq),
                                              _ptr(wk), _ptr(wv), _ptr(bq), _ptr(bk), _ptr(bv), _ptr(q_out),
                                              _ptr(k_fused), _ptr(v_fused), _stream(stream)),
           "a3_selected_qkv_proj_scatter")


def a3_kv_scatter(layout: Layout, k_new: torch.Tensor, v_new: torch.Tensor, row_idx: torch.Tensor, n_rows: int,
                  k_fused: torch.Tensor, v_fused: torch.Tensor, stream=None) -> None:
    _check(lib().a3_kv_scatter(layout.ref, _ptr(k_new), _ptr(v_new), _ptr(row_idx), int(n_rows), _ptr(k_fused),
                               _ptr(v_fused), _stream(stream)), "a3_kv_scatter")


def a3_fused_attention(layout: Layout, q_act: torch.Tensor, act_idx: torch.Tensor, n_act: int, k_fused: torch.Tensor,
                       v_fused: torch.Tensor, out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(lib().a3_fused_attention(layout.ref, _ptr(q_act), _ptr(act_idx), int(n_act), _ptr(k_fused), _ptr(v_fused),
                                    _ptr(out), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)),
           "a3_fused_attention")


def a3_active_rows(layout: Layout, sel_idx: Optional[torch.Tensor], sel_start: torch.Tensor, n_act: int,
                   act_idx: torch.Tensor, stream=None) -> None:
    _check(lib().a3_active_rows(layout.ref, _ptr(sel_idx), _ptr(sel_start), int(n_act), _ptr(act_idx),
                                _stream(stream)), "a3_active_rows")


def a3_block_tail_ws_bytes(layout: Layout, ffn: int, n_rows: int) -> int:
    return int(lib().a3_block_tail_ws_bytes(layout.ref, int(ffn), int(n_rows)))


def a3_block_tail(layout: Layout, attn_out: torch.Tensor, act_idx: Optional[torch.Tensor], n_act: int, wo, g_post,
                  w_gate, w_up, w_down, g_next, eps: float, resid: torch.Tensor, hidden_next: torch.Tensor,
                  ws: torch.Tensor, stream=None) -> None:
    w = a3_block_weights(_ptr(wo), _ptr(g_post), _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(g_next),
                         int(w_gate.shape[0]), float(eps))
    _check(lib().a3_block_tail(layout.ref, _ptr(attn_out), _ptr(act_idx), int(n_act), C.byref(w), _ptr(resid),
                               _ptr(hidden_next), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)),
           "a3_block_tail")


def a3_rms_norm(layout: Layout, x: torch.Tensor, row_idx: Optional[torch.Tensor], n_rows: int, g: torch.Tensor,
                eps: float, out: torch.Tensor, stream=None) -> None:
    _check(lib().a3_rms_norm(layout.ref, _ptr(x), _ptr(row_idx), int(n_rows), _ptr(g), float(eps), _ptr(out),
                             _stream(stream)), "a3_rms_norm")


def a3_question_scores_causal(layout: Layout, q_question: torch.Tensor, k_fused: torch.Tensor, scores: torch.Tensor,
                              ws: torch.Tensor, stream=None) -> None:
    _check(lib().a3_question_scores_causal(layout.ref, _ptr(q_question), _ptr(k_fused), _ptr(scores), _ptr(ws),
                                           ws.numel() if ws is not None else 0, _stream(stream)),
           "a3_question_scores_causal")


def a3_window_votes(layout: Layout, q_question: torch.Tensor, k_fused: torch.Tensor, votes: torch.Tensor,
                    ws: torch.Tensor, stream=None) -> None:
    _check(lib().a3_window_votes(layout.ref, _ptr(q_question), _ptr(k_fused), _ptr(votes), _ptr(ws),
                                 ws.numel() if ws is not None else 0, _stream(stream)), "a3_window_votes")


def a3_evict_ws_bytes(layout: Layout) -> int:
    return int(lib().a3_evict_ws_bytes(layout.ref))


def a3_evict_select(layout: Layout, votes: torch.Tensor, sys_len: torch.Tensor, keep_start: torch.Tensor,
                    total_keep: int, keep_idx: torch.Tensor, pool_width: int = 1, pool_mode: int = A3_POOL_MAX,
                    ws: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().a3_evict_select(layout.ref, _ptr(votes), _ptr(sys_len), _ptr(keep_start), int(total_keep),
                                 int(pool_width), int(pool_mode), _ptr(keep_idx), _ptr(ws),
                                 ws.numel() if ws is not None else 0, _stream(stream)), "a3_evict_select")


def a3_evict_compact(layout: Layout, k_fused: torch.Tensor, v_fused: torch.Tensor, keep_idx: torch.Tensor,
                     total_keep: int, k_out: torch.Tensor, v_out: torch.Tensor, stream=None) -> None:
    _check(lib().a3_evict_compact(layout.ref, _ptr(k_fused), _ptr(v_fused), _ptr(keep_idx), int(total_keep),
                                  _ptr(k_out), _ptr(v_out), _stream(stream)), "a3_evict_compact")


def a3_value_deviation_scores(layout: Layout, v_true: torch.Tensor, v_cat: torch.Tensor, scores: torch.Tensor,
                              stream=None) -> None:
    _check(lib().a3_value_deviation_scores(layout.ref, _ptr(v_true), _ptr(v_cat), _ptr(scores), _stream(stream)),
           "a3_value_deviation_scores")


def a3_recompute_count(n_ctx: int, ratio_num: int, ratio_den: int) -> int:
    k = int(lib().a3_recompute_count(int(n_ctx), int(ratio_num), int(ratio_den)))
    if k < 0:
        raise A3Error(A3_ERR_INVALID_ARG, "a3_recompute_count", lib().a3_last_error().decode())
    return k


def a3_chunk_edge_sel_start(seg_start, ctx_len, chunk_start, chunk_len, n_head: int, n_tail: int) -> np.ndarray:
    """sel_start [R+1] for a3_select_chunk_edges, from host arrays."""
    i32 = lambda a: np.ascontiguousarray(a, dtype=np.int32)
    seg, ctx, cs, cl = i32(seg_start), i32(ctx_len), i32(chunk_start), i32(chunk_len)
    out = np.zeros(len(ctx) + 1, dtype=np.int32)
    p = lambda a: a.ctypes.data_as(C.POINTER(C.c_int))
    _check(lib().a3_chunk_edge_sel_start(len(ctx), p(seg), p(ctx), len(cs), p(cs), p(cl), int(n_head), int(n_tail), p(out)),
           "a3_chunk_edge_sel_start")
    return out


def a3_select_chunk_edges(layout: Layout, n_head: int, n_tail: int, sel_start: torch.Tensor, total_k: int,
                          sel_idx: torch.Tensor, stream=None) -> None:
    _check(lib().a3_select_chunk_edges(layout.ref, int(n_head), int(n_tail), _ptr(sel_start), int(total_k),
                                       _ptr(sel_idx), _stream(stream)), "a3_select_chunk_edges")


def a3_chunk_cache_load(layout: Layout, chunk_start, chunk_len, host_k, host_v, k_cat: torch.Tensor,
                        v_cat: torch.Tensor, stream=None) -> None:
    """host_k / host_v: one CPU tensor per chunk ([chunk_len, Hkv, d], pinned for asynchronous copies); the
    caller keeps them alive until the stream has passed the copies."""
    n = len(chunk_start)
    starts = (C.c_int * n)(*[int(x) for x in chunk_start])
    lens = (C.c_int * n)(*[int(x) for x in chunk_len])
    for t in list(host_k) + list(host_v):
        assert t is None or (t.device.type == "cpu" and t.is_contiguous())
    pk = (C.c_void_p * n)(*[t.data_ptr() if t is not None else None for t in host_k])
    pv = (C.c_void_p * n)(*[t.data_ptr() if t is not None else None for t in host_v])
    _check(lib().a3_chunk_cache_load(layout.ref, starts, lens, n, pk, pv, _ptr(k_cat), _ptr(v_cat), _stream(stream)),
           "a3_chunk_cache_load")


def a3_attention_plan(layout: Layout, act_idx: torch.Tensor, n_act: int, ws: torch.Tensor, stream=None) -> None:
    _check(lib().a3_attention_plan(layout.ref, _ptr(act_idx), int(n_act), _ptr(ws), ws.numel() if ws is not None else 0,
                                   _stream(stream)), "a3_attention_plan")


def a3_fused_attention_planned(layout: Layout, q_act: torch.Tensor, act_idx: torch.Tensor, n_act: int,
                               k_fused: torch.Tensor, v_fused: torch.Tensor, out: torch.Tensor, ws: torch.Tensor,
                               stream=None) -> None:
    _check(lib().a3_fused_attention_planned(layout.ref, _ptr(q_act), _ptr(act_idx), int(n_act), _ptr(k_fused),
                                            _ptr(v_fused), _ptr(out), _ptr(ws), ws.numel() if ws is not None else 0,
                                            _stream(stream)), "a3_fused_attention_planned")


def a3_fused_attention_planned_events(layout: Layout, q_act: torch.Tensor, act_idx: torch.Tensor, n_act: int,
                                      k_fused: torch.Tensor, v_fused: torch.Tensor, out: torch.Tensor, ws: torch.Tensor,
                                      ev_main_begin: Optional[int], ev_main_end: Optional[int], stream=None) -> None:
    """ev_main_begin / ev_main_end: raw hipEvent_t handles (integers) or None."""
    _check(lib().a3_fused_attention_planned_events(layout.ref, _ptr(q_act), _ptr(act_idx), int(n_act), _ptr(k_fused),
                                                   _ptr(v_fused), _ptr(out), _ptr(ws),
                                                   ws.numel() if ws is not None else 0, _stream(stream), ev_main_begin,
                                                   ev_main_end), "a3_fused_attention_planned_events")


def a3_q8_row_bytes(layout: Layout) -> int:
    return int(lib().a3_q8_row_bytes(layout.ref))


def a3_quantize_q8(layout: Layout, k: torch.Tensor, v: torch.Tensor, cache_q8: torch.Tensor, stream=None) -> None:
    _check(lib().a3_quantize_q8(layout.ref, _ptr(k), _ptr(v), _ptr(cache_q8), _stream(stream)), "a3_quantize_q8")


def a3_rope_realign_q8(layout: Layout, cache_q8: torch.Tensor, k_fused: Optional[torch.Tensor],
                       v_fused: Optional[torch.Tensor], stream=None) -> None:
    _check(lib().a3_rope_realign_q8(layout.ref, _ptr(cache_q8), _ptr(k_fused), _ptr(v_fused), _stream(stream)),
           "a3_rope_realign_q8")


def a3_chunk_cache_load_q8(layout: Layout, chunk_start, chunk_len, host_q8, cache_q8: torch.Tensor, stream=None) -> None:
    n = len(chunk_start)
    starts = (C.c_int * n)(*[int(x) for x in chunk_start])
    lens = (C.c_int * n)(*[int(x) for x in chunk_len])
    for t in host_q8:
        assert t is None or (t.device.type == "cpu" and t.is_contiguous())
    blocks = (C.c_void_p * n)(*[t.data_ptr() if t is not None else None for t in host_q8])
    _check(lib().a3_chunk_cache_load_q8(layout.ref, starts, lens, n, blocks, _ptr(cache_q8), _stream(stream)),
           "a3_chunk_cache_load_q8")


def a3_chunk_file_read(fds, file_offset, n_bytes, host_dst, n_threads: int = 4) -> None:
    """Blocking: block c = n_bytes[c] bytes at file_offset[c] of descriptor fds[c] into the CPU tensor host_dst[c]
    (the GIL is released meanwhile, so a Python thread can run it beside the launches)."""
    n = len(fds)
    for t, b in zip(host_dst, n_bytes):
        assert t is None or (t.device.type == "cpu" and t.is_contiguous() and t.numel() * t.element_size() >= b)
    _check(lib().a3_chunk_file_read(n, (C.c_int * n)(*[int(f) for f in fds]),
                                    (C.c_longlong * n)(*[int(o) for o in file_offset]),
                                    (C.c_size_t * n)(*[int(b) for b in n_bytes]),
                                    (C.c_void_p * n)(*[t.data_ptr() if t is not None else None for t in host_dst]),
                                    int(n_threads)), "a3_chunk_file_read")


# ---- generating on the fused cache -------------------------------------------------------------------

def a3_page_bytes(pages: Pages) -> int:
    return int(lib().a3_page_bytes(pages.ref))


def a3_pages_prepare(pages: Pages, stream=None) -> None:
    _current(pages.device)
    _check(lib().a3_pages_prepare(pages.ref, _stream(stream)), "a3_pages_prepare")


def _current(where: torch.device) -> int:
    """The index of the device a call's tensors are on, which has to be the current one."""
    if where.type != "cuda" or where.index not in (None, torch.cuda.current_device()):
        raise ValueError(f"the call's tensors are on {where}, the current device is another one")
    return torch.cuda.current_device()


def _hold(dev: int, dtype: torch.dtype, elems: int, *tensors) -> None:
    """Refuses tensors that are not ``elems`` elements (or more) of a type on device ``dev``."""
    for t in tensors:
        if t is not None and (t.get_device() != dev or t.dtype is not dtype or t.numel() < elems):
            raise ValueError(f"{elems} elements of {dtype} on cuda:{dev} are needed, got {tuple(t.shape)} {t.dtype} on {t.device}")


def a3_paged_append(pages: Pages, k: torch.Tensor, v: torch.Tensor, row_req: Optional[torch.Tensor], row_slot: torch.Tensor,
                    row_pos: Optional[torch.Tensor], n_rows: int, q: Optional[torch.Tensor] = None,
                    q_out: Optional[torch.Tensor] = None, stream=None) -> None:
    dev = _current(pages.device)
    _hold(dev, pages.torch_dtype, n_rows * pages.kv_elems, k, v)
    _hold(dev, pages.torch_dtype, n_rows * pages.q_elems, q, q_out)
    _hold(dev, torch.int32, n_rows, row_req, row_slot, row_pos)
    _check(lib().a3_paged_append(pages.ref, _ptr(k), _ptr(v), _ptr(row_req), _ptr(row_slot), _ptr(row_pos), int(n_rows), _ptr(q),
                                 _ptr(q_out), _stream(stream)), "a3_paged_append")


def a3_paged_attention_ws_bytes(pages: Pages, n_rows: int) -> int:
    return int(lib().a3_paged_attention_ws_bytes(pages.ref, int(n_rows)))


def a3_paged_attention(pages: Pages, q: torch.Tensor, row_req: Optional[torch.Tensor], row_len: torch.Tensor, n_rows: int,
                       out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    dev = _current(pages.device)
    _hold(dev, pages.torch_dtype, n_rows * pages.q_elems, q, out)
    _hold(dev, torch.int32, n_rows, row_req, row_len)
    _hold(dev, torch.uint8, 0, ws)
    _check(lib().a3_paged_attention(pages.ref, _ptr(q), _ptr(row_req), _ptr(row_len), int(n_rows), _ptr(out), _ptr(ws),
                                    ws.numel() if ws is not None else 0, _stream(stream)), "a3_paged_attention")


def a3_lm_head(layout: Layout, hidden: torch.Tensor, row_idx: Optional[torch.Tensor], n_rows: int, w: torch.Tensor,
               logits: torch.Tensor, stream=None) -> None:
    """``hidden`` [total_tokens, hidden] (without ``row_idx`` n_rows rows do); ``w`` [vocab, hidden]; ``logits`` float32 [>= n_rows,
    vocab], rows may be further apart than vocab."""
    h, vocab = layout.struct.hidden, w.shape[0]
    dev = _current(layout.device)
    _hold(dev, torch_dtype(layout.dtype), (layout.total_tokens if row_idx is not None else n_rows) * h, hidden)
    _hold(dev, torch_dtype(layout.dtype), vocab * h, w)
    _hold(dev, torch.int32, n_rows, row_idx)
    _hold(dev, torch.float32, 0, logits)
    if w.dim() != 2 or w.shape[1] != h or logits.dim() != 2 or logits.shape[0] < n_rows or logits.shape[1] != vocab \
            or logits.stride(1) != 1 or (logits.shape[0] > 1 and logits.stride(0) < vocab):
        raise ValueError(f"a3_lm_head: w is [vocab, {h}] and logits rows of vocab consecutive elements, got {tuple(w.shape)} and "
                         f"{tuple(logits.shape)}")
    _check(lib().a3_lm_head(layout.ref, _ptr(hidden), _ptr(row_idx), int(n_rows), _ptr(w), int(w.shape[0]), logits.data_ptr(),
                            logits.stride(0) if logits.shape[0] > 1 else w.shape[0], _stream(stream)), "a3_lm_head")


def a3_token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor], out: TokenLogprobs, stream=None) -> TokenLogprobs:
    """``logits`` [n_rows, vocab] float32 or bfloat16, rows may be further apart than vocab; ``tokens`` int32
    [n_rows, out.n_given].  Writes the first n_rows rows of ``out`` and returns it."""
    n_rows, vocab = logits.shape
    if logits.dtype not in (torch.float32, torch.bfloat16) or logits.stride(1) != 1 or (n_rows > 1 and logits.stride(0) < vocab):
        raise ValueError("a3_token_logprobs: logits are float32 or bfloat16 rows of consecutive elements")
    # (rows of tokens are n_given apart: a wider tensor would rate every row but the first on another row's tokens)
    if (tokens is None) != (out.n_given == 0) or (tokens is not None and tokens.dim() > 1 and tokens.shape[-1] != out.n_given):
        raise ValueError(f"a3_token_logprobs: tokens are int32 [{n_rows}, {out.n_given}], None for 0 given")
    dev = _current(logits.device)
    _hold(dev, torch.int32, n_rows * out.n_given, tokens)
    _hold(dev, torch.float32, n_rows, out.entropy)
    _hold(dev, torch.float32, n_rows * out.n_given, out.logprob)
    _hold(dev, torch.float32, n_rows * out.n_top, out.top_logprob)
    _hold(dev, torch.int32, n_rows * out.n_top, out.top_idx)
    _hold(dev, torch.uint8, 0, out.ws)
    _check(lib().a3_token_logprobs(A3_F32 if logits.dtype == torch.float32 else A3_BF16, logits.data_ptr(), n_rows, vocab,
                                   logits.stride(0) if n_rows > 1 else vocab, _ptr(tokens), out.n_given, out.n_top,
                                   _ptr(out.logprob), _ptr(out.entropy), _ptr(out.top_idx), _ptr(out.top_logprob), _ptr(out.ws),
                                   out.ws.numel(), _stream(stream)), "a3_token_logprobs")
    return out


# ---- several candidates of one request at once -------------------------------------------------------

def a3_tree_attention_ws_bytes(pages: Pages, n_groups: int, max_rows: int) -> int:
    return int(lib().a3_tree_attention_ws_bytes(pages.ref, int(n_groups), int(max_rows)))


def a3_tree_attention(pages: Pages, q: torch.Tensor, group_start: torch.Tensor, group_req: Optional[torch.Tensor],
                      group_len: torch.Tensor, mask: Optional[torch.Tensor], n_rows: int, max_rows: int, out: torch.Tensor,
                      ws: torch.Tensor, stream=None) -> None:
    """``group_start`` int32 [n_groups + 1]; ``mask`` int32 [n_rows, words] or None (chains)."""
    dev, n_groups = _current(pages.device), group_start.numel() - 1
    _hold(dev, pages.torch_dtype, n_rows * pages.q_elems, q, out)
    _hold(dev, torch.int32, n_groups, group_req, group_len)
    _hold(dev, torch.int32, 1, group_start)
    words = 0
    if mask is not None:
        if mask.dim() != 2 or mask.shape[0] < n_rows:
            raise ValueError(f"a3_tree_attention: mask is int32 [{n_rows}, words], got {tuple(mask.shape)}")
        _hold(dev, torch.int32, 0, mask)
        words = mask.shape[1]
    _hold(dev, torch.uint8, 0, ws)
    _check(lib().a3_tree_attention(pages.ref, _ptr(q), n_groups, _ptr(group_start), _ptr(group_req), _ptr(group_len), _ptr(mask), words,
                                   int(n_rows), int(max_rows), _ptr(out), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)),
           "a3_tree_attention")


def a3_tree_accept(logits: Optional[torch.Tensor], tokens: torch.Tensor, parent: torch.Tensor, group_start: torch.Tensor,
                   group_len: torch.Tensor, n_rows: int, max_rows: int, out: TreeAccepted, stream=None) -> TreeAccepted:
    """``logits`` [n_rows, vocab] float32 or bfloat16, rows may be further apart than vocab; None: ``out.picked`` holds the picked
    tokens.  ``tokens``, ``parent`` int32 [n_rows].  Writes the first n_groups rows of ``out`` and returns it."""
    n_groups = group_start.numel() - 1
    vocab = ld = dtype = 0
    if logits is not None:
        vocab, ld, dtype = _logit_rows("a3_tree_accept", logits, n_rows)
    dev = _current(out.picked.device)
    if logits is not None and logits.get_device() != dev:
        raise ValueError(f"a3_tree_accept: logits are on {logits.device}, the outputs on cuda:{dev}")
    _hold(dev, torch.int32, n_rows, tokens, parent, out.picked)
    _hold(dev, torch.int32, n_groups, group_len, out.count, out.next_token)
    _hold(dev, torch.int32, 1, group_start)
    _hold(dev, torch.int32, n_groups * out.max_path, out.path, out.src_slot, out.dst_slot)
    _hold(dev, torch.uint8, 0, out.ws)
    _check(lib().a3_tree_accept(dtype, None if logits is None else logits.data_ptr(), vocab, ld, _ptr(out.picked), _ptr(tokens), _ptr(parent),
                                n_groups, _ptr(group_start), _ptr(group_len), int(n_rows), int(max_rows), out.max_path, _ptr(out.count),
                                _ptr(out.path), _ptr(out.next_token), _ptr(out.src_slot), _ptr(out.dst_slot), _ptr(out.ws), out.ws.numel(),
                                _stream(stream)), "a3_tree_accept")
    return out


def a3_paged_move(layers: PageLayers, src_req: Optional[torch.Tensor], src_slot: torch.Tensor, dst_req: Optional[torch.Tensor],
                  dst_slot: torch.Tensor, n_slots: Optional[torch.Tensor], max_slots: int, n_sets: int, set_size: int, stream=None) -> None:
    """Index tensors int32 [n_sets, set_size]."""
    dev = _current(layers.device)
    _hold(dev, torch.int32, n_sets * set_size, src_req, src_slot, dst_req, dst_slot, n_slots)
    _check(lib().a3_paged_move(layers.structs, len(layers.structs), _ptr(src_req), _ptr(src_slot), _ptr(dst_req), _ptr(dst_slot), _ptr(n_slots),
                               int(max_slots), int(n_sets), int(set_size), _stream(stream)), "a3_paged_move")


def a3_beam_select(logits: torch.Tensor, score: torch.Tensor, done: Optional[torch.Tensor], end_token: int, out: BeamChoice,
                   stream=None) -> BeamChoice:
    """``logits`` [n_groups * out.n_beams, vocab] float32 or bfloat16, rows may be further apart than vocab; ``score`` float32 and
    ``done`` int32 (or None) of every row.  Writes the first n_groups rows of ``out`` and returns it."""
    n_rows = logits.shape[0]
    if n_rows % out.n_beams:
        raise ValueError(f"a3_beam_select: {n_rows} rows of logits are no groups of {out.n_beams} beams")
    vocab, ld, dtype = _logit_rows("a3_beam_select", logits, n_rows)
    dev, n_groups = _current(logits.device), n_rows // out.n_beams
    _hold(dev, torch.float32, n_rows, score)
    _hold(dev, torch.int32, n_rows, done)
    _hold(dev, torch.float32, n_groups * out.n_best, out.score)
    _hold(dev, torch.int32, n_groups * out.n_best, out.row, out.token)
    _hold(dev, torch.uint8, 0, out.ws)
    _check(lib().a3_beam_select(dtype, logits.data_ptr(), n_groups, out.n_beams, vocab, ld, _ptr(score), _ptr(done), int(end_token), out.n_best,
                                _ptr(out.score), _ptr(out.row), _ptr(out.token), _ptr(out.ws), out.ws.numel(), _stream(stream)), "a3_beam_select")
    return out


def _logit_rows(who: str, logits: torch.Tensor, n_rows: int):
    """(vocab, distance of rows, a3_dtype) of rows of logits."""
    if logits.dtype not in (torch.float32, torch.bfloat16) or logits.dim() != 2 or logits.shape[0] < n_rows or logits.stride(1) != 1 \
            or (logits.shape[0] > 1 and logits.stride(0) < logits.shape[1]):
        raise ValueError(f"{who}: logits are float32 or bfloat16 rows of consecutive elements, {n_rows} of them, got {tuple(logits.shape)} {logits.dtype}")
    vocab = logits.shape[1]
    return vocab, logits.stride(0) if logits.shape[0] > 1 else vocab, A3_F32 if logits.dtype == torch.float32 else A3_BF16
