"""The A^3 schedule over a stack of decoder blocks, as a sequence of C-ABI calls (Method, the paragraph in
front of Eq. 3, and Eq. 3-5).  Call sequencing and buffer allocation only; all arithmetic is in liba3.

    block 0        every row: input norm, Q/K/V, causal attention, H(.)
    layer 1        K, V of every row (the true keys of Eq. 3); Q of the question rows -> scores -> top-p (Re);
                   Q of the rows [Re, Q] -> attention (Eq. 4) -> H(.)
    layers >= 2    realign the layer's chunk cache (Eq. 2); Q/K/V of the rows [Re, Q] from X_l = H(O_{l-1}),
                   K/V stored into the cache (Eq. 5); attention; H(.)
    afterwards     one token per request and step: every layer's fused cache goes on as pages that grow (decode_stack); drafted
                   tokens of a request verified in one step (verify_stack), several beams of a request (beam_stack)
"""
from __future__ import annotations

import math
from typing import Dict, List, Sequence

import numpy as np
import torch

from . import api


def _bias(lw):
    return dict(bq=lw.get("bq"), bk=lw.get("bk"), bv=lw.get("bv"))


def _fit(pages, n_layers: int, n_req: int, tokens: int, layout: api.Layout, prompt: bool) -> None:
    """Refuses pages that cannot take what a call writes (a slot outside the page table would be skipped), and pages of another
    model than the layout's.  A prompt's keys come turned by the layout and its rows attended with the layout's scale, and the pages do
    both from then on; in a decoding step the pages alone do (its layout's rotation is the identity)."""
    if len(pages) < n_layers:
        raise ValueError(f"pages of {n_layers} layers are needed, got {len(pages)}")
    L = layout.struct
    for p in pages[:n_layers]:
        s = p.struct
        same = ["dtype", "n_q_heads", "n_kv_heads", "head_dim"]
        if prompt and s.n_pos > 0:                               # (without positions the pages turn nothing)
            same += ["rope_layout", "rope_base"] if p.own_rope else ["rope_layout"]
        for name in same:
            if getattr(s, name) != getattr(L, name):
                raise ValueError(f"pages: their {name} is {getattr(s, name)}, the layout's {getattr(L, name)}")
        scale = [x.sm_scale or x.head_dim ** -0.5 for x in (s, L)]
        if prompt and not math.isclose(*scale, rel_tol=1e-6):     # (0 stands for 1 / sqrt(head_dim); floats)
            raise ValueError("pages: their sm_scale is %g, the layout's %g" % tuple(scale))
        if s.n_req < n_req or s.max_pages * s.page_size < tokens:
            raise ValueError(f"pages: {n_req} requests of up to {tokens} tokens are needed, "
                             f"the table has {s.n_req} of {s.max_pages * s.page_size}")


def fuse_stack(layout: api.Layout, shape, layers: Sequence[Dict[str, torch.Tensor]], g_final: torch.Tensor,
               resid: torch.Tensor, k_cat: List[torch.Tensor], v_cat: List[torch.Tensor], sel_start: np.ndarray,
               q_rows: np.ndarray, stream=None, keep: bool = False, cache_stream=None, pages=None) -> dict:
    """``resid`` [T, h] holds the embedding output and is overwritten by the residual stream (all rows after
    block 0, the active rows afterwards).  ``k_cat[l]`` / ``v_cat[l]`` are the chunk caches of layer l >= 2
    (entries 0 and 1 are ignored); ``v_cat[l]`` is updated in place.  Every layer dict holds wq, wk, wv, wo,
    g_in, g_post, w_gate, w_up, w_down and optionally bq, bk, bv.
    With ``cache_stream`` (a loader.ChunkCacheStream) the caches are not resident: layer l's blocks are copied
    from host memory into a ring of device buffers while the layers before it compute, and ``k_cat`` / ``v_cat``
    are ignored; its blocks may be 8-bit (position recovery and dequantisation then run in one kernel).
    ``pages`` (one api.Pages per layer, a request of theirs for each of the layout's) receives every layer's fused cache,
    token p of a request in slot p, so that decode_stack can go on; type, heads, rotation and scale of both have to be the same.
    Returns dict(sel_idx, act_idx, n_act, scores, resid, hidden): ``hidden`` [T, h] holds the final-normed
    output at the active rows.  With ``keep`` every layer's attention output, caches, residual stream and the
    hidden states handed to the next layer are kept too (``per_layer[l]``: k, v, out, resid, x_next; whole arrays
    for block 0, the active rows afterwards), so that a test can check each layer on the inputs it really had."""
    dev, dt = layout.device, api.torch_dtype(layout.dtype)
    T, h = layout.total_tokens, shape.hidden
    Hq, Hkv, d = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    n_layers = len(layers)
    assert n_layers >= 2
    if pages is not None:
        _fit(pages, n_layers, layout.n_req, layout.max_len, layout, prompt=True)
    total_k, nq = int(sel_start[-1]), int(len(q_rows))
    n_act = total_k + nq
    eps = float(shape.rms_eps)
    ffn = int(layers[0]["w_gate"].shape[0])
    ws_attn = layout.workspace(T)
    # (few rows can need more than many: their reductions are split, and the partial results want room)
    ws_tail = torch.empty(max(*(api.a3_block_tail_ws_bytes(layout, ffn, n) for n in (T, n_act)), 256), dtype=torch.uint8, device=dev)
    x = torch.empty((T, h), dtype=dt, device=dev)
    kept = []

    def g_next(l):
        return layers[l + 1]["g_in"] if l + 1 < n_layers else g_final

    def tail(l, out, idx, n):
        lw = layers[l]
        api.a3_block_tail(layout, out, idx, n, lw["wo"], lw["g_post"], lw["w_gate"], lw["w_up"], lw["w_down"],
                          g_next(l), eps, resid, x, ws_tail, stream=stream)

    def to_pages(l, k, v):
        if pages is not None:
            api.a3_paged_append(pages[l], k, v, layout.tok_req, layout.tok_pos, None, T, stream=stream)

    if cache_stream is not None:
        for l in range(2, min(2 + cache_stream.depth, n_layers)):
            cache_stream.prefetch(l)

    # ---- block 0 on every row ---------------------------------------------------------------------------
    lw = layers[0]
    all_idx = torch.arange(T, dtype=torch.int32, device=dev)
    api.a3_rms_norm(layout, resid, None, T, lw["g_in"], eps, x, stream=stream)
    k_l = torch.empty((T, Hkv, d), dtype=dt, device=dev)
    v_l = torch.empty((T, Hkv, d), dtype=dt, device=dev)
    q_all = torch.empty((T, Hq, d), dtype=dt, device=dev)
    out_all = torch.empty((T, Hq, d), dtype=dt, device=dev)
    api.a3_selected_qkv_proj_scatter(layout, x, None, T, lw["wq"], lw["wk"], lw["wv"], q_out=q_all, k_fused=k_l,
                                     v_fused=v_l, stream=stream, **_bias(lw))
    api.a3_fused_attention(layout, q_all, all_idx, T, k_l, v_l, out_all, ws_attn, stream=stream)
    to_pages(0, k_l, v_l)
    tail(0, out_all, None, T)
    if keep:
        kept.append(dict(k=k_l.clone(), v=v_l.clone(), out=out_all.clone(), resid=resid.clone(), x_next=x.clone()))
    del q_all

    # ---- layer 1: true keys, scores, Re, attention of the rows [Re, Q] --------------------------------------
    lw = layers[1]
    q_rows_d = torch.as_tensor(np.ascontiguousarray(q_rows, dtype=np.int32), device=dev)
    sel_start_d = torch.as_tensor(np.ascontiguousarray(sel_start, dtype=np.int32), device=dev)
    q_question = torch.empty((max(nq, 1), Hq, d), dtype=dt, device=dev)
    scores = torch.empty(T, dtype=torch.float32, device=dev)
    sel_idx = torch.zeros(max(total_k, 1), dtype=torch.int32, device=dev)
    act_idx = torch.zeros(max(n_act, 1), dtype=torch.int32, device=dev)
    q_act = torch.empty((max(n_act, 1), Hq, d), dtype=dt, device=dev)
    out = out_all[:max(n_act, 1)]
    api.a3_selected_qkv_proj_scatter(layout, x, None, T, None, lw["wk"], lw["wv"], k_fused=k_l, v_fused=v_l,
                                     stream=stream, **_bias(lw))
    api.a3_selected_qkv_proj(layout, x, q_rows_d, nq, lw["wq"], None, None, bq=lw.get("bq"), q_out=q_question,
                             stream=stream)
    api.a3_question_scores(layout, q_question, k_l, scores, ws_attn, stream=stream)
    # selection, the row list [Re, Q] and the layout of the attention's work in one call.  The rows stay the same
    # from here on: the plan is made once and reused by every layer
    api.a3_topk_select_plan(layout, scores, sel_start_d, total_k, sel_idx, n_act, act_idx, ws_attn, stream=stream)
    api.a3_selected_qkv_proj(layout, x, act_idx, n_act, lw["wq"], None, None, bq=lw.get("bq"), q_out=q_act,
                             stream=stream)
    api.a3_fused_attention_planned(layout, q_act, act_idx, n_act, k_l, v_l, out, ws_attn, stream=stream)
    to_pages(1, k_l, v_l)
    tail(1, out, act_idx, n_act)
    act_long = act_idx[:n_act].long()
    if keep:
        kept.append(dict(k=k_l.clone(), v=v_l.clone(), out=out[:n_act].clone(), resid=resid[act_long], x_next=x[act_long]))

    # ---- layers 2 ..: Eq. 2, Eq. 5 --------------------------------------------------------------------------
    for l in range(2, n_layers):
        lw = layers[l]
        if cache_stream is not None and cache_stream.q8:
            # 8-bit blocks: both caches are expanded into the layer's own buffers and the ring slot is free again
            api.a3_rope_realign_q8(layout, cache_stream.acquire(l, stream), k_l, v_l, stream=stream)
            v_c = v_l
            cache_stream.release(l, stream)
            cache_stream.prefetch(l + cache_stream.depth)
        else:
            k_c, v_c = (k_cat[l], v_cat[l]) if cache_stream is None else cache_stream.acquire(l, stream)
            api.a3_rope_realign(layout, k_c, k_l, stream=stream)
        api.a3_selected_qkv_proj_scatter(layout, x, act_idx, n_act, lw["wq"], lw["wk"], lw["wv"], q_out=q_act,
                                         k_fused=k_l, v_fused=v_c, stream=stream, **_bias(lw))
        api.a3_fused_attention_planned(layout, q_act, act_idx, n_act, k_l, v_c, out, ws_attn, stream=stream)
        to_pages(l, k_l, v_c)
        if keep:
            kept.append(dict(k=k_l.clone(), v=v_c.clone(), out=out[:n_act].clone()))
        if cache_stream is not None and not cache_stream.q8:
            cache_stream.release(l, stream)
            cache_stream.prefetch(l + cache_stream.depth)
        tail(l, out, act_idx, n_act)
        if keep:
            kept[-1].update(resid=resid[act_long], x_next=x[act_long])
    return dict(sel_idx=sel_idx[:total_k], act_idx=act_idx[:n_act], n_act=n_act, scores=scores, resid=resid, hidden=x,
                per_layer=kept)


def prefill_stack(layout: api.Layout, shape, layers: Sequence[Dict[str, torch.Tensor]], g_final: torch.Tensor,
                  resid: torch.Tensor, stream=None, keep_kv: bool = False, pages=None) -> dict:
    """Every block on every row: the plain prefill the schedule above is measured against (and, run on one
    chunk alone, the precompute of Eq. 1 that produces a chunk's per-layer K/V).  ``resid`` [T, h] holds the
    embedding output and is overwritten.  ``pages`` as in fuse_stack.  Returns dict(resid, hidden, k=[...], v=[...] if
    keep_kv)."""
    dev, dt = layout.device, api.torch_dtype(layout.dtype)
    T, h = layout.total_tokens, shape.hidden
    Hq, Hkv, d = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    n_layers = len(layers)
    if pages is not None:
        _fit(pages, n_layers, layout.n_req, layout.max_len, layout, prompt=True)
    eps = float(shape.rms_eps)
    ffn = int(layers[0]["w_gate"].shape[0])
    ws_attn = layout.workspace(T)
    ws_tail = torch.empty(max(api.a3_block_tail_ws_bytes(layout, ffn, T), 256), dtype=torch.uint8, device=dev)
    x = torch.empty((T, h), dtype=dt, device=dev)
    all_idx = torch.arange(T, dtype=torch.int32, device=dev)
    q_all = torch.empty((T, Hq, d), dtype=dt, device=dev)
    out_all = torch.empty((T, Hq, d), dtype=dt, device=dev)
    k_l = torch.empty((T, Hkv, d), dtype=dt, device=dev)
    v_l = torch.empty((T, Hkv, d), dtype=dt, device=dev)
    ks, vs = [], []
    api.a3_rms_norm(layout, resid, None, T, layers[0]["g_in"], eps, x, stream=stream)
    for l, lw in enumerate(layers):
        if keep_kv and l > 0:
            k_l, v_l = torch.empty_like(k_l), torch.empty_like(v_l)
        api.a3_selected_qkv_proj_scatter(layout, x, None, T, lw["wq"], lw["wk"], lw["wv"], q_out=q_all, k_fused=k_l,
                                         v_fused=v_l, stream=stream, **_bias(lw))
        api.a3_fused_attention(layout, q_all, all_idx, T, k_l, v_l, out_all, ws_attn, stream=stream)
        if pages is not None:
            api.a3_paged_append(pages[l], k_l, v_l, layout.tok_req, layout.tok_pos, None, T, stream=stream)
        g_next = layers[l + 1]["g_in"] if l + 1 < n_layers else g_final
        api.a3_block_tail(layout, out_all, None, T, lw["wo"], lw["g_post"], lw["w_gate"], lw["w_up"], lw["w_down"],
                          g_next, eps, resid, x, ws_tail, stream=stream)
        if keep_kv:
            ks.append(k_l)
            vs.append(v_l)
    return dict(resid=resid, hidden=x, k=ks, v=vs)


def _ready(dev: int, dtype: torch.dtype, elems: int, *tensors) -> None:
    """Refuses what one of a step's last calls would refuse, after the others have changed the caches: tensors of another type or device,
    of fewer elements, or apart."""
    api._hold(dev, dtype, elems, *tensors)
    if not all(t is None or t.is_contiguous() for t in tensors):
        raise ValueError("the tensors of a step are contiguous")


def _workspace(dev: int, need: int, what: str, *tensors) -> None:
    """Refuses workspaces smaller than ``need`` (0: what they are for is not supported)."""
    if need == 0:
        raise ValueError(f"{what} of such sizes are not supported")
    _ready(dev, torch.uint8, need, *tensors)


class DecodeBuffers:
    """What one decoding step of up to ``layout.n_req`` rows writes, allocated once (a captured graph keeps using them).
    ``layout`` is an api.Layout.decode; ``pages`` one api.Pages per layer; ``vocab`` > 0 asks for logits too; ``tree`` (trees, most
    tokens of one) for steps over drafted trees."""

    def __init__(self, layout: api.Layout, shape, ffn: int, pages: Sequence[api.Pages], vocab: int = 0, tree=None):
        dev, dt, n = layout.device, api.torch_dtype(layout.dtype), layout.n_req
        new = lambda *s: torch.empty(s, dtype=dt, device=dev)
        self.x = new(n, shape.hidden)
        self.q, self.out = new(n, shape.n_q_heads, shape.head_dim), new(n, shape.n_q_heads, shape.head_dim)
        self.k, self.v = new(n, shape.n_kv_heads, shape.head_dim), new(n, shape.n_kv_heads, shape.head_dim)
        self.ws_attn = pages[0].workspace(n)
        self.ws_tree = pages[0].tree_workspace(*tree) if tree else None
        self.rows = torch.arange(n, dtype=torch.int32, device=dev)
        self.source, self.runs = torch.empty_like(self.rows), torch.empty_like(self.rows)    # of steps of beams
        # (few rows can need more than many: their reductions are split, and the partial results want room)
        self.ws_tail = torch.empty(max([256] + [api.a3_block_tail_ws_bytes(layout, ffn, m) for m in range(1, n + 1)]), dtype=torch.uint8, device=dev)
        self.logits = torch.empty((n, vocab), dtype=torch.float32, device=dev) if vocab else None


def decode_stack(layout: api.Layout, shape, layers: Sequence[Dict[str, torch.Tensor]], g_final: torch.Tensor,
                 resid: torch.Tensor, pages: Sequence[api.Pages], row_slot: torch.Tensor, row_pos: torch.Tensor,
                 row_len, bufs: DecodeBuffers, row_req=None, w_vocab=None, stream=None, tree: "TreeRows" = None) -> dict:
    """One new token per row through every block.  ``resid`` [n_req, h] holds the tokens' embeddings and is overwritten by
    the residual stream.  Row i belongs to request ``row_req[i]`` of the pages (None: i); its K and V go to slot
    ``row_slot[i]``, turned to position ``row_pos[i]``, and it sees the slots below ``row_len[i]`` (its own included: row_slot +
    1).  All four are device int32, so that a captured step is replayed with the next values in them; a row whose request
    is -1 is padding: no cache row is written for it and its outputs mean nothing (nor do those of a row whose slot or position
    lies outside the pages).  ``w_vocab`` [vocab, h]: logits of every row too.  With ``tree`` the rows are drafted tokens, which see what
    it says (``row_len`` is not looked at).  Returns dict(hidden, resid, logits)."""
    n, eps, b = layout.n_req, float(shape.rms_eps), bufs
    if len(b.x) < n or (w_vocab is not None and b.logits is None):
        raise ValueError(f"buffers of {len(b.x)} rows{' without logits' if b.logits is None else ''} for a step of {n}")
    if w_vocab is not None and w_vocab.shape[0] != b.logits.shape[1]:
        raise ValueError(f"buffers of {b.logits.shape[1]} logits for a vocabulary of {w_vocab.shape[0]}")
    if tree is not None and b.ws_tree is None:
        raise ValueError("buffers without room for trees for a step over trees")
    if tree is not None and tree.n_rows != n:
        raise ValueError(f"trees of {tree.n_rows} rows for a step of {n}")
    _fit(pages, len(layers), n if row_req is None else 0, 0, layout, prompt=False)
    dev = b.x.get_device()
    if row_slot is None or (row_len is None and tree is None):
        raise ValueError("a step needs every row's slot and length")
    _ready(dev, api.torch_dtype(layout.dtype), n * layout.struct.hidden, resid, b.x)
    _ready(dev, torch.int32, n, row_req, row_slot, row_pos, row_len)
    if w_vocab is not None:
        if w_vocab.dim() != 2 or w_vocab.shape[1] != layout.struct.hidden:
            raise ValueError(f"w_vocab is [vocab, {layout.struct.hidden}], got {tuple(w_vocab.shape)}")
        _ready(dev, api.torch_dtype(layout.dtype), w_vocab.numel(), w_vocab)
    if tree is None:
        _workspace(dev, max(api.a3_paged_attention_ws_bytes(pages[0], n), 1), "rows", b.ws_attn)
    else:
        groups = tree.group_start.numel() - 1
        _ready(dev, torch.int32, groups, tree.group_start, tree.group_req, tree.group_len)
        _workspace(dev, api.a3_tree_attention_ws_bytes(pages[0], groups, tree.max_rows), "trees", b.ws_tree)
    _workspace(dev, max(api.a3_block_tail_ws_bytes(layout, int(layers[0]["w_gate"].shape[0]), n), 1), "rows", b.ws_tail)
    api.a3_rms_norm(layout, resid, None, n, layers[0]["g_in"], eps, b.x, stream=stream)
    for l, lw in enumerate(layers):
        api.a3_selected_qkv_proj(layout, b.x, None, n, lw["wq"], lw["wk"], lw["wv"], q_out=b.q, k_out=b.k, v_out=b.v,
                                 stream=stream, **_bias(lw))
        api.a3_paged_append(pages[l], b.k, b.v, row_req, row_slot, row_pos, n, q=b.q, q_out=b.q, stream=stream)
        if tree is None:
            api.a3_paged_attention(pages[l], b.q, row_req, row_len, n, b.out, b.ws_attn, stream=stream)
        else:
            api.a3_tree_attention(pages[l], b.q, tree.group_start, tree.group_req, tree.group_len, tree.mask, n, tree.max_rows, b.out,
                                  b.ws_tree, stream=stream)
        g_next = layers[l + 1]["g_in"] if l + 1 < len(layers) else g_final
        api.a3_block_tail(layout, b.out, None, n, lw["wo"], lw["g_post"], lw["w_gate"], lw["w_up"], lw["w_down"], g_next, eps,
                          resid, b.x, b.ws_tail, stream=stream)
    if w_vocab is not None:
        api.a3_lm_head(layout, b.x, None, n, w_vocab, b.logits, stream=stream)
    return dict(hidden=b.x[:n], resid=resid, logits=b.logits[:n] if w_vocab is not None else None)


class TreeRows:
    """Drafted trees of a batch as one step takes them, device int32 all (a captured step is replayed with the next ones in them).
    ``parents[g]``: the parent of every token of tree g inside it, -1 for the root in front; ``lens[g]``: the committed slots of its
    request, ``reqs[g]`` (None: g); ``tokens``: of all rows, the roots' ones are not looked at; ``positions[g]`` of the root (None:
    lens[g]; after an eviction another); ``max_path``: of the api.TreeAccepted that the step writes."""

    def __init__(self, parents, lens, tokens=None, reqs=None, positions=None, max_rows: int = 0, max_path: int = 16, device="cuda"):
        i32 = lambda a: torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=device)
        rows = [len(p) for p in parents]
        n, self.max_rows = sum(rows), max(rows + [1, max_rows])
        if self.max_rows > 1024 or not 1 <= max_path <= 64:
            raise ValueError(f"TreeRows: trees of {self.max_rows} rows (1024 at most), paths of {max_path} (1 to 64)")
        for name, of, many in (("lens", lens, len(rows)), ("reqs", reqs, len(rows)), ("positions", positions, len(rows)), ("tokens", tokens, n)):
            if of is not None and math.prod(np.shape(of)) != many:
                raise ValueError(f"TreeRows: {many} {name} are needed for {len(rows)} trees of {n} rows, got {np.shape(of)}")
        words = -(-self.max_rows // 32)
        seen, depth = np.zeros((n, 32 * words), dtype=np.uint8), np.zeros(n, dtype=np.int64)
        start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int64)
        for g, tree in enumerate(parents):
            for j, p in enumerate(tree):
                if not (p == -1 if j == 0 else 0 <= p < j):
                    raise ValueError(f"TreeRows: row {j} of tree {g} has parent {p}: row 0 is the root, parents stand in front")
                row = start[g] + j
                if j:
                    seen[row], depth[row] = seen[start[g] + p], depth[start[g] + p] + 1
                seen[row, j] = 1
        reqs = np.arange(len(rows)) if reqs is None else np.asarray(reqs)
        lens = np.maximum(np.asarray(lens, dtype=np.int64), 0)       # (below 0: none, as a3_tree_attention takes it)
        first = lens if positions is None else np.asarray(positions, dtype=np.int64)
        inside = np.arange(n) - np.repeat(start[:-1], rows)
        self.n_rows, self.tokens = n, i32(np.zeros(n) if tokens is None else tokens)
        self.group_start, self.group_req, self.group_len = i32(start), i32(reqs), i32(lens)
        self.parent = i32(np.concatenate([np.asarray(p, dtype=np.int32) for p in parents] + [np.zeros(0, dtype=np.int32)]))
        self.mask = i32(np.packbits(seen, axis=1, bitorder="little").view(np.int32)) if n else i32(np.zeros((0, words)))
        self.path_req = i32(np.repeat(reqs[:, None], max_path, 1))
        self.row_req, self.row_slot = i32(np.repeat(reqs, rows)), i32(np.repeat(lens, rows) + inside)
        self.row_pos = i32(np.repeat(first, rows) + depth)


def verify_stack(layout: api.Layout, shape, layers: Sequence[Dict[str, torch.Tensor]], g_final: torch.Tensor, resid: torch.Tensor,
                 pages: api.PageLayers, tree: TreeRows, bufs: DecodeBuffers, w_vocab: torch.Tensor, out: api.TreeAccepted,
                 stream=None) -> dict:
    """Drafted tokens through every block at once, and what of them the model would have said: ``resid`` [tree.n_rows, h] holds the
    embeddings of the trees' tokens (row 0 of a tree: its request's last certain token, whose K and V are not in the cache yet).
    ``out`` receives the picked tokens (largest logits), the accepted paths and the tokens behind them; the accepted rows of every
    layer's cache move to the slots behind the committed ones, so that a request has ``group_len + count`` of them afterwards (what
    lies behind is free).  ``layout`` has a row for each drafted token.  Returns decode_stack's dict."""
    if w_vocab is None:
        raise ValueError("verify_stack: the picks are of the step's logits: w_vocab is needed")
    if out.max_path != tree.path_req.shape[1]:
        raise ValueError(f"verify_stack: paths of {out.max_path} for trees of paths of {tree.path_req.shape[1]}")
    dev, groups = resid.get_device(), len(tree.path_req)
    if groups > 65535:
        raise ValueError(f"verify_stack: {groups} trees (65535 at most)")
    _ready(dev, torch.int32, tree.n_rows, tree.tokens, tree.parent, out.picked)
    _ready(dev, torch.int32, groups, tree.group_start, tree.group_len, out.count, out.next_token)
    _ready(dev, torch.int32, groups * out.max_path, tree.path_req, out.path, out.src_slot, out.dst_slot)
    _workspace(dev, int(api.lib().a3_tree_accept_ws_bytes(tree.n_rows, w_vocab.shape[0])), "picks", out.ws)
    r = decode_stack(layout, shape, layers, g_final, resid, pages.pages, tree.row_slot, tree.row_pos, None, bufs, row_req=tree.row_req,
                     w_vocab=w_vocab, stream=stream, tree=tree)
    api.a3_tree_accept(r["logits"], tree.tokens, tree.parent, tree.group_start, tree.group_len, layout.n_req, tree.max_rows, out, stream=stream)
    api.a3_paged_move(pages, tree.path_req, out.src_slot, tree.path_req, out.dst_slot, None, 1, len(tree.path_req), out.max_path, stream=stream)
    return r


def beam_stack(layout: api.Layout, shape, layers: Sequence[Dict[str, torch.Tensor]], g_final: torch.Tensor, resid: torch.Tensor,
               pages: api.PageLayers, row_slot: torch.Tensor, row_pos: torch.Tensor, row_len: torch.Tensor, bufs: DecodeBuffers,
               w_vocab: torch.Tensor, score: torch.Tensor, first_slot: torch.Tensor, n_slots: torch.Tensor, max_slots: int,
               out: api.BeamChoice, done=None, end_token: int = 0, stream=None) -> dict:
    """One step of beam search: a token of every beam through every block, the best continuations of every group of ``out.n_beams`` rows
    (row = beam = request of the pages), and the caches of the beams that go on in place of the others: beam j of a group takes over
    slots ``first_slot`` .. + ``n_slots`` (at most ``max_slots``) of row ``out.row[g, j]``, as many as that row has; in front of them the beams of
    a group have the same tokens, in pages of their own or shared.  ``first_slot`` (equal within a group), ``n_slots`` (of every row its own: beams
    that have ended may hold fewer; None: 1): device int32 [rows], the latter counting the new token.
    ``score`` of every row, ``done`` and ``end_token`` as for a3_beam_select; ``out`` has as many best ones as beams.  Returns decode_stack's
    dict."""
    if out.n_best != out.n_beams:
        raise ValueError(f"beam_stack: {out.n_best} continuations for {out.n_beams} beams")
    if layout.n_req % out.n_beams:
        raise ValueError(f"beam_stack: {layout.n_req} rows are no groups of {out.n_beams} beams")
    if w_vocab is None:
        raise ValueError("beam_stack: the choice is of the step's logits: w_vocab is needed")
    dev, n, groups = resid.get_device(), layout.n_req, layout.n_req // out.n_beams
    if score is None or first_slot is None or max_slots < 0 or (done is not None and end_token < 0) or groups > 65535:
        raise ValueError(f"beam_stack: every beam's score and first slot are needed, max_slots {max_slots}, end_token {end_token}, {groups} groups")
    _ready(dev, torch.float32, n, score, out.score)
    _ready(dev, torch.int32, n, done, first_slot, n_slots, out.row, out.token)
    _workspace(dev, int(api.lib().a3_beam_select_ws_bytes(groups, out.n_beams, w_vocab.shape[0], out.n_best)), "beams", out.ws)
    r = decode_stack(layout, shape, layers, g_final, resid, pages.pages, row_slot, row_pos, row_len, bufs, w_vocab=w_vocab, stream=stream)
    api.a3_beam_select(r["logits"], score, done, end_token, out, stream=stream)
    # a move is as long as its source's run (where there is no source, -1, nothing moves, whatever the length)
    runs = None
    if n_slots is not None:
        runs = bufs.runs[:n]
        with torch.cuda.stream(api.torch_stream(stream)):
            torch.clamp(out.row.view(-1)[:n], min=0, out=bufs.source[:n])
            torch.index_select(n_slots.view(-1), 0, bufs.source[:n], out=runs)
    api.a3_paged_move(pages, out.row, first_slot, bufs.rows, first_slot, runs, max_slots, n // out.n_beams, out.n_beams, stream=stream)
    return r


def score_tokens(layout: api.Layout, hidden: torch.Tensor, row_idx, n_rows: int, w_vocab: torch.Tensor, tokens,
                 out: api.TokenLogprobs, rows_at_once: int = 1024, stream=None) -> api.TokenLogprobs:
    """Log probabilities of given tokens (and entropy, alternatives) behind rows of final-normed hidden states, as fuse_stack,
    prefill_stack and decode_stack return them: ``tokens`` int32 [n_rows, out.n_given] beside the packed rows ``row_idx`` (None:
    the first n_rows; of a row outside [0, total_tokens) the outputs mean nothing).  The logits of ``rows_at_once`` rows at a
    time are formed and read (1024 rows of 128256: 0.5 GB).  ``stream``: a torch stream or a raw handle."""
    with torch.cuda.stream(api.torch_stream(stream)):                # the logits live and die on it
        logits = torch.empty((min(max(n_rows, 1), rows_at_once), w_vocab.shape[0]), dtype=torch.float32, device=hidden.device)
        for i in range(0, n_rows, rows_at_once):
            m = min(rows_at_once, n_rows - i)
            if row_idx is None:
                api.a3_lm_head(layout, hidden[i:i + m], None, m, w_vocab, logits[:m])
            else:
                api.a3_lm_head(layout, hidden, row_idx[i:i + m], m, w_vocab, logits[:m])
            api.a3_token_logprobs(logits[:m], None if tokens is None else tokens[i:i + m], out.rows(i, i + m))
    return out
