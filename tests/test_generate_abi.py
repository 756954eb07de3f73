"""What the entry points for generating refuse on the host, before anything is launched (no GPU needed)."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2511_17560_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X = 0x1000          # never dereferenced on the host


def _pages(**over):
    s = api.a3_pages()
    s.dtype, s.format, s.n_q_heads, s.n_kv_heads, s.head_dim = api.A3_BF16, api.A3_PAGES_PLAIN, 32, 8, 128
    s.rope_layout, s.rope_base, s.sm_scale = 1, 5e5, 0.0
    s.page_size, s.n_pages, s.n_req, s.max_pages, s.n_pos = 64, 1000, 4, 300, 20000
    s.k_pool = s.v_pool = s.page_table = s.rope_cs = X
    for k, v in over.items():
        setattr(s, k, v)
    return s


def test_structs_match_the_header():
    text = open(os.path.join(ROOT, "include", "a3.h")).read()
    body = re.sub(r"/\*.*?\*/", "", text[text.index("typedef struct a3_pages {"):text.index("} a3_pages;")], flags=re.S)
    assert re.findall(r"\b\*?\s*([a-z_]+)\s*;", body) == [f[0] for f in api.a3_pages._fields_]


@pytest.mark.parametrize("over,status", [
    (dict(dtype=5), api.A3_ERR_INVALID_ARG), (dict(format=2), api.A3_ERR_INVALID_ARG), (dict(rope_layout=2), api.A3_ERR_INVALID_ARG),
    (dict(n_q_heads=30), api.A3_ERR_INVALID_ARG), (dict(n_kv_heads=0), api.A3_ERR_INVALID_ARG), (dict(n_kv_heads=1), api.A3_ERR_UNSUPPORTED),
    (dict(head_dim=96), api.A3_ERR_UNSUPPORTED), (dict(rope_base=1.0), api.A3_ERR_INVALID_ARG), (dict(sm_scale=-1.0), api.A3_ERR_INVALID_ARG),
    (dict(page_size=16), api.A3_ERR_UNSUPPORTED), (dict(page_size=96), api.A3_ERR_UNSUPPORTED), (dict(page_size=2048), api.A3_ERR_UNSUPPORTED),
    (dict(page_size=0), api.A3_ERR_UNSUPPORTED), (dict(page_size=-64), api.A3_ERR_UNSUPPORTED), (dict(n_pages=0), api.A3_ERR_INVALID_ARG),
    (dict(n_req=0), api.A3_ERR_INVALID_ARG), (dict(max_pages=0), api.A3_ERR_INVALID_ARG), (dict(n_pos=-1), api.A3_ERR_INVALID_ARG),
    (dict(k_pool=None), api.A3_ERR_INVALID_ARG), (dict(v_pool=0x1008), api.A3_ERR_INVALID_ARG), (dict(page_table=None), api.A3_ERR_INVALID_ARG)])
def test_bad_pages_are_refused(over, status):
    L, p = api.lib(), C.byref(_pages(**over))
    assert L.a3_paged_append(p, X, X, None, X, X, 2, None, None, None) == status and L.a3_last_error() != b""
    assert L.a3_paged_attention(p, X, None, X, 2, X, X, 1 << 40, None) == status
    if not {"k_pool", "v_pool", "page_table"} & set(over):
        assert L.a3_page_bytes(p) == 0 and L.a3_paged_attention_ws_bytes(p, 2) == 0 and L.a3_pages_prepare(p, None) == status


def test_page_sizes():
    L = api.lib()
    assert L.a3_page_bytes(C.byref(_pages())) == 8 * 64 * 128 * 2
    assert L.a3_page_bytes(C.byref(_pages(dtype=api.A3_F32, head_dim=64, page_size=32))) == 8 * 32 * 64 * 4
    assert L.a3_page_bytes(C.byref(_pages(format=api.A3_PAGES_Q8))) == 8 * 64 * (128 + 4)
    assert L.a3_page_bytes(None) == 0


def test_append_refuses():
    L, p = api.lib(), C.byref(_pages())
    call = lambda *a: L.a3_paged_append(p, *a, None)
    bad = api.A3_ERR_INVALID_ARG
    assert call(None, None, None, None, None, 0, None, None) == api.A3_OK                # nothing to do
    assert call(X, X, None, X, X, -1, None, None) == bad
    assert call(None, X, None, X, X, 2, None, None) == bad and call(X, None, None, X, X, 2, None, None) == bad
    assert call(X, X, None, None, X, 2, None, None) == bad
    assert call(X, X, None, X, X, 5, None, None) == bad                                  # more rows than requests, and no row_req
    assert call(X, X, None, X, X, 2, X, None) == bad and call(X, X, None, X, X, 2, None, X) == bad
    assert call(X, X, None, X, None, 2, X, X) == bad                                     # q without positions
    assert call(X + 8, X, None, X, X, 2, None, None) == bad and call(X, X, None, X, X, 2, X, X + 4) == bad
    assert call(X, X, X, X, None, 2 ** 31 - 1, None, None) == api.A3_ERR_UNSUPPORTED
    assert L.a3_paged_append(C.byref(_pages(rope_cs=None)), X, X, None, X, X, 2, None, None, None) == bad
    assert L.a3_pages_prepare(C.byref(_pages(rope_cs=None)), None) == bad
    assert L.a3_pages_prepare(C.byref(_pages(rope_cs=None, n_pos=0)), None) == api.A3_OK


def test_attention_refuses():
    L, p = api.lib(), C.byref(_pages())
    call = lambda *a: L.a3_paged_attention(p, *a, None)
    bad, need = api.A3_ERR_INVALID_ARG, L.a3_paged_attention_ws_bytes(p, 4)
    assert need > 0 and L.a3_paged_attention_ws_bytes(p, -1) == 0
    assert call(None, None, None, 0, None, None, 0) == api.A3_OK
    assert call(X, None, X, -1, X, X, need) == bad and call(X, None, X, 5, X, X, need) == bad
    assert call(None, None, X, 4, X, X, need) == bad and call(X, None, None, 4, X, X, need) == bad and call(X, None, X, 4, None, X, need) == bad
    assert call(X + 8, None, X, 4, X, X, need) == bad and call(X, None, X, 4, X + 2, X, need) == bad
    for ws in ((None, 0), (None, need), (X, need - 1), (X + 8, need)):
        assert call(X, None, X, 4, X, *ws) == api.A3_ERR_WORKSPACE
    assert call(X, X, X, 2 ** 31 - 1, X, X, 1 << 60) == api.A3_ERR_UNSUPPORTED


def _layout(**over):
    s = api.a3_layout()
    s.dtype, s.n_q_heads, s.n_kv_heads, s.head_dim, s.hidden = api.A3_BF16, 32, 8, 128, 4096
    s.rope_layout, s.rope_base, s.n_req, s.total_tokens, s.max_q_len = 0, 5e5, 4, 4, 1
    for f in ("seg_start", "ctx_len", "q_len", "tok_pos", "tok_req", "tok_chunk", "q_start", "rope_chunk_cs", "rope_pos_cs"):
        setattr(s, f, X)
    for k, v in over.items():
        setattr(s, k, v)
    return s


def test_lm_head_refuses():
    L, p = api.lib(), C.byref(_layout())
    call = lambda *a: L.a3_lm_head(p, *a, None)
    bad = api.A3_ERR_INVALID_ARG
    assert call(None, None, 0, None, 100, None, 100) == api.A3_OK
    assert call(X, None, -1, X, 100, X, 100) == bad and call(X, None, 5, X, 100, X, 100) == bad
    assert call(X, None, 4, X, 0, X, 100) == bad and call(X, None, 4, X, 100, X, 99) == bad
    assert call(None, None, 4, X, 100, X, 100) == bad and call(X, None, 4, None, 100, X, 100) == bad and call(X, None, 4, X, 100, None, 100) == bad
    assert call(X + 8, None, 4, X, 100, X, 100) == bad and call(X, None, 4, X + 2, 100, X, 100) == bad and call(X, None, 4, X, 100, X + 2, 100) == bad
    assert L.a3_lm_head(None, X, None, 4, X, 100, X, 100, None) == bad
    assert L.a3_lm_head(C.byref(_layout(hidden=4096 + 32)), X, None, 4, X, 100, X, 100, None) == api.A3_ERR_UNSUPPORTED
    assert L.a3_lm_head(C.byref(_layout(total_tokens=1 << 20)), X, None, 4, X, 100, X, 100, None) == api.A3_ERR_UNSUPPORTED


def test_logprobs_refuses():
    L = api.lib()
    bad, need = api.A3_ERR_INVALID_ARG, L.a3_token_logprobs_ws_bytes(4, 1000, 20)
    call = lambda dtype=api.A3_F32, x=X, n=4, V=1000, ld=1000, tok=X, given=2, top=20, lp=X, ent=X, idx=X, tl=X, ws=X, size=need: \
        L.a3_token_logprobs(dtype, x, n, V, ld, tok, given, top, lp, ent, idx, tl, ws, size, None)
    assert need > 0 and L.a3_token_logprobs_ws_bytes(-1, 10, 1) == 0 and L.a3_token_logprobs_ws_bytes(1, 0, 1) == 0 \
        and L.a3_token_logprobs_ws_bytes(1, 10, -1) == 0
    assert call(n=0) == api.A3_OK
    assert call(dtype=3) == bad and call(n=-1) == bad and call(V=0) == bad and call(ld=999) == bad
    assert call(given=-1) == bad and call(top=-1) == bad and call(V=10, ld=10, top=11) == bad and call(top=65) == api.A3_ERR_UNSUPPORTED
    assert call(x=None) == bad and call(tok=None) == bad and call(lp=None) == bad and call(idx=None) == bad and call(tl=None) == bad
    assert call(x=X + 2) == bad and call(dtype=api.A3_BF16, x=X + 1) == bad and call(V=1 << 30, ld=1 << 30) == api.A3_ERR_UNSUPPORTED
    assert call(ws=None) == api.A3_ERR_WORKSPACE and call(size=need - 1) == api.A3_ERR_WORKSPACE and call(ws=X + 8) == api.A3_ERR_WORKSPACE


def test_binding_refuses_tensors_on_another_device():
    """CPU tensors never reach the library."""
    out = object.__new__(api.TokenLogprobs)
    out.n_given, out.n_top, out.entropy = 0, 0, torch.zeros(2)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        api.a3_token_logprobs(torch.zeros(2, 10), None, out)
    with pytest.raises(ValueError):
        api.a3_token_logprobs(torch.zeros(2, 10, dtype=torch.float16), None, out)
    with pytest.raises(ValueError):
        api.a3_token_logprobs(torch.zeros(10, 2).t(), None, out)


@pytest.mark.parametrize("vocab", [501, 8200, 32003, 128256])
@pytest.mark.parametrize("n_top", [0, 8, 64])
def test_a_workspace_of_log_probabilities_serves_fewer_rows(vocab, n_top):
    """What is allocated for n rows has to do for every smaller number of them (few rows are cut into slices, many are not)."""
    size = api.lib().a3_token_logprobs_ws_bytes
    sizes = [size(n, vocab, n_top) for n in (*range(0, 2100), 5000, 100000, 2 ** 31 - 1)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0
    assert sizes[-1] <= 2 << 20
