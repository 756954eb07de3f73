"""A paged cache for the tests: logical caches of requests spread over a shuffled pool, and read back from it."""
import numpy as np
import torch

from oracle import q8_oracle as q8
from paper_2511_17560_amd import api

STORAGE = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_pages(lens, *, dtype="bf16", Hq=8, Hkv=2, d=128, page=64, q8=False, base=1e4, layout=0, n_pos=None, seed=0, spare=2, fill=None,
               sm_scale=0.0, slack=1):
    """Pages for requests of up to lens[r] slots each, in a random order.  Pools are filled with ``fill`` (default: NaN, or code
    77 with scale NaN: what lies behind a request's end must not matter)."""
    rng = np.random.default_rng(seed)
    need = [-(-max(int(n), 0) // page) for n in lens]
    n_pages, width = sum(need) + spare, max(need + [0]) + slack
    order = rng.permutation(n_pages)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    p = api.Pages(dtype=dtype, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, page_size=page, n_pages=n_pages,
                  page_table=torch.from_numpy(table).cuda(), rope_base=base, rope_layout=layout, q8=q8, sm_scale=sm_scale,
                  n_pos=max(max(lens), 1) if n_pos is None else n_pos)
    for pool in (p.k_pool, p.v_pool):
        if q8:
            codes, scales = parts(p, pool)
            codes.fill_(77)
            scales.fill_(float("nan") if fill is None else fill)
        else:
            pool.fill_(float("nan") if fill is None else fill)
    return p


def parts(p, pool):
    """Codes [pages, heads, page, d] and scales [pages, heads, page] of a pool of 8-bit pages."""
    s = p.struct
    return (pool[..., :s.page_size * s.head_dim].view(s.n_pages, s.n_kv_heads, s.page_size, s.head_dim),
            pool[..., s.page_size * s.head_dim:].view(torch.float32))


def put(p, r, first, k, v):
    """Slots first .. of request r hold k, v [n, Hkv, d] (float64 arrays) exactly as stored; what they stand for then."""
    s, table = p.struct, p.page_table.cpu().numpy()
    slots = np.arange(first, first + len(k))
    page, at = torch.from_numpy(table[r, slots // s.page_size].astype(np.int64)).cuda(), torch.from_numpy(slots % s.page_size).cuda()
    held = []
    for x, pool in ((k, p.k_pool), (v, p.v_pool)):
        if p.q8:
            code, scale = q8.quantize_q8(x)
            codes, scales = parts(p, pool)
            codes[page, :, at] = torch.from_numpy(code).cuda()
            scales[page, :, at] = torch.from_numpy(scale).cuda()
            held.append(q8.dequantize_q8(code, scale))
        else:
            t = torch.from_numpy(np.asarray(x)).to(STORAGE[p.dtype])
            pool[page, :, at] = t.cuda()
            held.append(t.double().numpy())
    return held


def get(p, r, first, end):
    """What slots first .. end - 1 of request r stand for: k, v [n, Hkv, d] float64 arrays."""
    s, table = p.struct, p.page_table.cpu().numpy()
    slots = np.arange(first, end)
    page, at = torch.from_numpy(table[r, slots // s.page_size].astype(np.int64)).cuda(), torch.from_numpy(slots % s.page_size).cuda()
    out = []
    for pool in (p.k_pool, p.v_pool):
        if p.q8:
            codes, scales = parts(p, pool)
            out.append((codes[page, :, at].double() * scales[page, :, at].double()[..., None]).cpu().numpy())
        else:
            out.append(pool[page, :, at].double().cpu().numpy())
    return out
