"""Cases of the operators that generate text on a fused cache: appending to a paged K/V cache, attention of one new token
over it, the product with the vocabulary's weights, and log probabilities.

Kinds of case, one pass each:
  append    rows of K and V into their pages, keys (and queries) turned to their positions on the way
  import    a whole prompt's fused caches into pages: keys stand at their positions already
  attend    one query token per request over the request's pages
  step      append, then attend: what every layer of a decoding step does
  logits    hidden rows times the vocabulary's weights
  logprobs  log probabilities of given tokens, entropy and the best alternatives of rows of logits
  score     logits, then log probabilities: what rates given answers

A pool of pages is [pages, KV heads, page size, head size]; an 8-bit page of one KV head is its codes (int8) followed by one
float scale per token.  Pages of a request lie anywhere in the pool, in the order of a serving program that has run for a
while (a random permutation); table entries behind a request's last page are -1.

Values: K, V and queries with the standard deviation that a projection of N(0, 1) hidden states through N(0, 0.02^2) weights
gives them; hidden states N(0, 1); logits N(0, 2^2) with a few tokens per row well ahead, as a trained model's are.
"""
import math
import random

import numpy as np
import torch

own = False

#                 type, query heads, KV heads, head size, hidden, vocabulary, rotary base
SHAPES = {"tiny": ("f32", 8, 8, 64, 512, 4099, 1e4),
          "llama3-8b": ("bf16", 32, 8, 128, 4096, 128256, 5e5),
          "qwen2.5-7b": ("bf16", 28, 4, 128, 3584, 152064, 1e6)}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PAGE = 64


def _cache(name, kind, shape, requests, len_lo, len_hi, q8=False, half=True, page=PAGE):
    """requests: of len_lo .. len_hi tokens each, the new one included."""
    return dict(name=name, kind=kind, shape=shape, requests=requests, len_lo=len_lo, len_hi=len_hi, q8=q8, half=half, page=page,
                lens=1)


def _vocab(name, kind, shape, rows, vocab, dtype, given=1, top=0):
    return dict(name=name, kind=kind, shape=shape, rows=rows, vocab=vocab, dtype=dtype, given=given, top=top)


def listed():
    return [
        # one request's new token in one layer: all launch latency
        _cache("append_1", "append", "llama3-8b", 1, 5100, 5100),
        # the fused caches of a 16K prompt (32 chunks of 512 tokens and a question of 64) into pages
        _cache("import_16k", "import", "llama3-8b", 1, 16448, 16448),
        # the fp32 configuration: three requests, one of a single token
        _cache("attend_f32_short", "attend", "tiny", 3, 1, 545, half=False),
        # one user, the 16K prompt: the whole chip on one token
        _cache("attend_1x16k", "attend", "llama3-8b", 1, 16449, 16449),
        # a serving batch of ragged requests, seven query heads per KV head
        _cache("attend_48_ragged", "attend", "qwen2.5-7b", 48, 100, 8000),
        # long contexts
        _cache("attend_8x64k", "attend", "llama3-8b", 8, 65536, 65600, half=False),
        # a layer of a decoding step on 8-bit pages, ten retrieved chunks per request
        _cache("step_32_q8", "step", "llama3-8b", 32, 4000, 5400, q8=True),
        # the next token's logits for four users: a stream over the weights
        _vocab("logits_4", "logits", "llama3-8b", 4, 128256, "bf16"),
        # logits of a 512-token chunk: a matrix product
        _vocab("logits_512", "logits", "llama3-8b", 512, 128256, "bf16"),
        # one row of logits, twenty alternatives
        _vocab("logprobs_1", "logprobs", "llama3-8b", 1, 128256, "f32", top=20),
        # many rows of an odd length, three given tokens each
        _vocab("logprobs_1500_odd", "logprobs", "qwen2.5-7b", 1500, 32003, "bf16", given=3, top=8),
        # rating 64 answer tokens
        _vocab("score_64", "score", "qwen2.5-7b", 64, 152064, "bf16"),
    ]


def draw(rng):
    """One more case of the ranges above: sizes spread over their logarithm, odd ones among them."""
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choices(["append", "import", "attend", "step", "logits", "logprobs", "score"], [2, 1, 5, 2, 2, 3, 1])[0]
    shape = rng.choice(["tiny", "llama3-8b", "llama3-8b", "qwen2.5-7b", "qwen2.5-7b"])
    if kind in ("append", "import", "attend", "step"):
        tokens = log_int(20, 200000 if kind != "import" else 16448)     # of all requests, about
        requests = min(log_int(1, 128 if kind != "import" else 4), max(1, tokens // 2))
        hi = max(1, 2 * tokens // requests)
        lo = rng.randint(1, hi)
        return dict(kind=kind, shape=shape, requests=requests, len_lo=lo, len_hi=hi, q8=rng.random() < 0.3,
                    half=rng.random() < 0.7, page=rng.choice([32, 64, 64, 64, 128]), lens=rng.randrange(1, 1 << 20))
    vocab = rng.choice([SHAPES[shape][5], log_int(1000, 152064)])
    if kind == "logprobs":
        return dict(kind=kind, shape=shape, rows=log_int(1, max(1, 48000000 // vocab)), vocab=vocab, dtype=rng.choice(["f32", "bf16"]),
                    given=rng.randint(1, 4), top=rng.choice([0, 1, 5, 20]))
    return dict(kind=kind, shape=shape, rows=log_int(1, 512 if kind == "logits" else 128), vocab=vocab, dtype=SHAPES[shape][0],
                given=rng.randint(1, 4), top=0)


def _lens(case):
    """Tokens of every request, the new one included: the same for every seed.  A batch of several has one of the fewest."""
    r = random.Random(case["lens"])
    n = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["requests"])]
    if len(n) > 2:
        n[1] = case["len_lo"]
    return n


class State:
    pass


def prepare(case, seed):
    st = State()
    st.case, st.kind = case, case["kind"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    type_, hq, hkv, d, h, _, base = SHAPES[case["shape"]]
    dt = DTYPES[type_]
    normal = lambda *s, std=1.0, dtype=dt: torch.randn(*s, device="cuda", generator=g, dtype=dtype) * std
    if case["kind"] in ("append", "import", "attend", "step"):
        std, page, lens = 0.02 * math.sqrt(h), case["page"], _lens(case)
        used = [-(-n // page) for n in lens]
        st.n_pages, st.max_pages = sum(used) + 3, max(used) + 1
        order = torch.randperm(st.n_pages, device="cuda", generator=g).to(torch.int32)
        st.table = torch.full((len(lens), st.max_pages), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r, n in enumerate(used):
            st.table[r, :n] = order[at:at + n]
            at += n
        if case["q8"]:
            pools = []
            for _ in range(2):
                pool = torch.empty((st.n_pages, hkv, page * (d + 4)), dtype=torch.int8, device="cuda")
                code, scale = _q8_parts(pool, page, d)
                code.copy_(torch.randint(-127, 128, code.shape, device="cuda", generator=g, dtype=torch.int8))
                scale.copy_((std / 73) * (1 + 0.2 * torch.rand(scale.shape, device="cuda", generator=g)))
                pools.append(pool)
            st.k_pool, st.v_pool = pools
        else:
            st.k_pool, st.v_pool = (normal(st.n_pages, hkv, page, d, std=std) for _ in range(2))
        i32 = lambda v: torch.as_tensor(np.asarray(v, dtype=np.int32), device="cuda")
        st.req = st.pos = st.q = None
        if case["kind"] == "import":
            st.req = i32(np.repeat(np.arange(len(lens)), lens))
            st.slot = i32(np.concatenate([np.arange(n) for n in lens]))
            st.n = int(sum(lens))
        else:
            st.slot = i32([n - 1 for n in lens])
            st.pos, st.len, st.n = st.slot, i32(lens), len(lens)
            st.q = normal(st.n, hq, d, std=std)
        st.k, st.v = (normal(st.n, hkv, d, std=std) for _ in range(2))
        p = torch.arange(max(lens), dtype=torch.float64, device="cuda")
        angle = p[:, None] * base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
        st.cs = torch.stack([angle.cos(), angle.sin()], -1).float()      # [positions, d / 2, (cos, sin)]
        st.half, st.q8, st.page, st.hq, st.hkv, st.d, st.dt = case["half"], case["q8"], page, hq, hkv, d, dt
        if own:
            from paper_2511_17560_amd import api
            st.pages = api.Pages(dtype=type_, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=st.n_pages,
                                 page_table=st.table, q8=case["q8"], rope_base=base, n_pos=max(lens), rope_cs=st.cs,
                                 rope_layout=api.A3_ROPE_HALF if case["half"] else api.A3_ROPE_INTERLEAVED,
                                 k_pool=st.k_pool, v_pool=st.v_pool)
            if st.q is not None:
                st.q_out, st.out = torch.empty_like(st.q), torch.empty_like(st.q)
                st.ws = st.pages.workspace(st.n)
        return st
    rows, vocab, given = case["rows"], case["vocab"], case["given"]
    st.tokens = torch.randint(0, vocab, (rows, given), device="cuda", generator=g, dtype=torch.int32)
    if case["kind"] == "logprobs":
        st.logits = normal(rows, vocab, std=2.0, dtype=DTYPES[case["dtype"]])
        ahead = torch.randint(0, vocab, (rows, 8), device="cuda", generator=g)
        st.logits[torch.arange(rows, device="cuda")[:, None], ahead] += 6.0
        st.tokens[:, 0] = ahead[:, 0]
    else:
        st.x, st.w = normal(rows, h), normal(vocab, h, std=0.02)
    if own:
        from paper_2511_17560_amd import api
        if case["kind"] != "logprobs":       # the layout of a decoding batch: one row per request
            st.layout = api.Layout.decode(dtype=type_, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, hidden=h, rope_base=base, n_req=rows)
            st.logits = torch.empty((rows, vocab), dtype=torch.float32, device="cuda")
        st.probs = api.TokenLogprobs(rows, vocab, given, case["top"])
    return st


# ---- plain forms ----------------------------------------------------------------------------------------------

def _q8_parts(pool, page, d):
    """Codes [pages, heads, page, d] and scales [pages, heads, page] of a pool of 8-bit pages."""
    return pool[..., :page * d].view(*pool.shape[:2], page, d), pool[..., page * d:].view(torch.float32)


def _turn(st, x):
    """x [rows, heads, d] turned to the rows' positions, in x's precision."""
    c, s = (t[:, None].to(x.dtype) for t in st.cs[st.pos.long()].unbind(-1))
    a, b = x.chunk(2, -1) if st.half else (x[..., 0::2], x[..., 1::2])
    y = a * c - b * s, a * s + b * c
    return torch.cat(y, -1) if st.half else torch.stack(y, -1).flatten(-2)


def _append(st):
    # 8-bit pages: whether a quotient rounds up or down is decided in 64 bits
    x = st.k.double() if st.q8 else st.k.float()
    k, v = (_turn(st, x) if st.pos is not None else x), st.v.to(x.dtype)
    req = st.req.long() if st.req is not None else torch.arange(st.n, device="cuda")
    page, at = st.table[req, (st.slot // st.page).long()].long(), (st.slot % st.page).long()
    for x, pool in ((k, st.k_pool), (v, st.v_pool)):
        if st.q8:
            code, scale = _q8_parts(pool, st.page, st.d)
            s = (x.abs().amax(-1) / 127).float()
            code[page, :, at] = torch.where(s[..., None] > 0, torch.round(x / s.double()[..., None]), 0).to(torch.int8)
            scale[page, :, at] = s
        else:
            pool[page, :, at] = x.to(st.dt)
    return _turn(st, st.q.float()).to(st.dt) if st.q is not None else None


def _rows(st, pool):
    """The cache rows of every request in 32 bits, [requests, heads, longest, d] (behind a request's end: anything)."""
    n = int(st.case["len_hi"])
    t = st.table[:, :-(-n // st.page)].long().clamp(min=0)
    if st.q8:
        code, scale = _q8_parts(pool, st.page, st.d)
        x = code[t].float() * scale[t][..., None]
    else:
        x = pool[t].float()
    return x.transpose(1, 2).flatten(2, 3)


def _attend(st, q):
    k = _rows(st, st.k_pool)
    q = q.float().view(st.n, st.hkv, st.hq // st.hkv, st.d)
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(st.d)
    seen = torch.arange(s.shape[-1], device="cuda") < st.len[:, None]
    s = s.masked_fill(~seen[:, None, None], float("-inf"))
    e = (s - s.amax(-1, keepdim=True)).exp()
    o = torch.matmul(e, _rows(st, st.v_pool)) / e.sum(-1, keepdim=True)
    return o.reshape(st.n, st.hq, st.d).to(st.dt)


def _logprobs(st, x):
    x = x.float()
    m = x.amax(-1, keepdim=True)
    e = (x - m).exp()
    z = e.sum(-1, keepdim=True)
    res = dict(logprob=x.gather(1, st.tokens.long()) - m - z.log(), entropy=(z.log() - (e * (x - m)).sum(-1, keepdim=True) / z)[:, 0])
    if st.case["top"]:
        # the largest values, ties to the lowest index: one whole number holds both
        bits = (x + 0.0).view(torch.int32).long()
        key = (torch.where(bits < 0, -(bits & 0x7fffffff), bits) << 32) - torch.arange(x.shape[1], device="cuda")
        idx = -key.topk(st.case["top"], -1).values & 0xffffffff
        res.update(top_idx=idx.int(), top_logprob=x.gather(1, idx) - m - z.log())
    return res


def _written(st):
    """What the cache now holds at the rows just written (8-bit pages: the values that the codes stand for)."""
    req = st.req.long() if st.req is not None else torch.arange(st.n, device="cuda")
    page, at = st.table[req, (st.slot // st.page).long()].long(), (st.slot % st.page).long()
    parts = [_q8_parts(p, st.page, st.d) for p in (st.k_pool, st.v_pool)]
    return [code[page, :, at].float() * scale[page, :, at][..., None] for code, scale in parts]


def run(st):
    if st.kind in ("append", "import", "attend", "step"):
        q, out, res = st.q, None, {}
        if st.kind != "attend":
            if own:
                from paper_2511_17560_amd import api
                api.a3_paged_append(st.pages, st.k, st.v, st.req, st.slot, st.pos, st.n, q=st.q, q_out=st.q_out if st.q is not None else None)
                q = st.q_out if st.q is not None else None
            else:
                q = _append(st)
            if st.q8:
                res["k"], res["v"] = _written(st)
            else:
                res["k"], res["v"] = st.k_pool, st.v_pool
            if q is not None:
                res["q"] = q
        if st.kind in ("attend", "step"):
            if own:
                from paper_2511_17560_amd import api
                api.a3_paged_attention(st.pages, q, None, st.len, st.n, st.out, st.ws)
                res["out"] = st.out
            else:
                res["out"] = _attend(st, q)
        return res
    if not own:
        logits = st.logits if st.kind == "logprobs" else torch.matmul(st.x.float(), st.w.float().t())
        return logits if st.kind == "logits" else _logprobs(st, logits)
    from paper_2511_17560_amd import api
    if st.kind != "logprobs":
        api.a3_lm_head(st.layout, st.x, None, st.case["rows"], st.w, st.logits)
        if st.kind == "logits":
            return st.logits
    r = api.a3_token_logprobs(st.logits, st.tokens, st.probs)
    res = dict(logprob=r.logprob, entropy=r.entropy)
    if st.case["top"]:
        res.update(top_idx=r.top_idx, top_logprob=r.top_logprob)
    return res


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    st = prepare(case, seed)
    own = was
    f64 = torch.float64
    if case["kind"] in ("append", "import", "attend", "step"):
        d, page = st.d, st.page
        res, q = {}, None if st.q is None else st.q.to(f64)
        slot = st.slot.tolist()
        req = st.req.tolist() if st.req is not None else list(range(st.n))
        table = st.table.cpu().numpy()
        where = [torch.as_tensor(np.asarray(v), device="cuda") for v in
                 ([int(table[r, s // page]) for r, s in zip(req, slot)], [s % page for s in slot])]
        k_pool, v_pool = st.k_pool, st.v_pool
        if case["kind"] != "attend":
            k, v = st.k.to(f64), st.v.to(f64)
            if st.pos is not None:
                z = torch.view_as_complex(st.cs.to(f64).contiguous())[st.pos.long()][:, None]      # cos + i sin

                def turned(x):
                    pair = x.unflatten(-1, (2, d // 2)).transpose(-1, -2) if st.half else x.unflatten(-1, (d // 2, 2))
                    y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
                    return (y.transpose(-1, -2) if st.half else y).flatten(-2)

                k, q = turned(k), turned(q)
                res["q"] = q
            if st.q8:
                held = []
                for x, pool in ((k, k_pool), (v, v_pool)):
                    s = (x.abs().amax(-1, keepdim=True) / 127).float().to(f64)
                    c = (x / s).nan_to_num(0).round()
                    held.append(c * s)
                    body, scales = pool[..., :page * d].view(*pool.shape[:2], page, d), pool[..., page * d:].view(torch.float32)
                    body[where[0], :, where[1]] = c.to(torch.int8)
                    scales[where[0], :, where[1]] = s[..., 0].float()
                res["k"], res["v"] = held
            else:
                pools = [p.to(f64) for p in (k_pool, v_pool)]
                for p, x in zip(pools, (k, v)):
                    p[where[0], :, where[1]] = x
                res["k"], res["v"] = pools
                k_pool, v_pool = pools
            if q is not None and case["kind"] == "step":
                q = q.to(st.dt).to(f64)              # the queries and keys that the attention gets are the stored ones
                if not st.q8:
                    k_pool, v_pool = (p.to(st.dt) for p in (k_pool, v_pool))
        if case["kind"] in ("attend", "step"):
            outs = []
            for r, n in enumerate(_lens(case)):
                ids = torch.as_tensor(table[r, :-(-n // page)].astype(np.int64), device="cuda")
                both = []
                for pool in (k_pool, v_pool):
                    if st.q8:
                        x = pool[ids][..., :page * d].unflatten(-1, (page, d)).to(f64)
                        x = x * pool[ids][..., page * d:].contiguous().view(torch.float32).to(f64)[..., None]
                    else:
                        x = pool[ids].to(f64)
                    both.append(x.permute(1, 0, 2, 3).reshape(st.hkv, -1, d)[:, :n])
                w = torch.softmax(torch.bmm(q[r].view(st.hkv, -1, d), both[0].transpose(1, 2).contiguous()) * d ** -0.5, -1)
                outs.append(torch.bmm(w, both[1]).reshape(st.hq, d))
            res["out"] = torch.stack(outs)
        return res
    if case["kind"] == "logprobs":
        x = st.logits.to(f64)
    else:
        x = torch.cat([torch.mm(st.x.to(f64), w.to(f64).t()) for w in st.w.split(16384)], 1)
        if case["kind"] == "logits":
            return x
    lp = torch.log_softmax(x, -1)
    res = dict(logprob=torch.take_along_dim(lp, st.tokens.long(), 1), entropy=-(lp.exp() * lp).sum(-1))
    if case["top"]:
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :case["top"]]
        res.update(top_idx=order.int(), top_logprob=torch.take_along_dim(lp, order, 1))
    return res


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    """Inputs read once, outputs written once; multiply-adds count two."""
    type_, hq, hkv, d, h, _, _ = SHAPES[case["shape"]]
    e = {"f32": 4, "bf16": 2}[type_]
    if case["kind"] in ("append", "import", "attend", "step"):
        lens = _lens(case)
        rows, tokens = (sum(lens) if case["kind"] == "import" else len(lens)), float(sum(lens))
        held = hkv * (d + 4.0 if case["q8"] else d * e)                # one token of one cache, bytes
        w = dict(bytes=0.0, flops=0.0)
        if case["kind"] != "attend":
            w["bytes"] += rows * 2.0 * (hkv * d * e + held)
            if case["kind"] != "import":
                w["bytes"] += rows * (2.0 * hq * d * e + 4.0 * d)
                w["flops"] += rows * 3.0 * (hq + hkv) * d
        if case["kind"] in ("attend", "step"):
            w["bytes"] += tokens * 2.0 * held + rows * 2.0 * hq * d * e
            w["flops"] += 4.0 * tokens * hq * d
        return w
    rows, vocab = float(case["rows"]), float(case["vocab"])
    outs = rows * (case["given"] * 8.0 + 4.0 + case["top"] * 8.0)
    if case["kind"] == "logprobs":
        return dict(bytes=rows * vocab * {"f32": 4, "bf16": 2}[case["dtype"]] + outs, flops=6.0 * rows * vocab)
    w = dict(bytes=(vocab + rows) * h * e + rows * vocab * 4, flops=2.0 * rows * vocab * h)
    if case["kind"] == "score":        # logits and what is read of them need not leave the chip
        w["bytes"] += outs - rows * vocab * 4
        w["flops"] += 6.0 * rows * vocab
    return w
