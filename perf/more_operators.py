"""Cases of the operators that follow several candidates of one request at once over the paged K/V cache: drafted tokens that a
model verifies as a tree, and beams.

Kinds of case, one pass each:
  tree    attention of every request's drafted tokens: each sees the request's whole cache and its own ancestors among the drafted
  verify  append the drafted tokens' K and V, keys and queries turned to their positions, then their attention
  accept  from logits of the drafted tokens to the accepted path: the best token behind every one of them, followed from the root
  move    token rows of all layers' caches to other slots or requests: the accepted path's to the front (of a tree), a
          surviving beam's newest to the beams that go on from it (of beams)
  beam    the best continuations over all beams of a request and the whole vocabulary

A drafted tree of n tokens stands in the n slots behind the request's committed tokens, parents in front of their children; row 0 is
its root, the last token that is certain.  mask[row, w] has bit b set where the row sees the tree's token 32 w + b; a chain, where
every row sees those in front of it and itself, needs none.  Pools, pages and 8-bit pages are as in perf/operators.py.

Values: K, V and queries with the standard deviation that a projection of N(0, 1) hidden states through N(0, 0.02^2) weights
gives them; logits N(0, 2^2) with a few tokens per row well ahead, as a trained model's are; along each tree one path whose tokens the
model picks too, as far as such paths go in earnest.
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


def _tree(name, kind, shape, requests, len_lo, len_hi, rows_lo, rows_hi, chain=False, q8=False, half=True, page=PAGE):
    """requests: of len_lo .. len_hi committed tokens and rows_lo .. rows_hi drafted ones each."""
    return dict(name=name, kind=kind, shape=shape, requests=requests, len_lo=len_lo, len_hi=len_hi, rows_lo=rows_lo, rows_hi=rows_hi,
                chain=chain, q8=q8, half=half, page=page, plan=1)


def _accept(name, requests, rows_lo, rows_hi, vocab, dtype):
    return dict(name=name, kind="accept", requests=requests, rows_lo=rows_lo, rows_hi=rows_hi, vocab=vocab, dtype=dtype, plan=1)


def _move(name, shape, layers, requests, beams, len_lo, len_hi, page=PAGE):
    """beams 0: trees of 24 drafted tokens behind len_lo .. len_hi committed ones; else len_lo .. len_hi newest tokens of each of them."""
    return dict(name=name, kind="move", shape=shape, layers=layers, requests=requests, beams=beams, len_lo=len_lo, len_hi=len_hi,
                page=page, plan=1)


def _beam(name, requests, beams, vocab, dtype, best, done):
    return dict(name=name, kind="beam", requests=requests, beams=beams, vocab=vocab, dtype=dtype, best=best, done=done)


def listed():
    return [
        # the fp32 configuration: three requests, one of them new
        _tree("tree_f32_short", "tree", "tiny", 3, 0, 540, 1, 5, half=False),
        # one user, the 16K prompt, a tree of 16
        _tree("tree_1x16k", "tree", "llama3-8b", 1, 16448, 16448, 16, 16),
        # a serving batch of ragged requests, a few tokens copied from the prompt drafted behind each: a chain, seven query heads per KV head
        _tree("verify_48_chain", "verify", "qwen2.5-7b", 48, 100, 8000, 1, 6, chain=True),
        # wide trees: the work goes from memory to the matrix pipe
        _tree("tree_8x8k_64", "tree", "llama3-8b", 8, 7000, 8200, 64, 64),
        # long contexts
        _tree("tree_4x64k", "tree", "llama3-8b", 4, 65500, 65600, 24, 32, half=False),
        # 8-bit pages, ten retrieved chunks per request
        _tree("tree_32_q8", "tree", "llama3-8b", 32, 4000, 5400, 8, 13, q8=True),
        # one user's tree
        _accept("accept_1", 1, 16, 16, 128256, "f32"),
        # many of them, an odd vocabulary
        _accept("accept_48_odd", 48, 4, 12, 32003, "bf16"),
        # all layers of a model after a verification
        _move("move_tree", "llama3-8b", 32, 8, 0, 100, 500),
        # all layers, eight requests of four beams, some hundred tokens generated
        _move("move_beams", "llama3-8b", 32, 8, 4, 90, 230),
        # one user's four beams
        _beam("beam_1x4", 1, 4, 128256, "f32", 8, False),
        # many users' eight beams, some of them ended
        _beam("beam_64x8", 64, 8, 152064, "f32", 16, True),
    ]


def draw(rng):
    """One more case of the ranges above: sizes spread over their logarithm, odd ones among them."""
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choices(["tree", "verify", "accept", "move", "beam"], [5, 2, 2, 2, 3])[0]
    plan = rng.randrange(1, 1 << 20)
    if kind in ("tree", "verify"):
        shape = rng.choice(["tiny", "llama3-8b", "llama3-8b", "qwen2.5-7b", "qwen2.5-7b"])
        tokens = log_int(20, 130000)                     # of all requests, about
        requests = min(log_int(1, 64), max(1, tokens // 2))
        hi = max(1, 2 * tokens // requests)
        rows = log_int(1, max(1, min(64, 4000000 // tokens)))
        return dict(kind=kind, shape=shape, requests=requests, len_lo=rng.randint(0, hi), len_hi=hi, rows_lo=rng.randint(1, rows),
                    rows_hi=rows, chain=rng.random() < 0.3, q8=kind == "tree" and rng.random() < 0.3, half=rng.random() < 0.7,
                    page=rng.choice([32, 64, 64, 64, 128]), plan=plan)
    vocab = rng.choice([4099, 32003, 128256, 152064, log_int(1000, 152064)])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "accept":
        requests = log_int(1, 64)
        rows = log_int(1, max(1, min(64, 48000000 // vocab // requests)))
        return dict(kind=kind, requests=requests, rows_lo=rng.randint(1, rows), rows_hi=rows, vocab=vocab, dtype=dtype, plan=plan)
    if kind == "move":
        requests, beams = log_int(1, 8), rng.choice([0, 0, 2, 3, 4, 5])
        hi = log_int(30, 500 if beams == 0 else 230)
        return dict(kind=kind, shape=rng.choice(["tiny", "llama3-8b", "qwen2.5-7b"]), layers=rng.choice([1, 4, 28, 32]), requests=requests,
                    beams=beams, len_lo=rng.randint(1, hi), len_hi=hi, page=rng.choice([32, 64, 64, 64, 128]), plan=plan)
    beams = rng.choice([1, 2, 3, 4, 4, 5, 8, 8, 16])
    return dict(kind=kind, requests=log_int(1, max(1, min(64, 60000000 // vocab // beams))), beams=beams, vocab=vocab, dtype=dtype,
                best=rng.choice([beams, 2 * beams]), done=rng.random() < 0.5)


def _plan(case):
    """What a case's seed leaves alone: [(committed tokens, parents of the drafted ones)] of every request.  One of a batch is as short as any."""
    r, plan = random.Random(case["plan"]), []
    for i in range(case["requests"]):
        n = r.randint(case["len_lo"], case["len_hi"]) if i != 1 or case["requests"] < 3 else case["len_lo"]
        rows = r.randint(case["rows_lo"], case["rows_hi"])
        # a tree grown from the root outwards, about three children a token
        plan.append((n, [-1] + [j - 1 if case["chain"] else r.randint((j - 1) // 3, min(j - 1, (j + 1) // 2)) for j in range(1, rows)]))
    return plan


def _trees(case):
    r = random.Random(case["plan"])
    return [[-1] + [r.randint((j - 1) // 3, min(j - 1, (j + 1) // 2)) for j in range(1, r.randint(case["rows_lo"], case["rows_hi"]))]
            for _ in range(case["requests"])]


def _ancestors(parents):
    seen = np.zeros((len(parents), len(parents)), dtype=bool)
    for j, p in enumerate(parents):
        if p >= 0:
            seen[j] = seen[p]
        seen[j, j] = True
    return seen


def _moves(case):
    """[(source request, first slot, target request, first slot, slots)] of every set of moves."""
    r, sets = random.Random(case["plan"]), []
    for i in range(case["requests"]):
        if case["beams"] == 0:
            n, path = r.randint(case["len_lo"], case["len_hi"]), [0]
            while path[-1] < 20 and len(path) < 6:                   # a path through a tree of 24
                path.append(path[-1] + r.randint(1, 5))
            path = path[:r.randint(1, len(path))]
            sets.append([(i, n + p, i, n + m, 1) for m, p in enumerate(path)])
        else:
            b, n = case["beams"], r.randint(case["len_lo"], case["len_hi"])
            first = PROMPT // case["page"] * case["page"]            # the prompt's full pages are shared
            sets.append([(i * b + r.randrange(b), first, i * b + j, first, PROMPT - first + n) for j in range(b)])
    return sets


PROMPT = 500         # tokens that a request's beams have in common
TREE = 24


class State:
    pass


def _i32(v):
    return torch.as_tensor(np.asarray(v, dtype=np.int32), device="cuda")


def _pools(case, shape, pages, layers, normal, g):
    type_, hq, hkv, d, h, _, _ = SHAPES[shape]
    std, page = 0.02 * math.sqrt(h), case["page"]
    pools = []
    for _ in range(2):
        if not case.get("q8"):
            pools.append(normal(layers * pages, hkv, page, d, std=std, dtype=DTYPES[type_]))
            continue
        pool = torch.empty((layers * pages, hkv, page * (d + 4)), dtype=torch.int8, device="cuda")
        code, scale = _q8_parts(pool, page, d)
        code.copy_(torch.randint(-127, 128, code.shape, device="cuda", generator=g, dtype=torch.int8))
        scale.copy_((std / 73) * (1 + 0.2 * torch.rand(scale.shape, device="cuda", generator=g)))
        pools.append(pool)
    return [p.view(layers, pages, *p.shape[1:]) for p in pools]


def prepare(case, seed):
    st = State()
    st.case, st.kind = case, case["kind"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *s, std=1.0, dtype: torch.randn(*s, device="cuda", generator=g, dtype=dtype) * std
    if case["kind"] in ("tree", "verify"):
        _prepare_tree(st, case, normal, g)
    elif case["kind"] == "move":
        _prepare_move(st, case, normal, g)
    elif case["kind"] == "accept":
        _prepare_accept(st, case, normal, g, random.Random(int(seed)))
    else:
        _prepare_beam(st, case, normal, g)
    return st


def _prepare_tree(st, case, normal, g):
    type_, hq, hkv, d, h, _, base = SHAPES[case["shape"]]
    dt, page, plan = DTYPES[type_], case["page"], _plan(case)
    used = [-(-(n + len(t)) // page) for n, t in plan]
    st.n_pages, max_pages = sum(used) + 3, max(used) + 1
    order = torch.randperm(st.n_pages, device="cuda", generator=g).to(torch.int32)
    st.table = torch.full((len(plan), max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(used):
        st.table[r, :n] = order[at:at + n]
        at += n
    st.k_pool, st.v_pool = (p[0] for p in _pools(case, case["shape"], st.n_pages, 1, normal, g))
    rows = [len(t) for _, t in plan]
    st.n, st.max_rows = sum(rows), max(rows)
    st.start, st.len = _i32(np.concatenate([[0], np.cumsum(rows)])), _i32([n for n, _ in plan])
    st.mask = None
    if not case["chain"]:
        bits = np.zeros((st.n, 32 * -(-st.max_rows // 32)), dtype=np.uint8)
        at = 0
        for _, t in plan:
            bits[at:at + len(t), :len(t)] = _ancestors(t)
            at += len(t)
        st.mask = torch.as_tensor(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy(), device="cuda")
    st.q = normal(st.n, hq, d, std=0.02 * math.sqrt(h), dtype=dt)
    st.half, st.q8, st.page, st.hq, st.hkv, st.d, st.dt = case["half"], case["q8"], page, hq, hkv, d, dt
    if case["kind"] == "verify":
        depth = [_ancestors(t).sum(1) - 1 for _, t in plan]
        st.k, st.v = (normal(st.n, hkv, d, std=0.02 * math.sqrt(h), dtype=dt) for _ in range(2))
        st.req = _i32(np.repeat(np.arange(len(plan)), rows))
        st.slot = _i32(np.concatenate([n + np.arange(len(t)) for n, t in plan]))
        st.pos = _i32(np.concatenate([n + x for (n, _), x in zip(plan, depth)]))
    n_pos = max(n + len(t) for n, t in plan)
    angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * base ** (
        -2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    st.cs = torch.stack([angle.cos(), angle.sin()], -1).float()          # [positions, d / 2, (cos, sin)]
    if own:
        from paper_2511_17560_amd import api
        st.pages = api.Pages(dtype=type_, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=st.n_pages,
                             page_table=st.table, q8=case["q8"], rope_base=base, n_pos=n_pos, rope_cs=st.cs,
                             rope_layout=api.A3_ROPE_HALF if case["half"] else api.A3_ROPE_INTERLEAVED, k_pool=st.k_pool, v_pool=st.v_pool)
        st.q_out, st.out = torch.empty_like(st.q), torch.empty_like(st.q)
        st.ws = st.pages.tree_workspace(len(plan), st.max_rows)


def _prepare_move(st, case, normal, g):
    type_, hq, hkv, d, h, _, base = SHAPES[case["shape"]]
    page, layers, sets = case["page"], case["layers"], _moves(case)
    st.page, st.sets = page, len(sets)
    st.size = max(len(s) for s in sets)
    if case["beams"] == 0:
        lens = [s[0][1] + TREE for s in sets]
        shared = [[]] * len(sets)
    else:                                                                # every beam: its request's prompt, then pages of its own
        lens = [s[0][4] for s in sets for _ in s]
        shared = [[i] * (PROMPT // page) for i in range(len(sets)) for _ in range(case["beams"])]
    mine = [-(-n // page) for n in lens]
    common = (PROMPT // page) * len(sets) if case["beams"] else 0
    n_pages = sum(mine) + common + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu().numpy()
    table, at = np.full((len(lens), max(len(s) + m for s, m in zip(shared, mine)) + 1), -1, dtype=np.int32), common
    for r, (s, m) in enumerate(zip(shared, mine)):
        if s:
            table[r, :len(s)] = order[s[0] * len(s):(s[0] + 1) * len(s)]
        table[r, len(s):len(s) + m] = order[at:at + m]
        at += m
    st.table = torch.as_tensor(table, device="cuda")
    st.k_pool, st.v_pool = _pools(case, case["shape"], n_pages, layers, normal, g)
    none = (-1, -1, -1, -1, 0)                                           # sets may be shorter than the longest
    cols = np.asarray([[s[m] if m < len(s) else none for m in range(st.size)] for s in sets], dtype=np.int32)
    st.src_req, st.src_slot, st.dst_req, st.dst_slot, st.slots = (_i32(cols[..., i]) for i in range(5))
    st.max_slots = int(cols[..., 4].max())
    if own:
        from paper_2511_17560_amd import api
        st.layers = api.PageLayers([
            api.Pages(dtype=type_, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, page_table=st.table,
                      rope_base=base, n_pos=0, k_pool=st.k_pool[i], v_pool=st.v_pool[i]) for i in range(layers)])


def _prepare_accept(st, case, normal, g, rng):
    trees = _trees(case)
    rows, vocab = [len(t) for t in trees], case["vocab"]
    st.n, st.max_rows = sum(rows), max(rows)
    st.start = _i32(np.concatenate([[0], np.cumsum(rows)]))
    st.parent = _i32(np.concatenate(trees))
    st.logits = normal(st.n, vocab, std=2.0, dtype=DTYPES[case["dtype"]])
    tokens, at = np.empty(st.n, dtype=np.int32), 0
    ahead, ahead_of = [], []
    for t in trees:
        # siblings are different tokens; the model agrees with the draft on one child of a token three times in four
        tokens[at:at + len(t)] = (rng.randrange(vocab) + np.arange(len(t)) * (vocab // 67)) % vocab
        for j in range(len(t)):
            children = [c for c in range(j + 1, len(t)) if t[c] == j]
            ahead_of.append(at + j)
            ahead.append(int(tokens[at + rng.choice(children)]) if children and rng.random() < 0.75 else rng.randrange(vocab))
        at += len(t)
    st.logits[torch.as_tensor(ahead_of, device="cuda"), torch.as_tensor(ahead, device="cuda")] += 16.0
    st.tokens = _i32(tokens)
    st.len = _i32([rng.randint(1, 9000) for _ in trees])
    st.max_path = min(st.max_rows, 16)
    if own:
        from paper_2511_17560_amd import api
        st.out = api.TreeAccepted(len(trees), st.n, st.max_path, vocab)


def _prepare_beam(st, case, normal, g):
    n, b, vocab = case["requests"], case["beams"], case["vocab"]
    st.logits = normal(n * b, vocab, std=2.0, dtype=DTYPES[case["dtype"]])
    ahead = torch.randint(0, vocab, (n * b, 8), device="cuda", generator=g)
    st.logits[torch.arange(n * b, device="cuda")[:, None], ahead] += 8.0
    st.score = -20 * torch.rand(n * b, device="cuda", generator=g)
    st.done = (torch.rand(n * b, device="cuda", generator=g) < 0.2).to(torch.int32) if case["done"] else None
    st.end = vocab - 1
    if own:
        from paper_2511_17560_amd import api
        st.out = api.BeamChoice(n, b, vocab, case["best"])


# ---- plain forms ----------------------------------------------------------------------------------------------

def _q8_parts(pool, page, d):
    """Codes [pages, heads, page, d] and scales [pages, heads, page] of a pool of 8-bit pages."""
    return pool[..., :page * d].view(*pool.shape[:2], page, d), pool[..., page * d:].view(torch.float32)


def _turn(st, x):
    """x [rows, heads, d] in 32 bits, turned to the rows' positions."""
    c, s = (t[:, None] for t in st.cs[st.pos.long()].unbind(-1))
    a, b = x.chunk(2, -1) if st.half else (x[..., 0::2], x[..., 1::2])
    y = a * c - b * s, a * s + b * c
    return torch.cat(y, -1) if st.half else torch.stack(y, -1).flatten(-2)


def _append(st):
    page, at = st.table[st.req.long(), (st.slot // st.page).long()].long(), (st.slot % st.page).long()
    st.k_pool[page, :, at] = _turn(st, st.k.float()).to(st.dt)
    st.v_pool[page, :, at] = st.v
    return _turn(st, st.q.float()).to(st.dt)


def _rows(st, pool, n):
    """The first n cache rows of every request in 32 bits, [requests, heads, n and more, d] (behind a request's end: anything)."""
    t = st.table[:, :-(-n // st.page)].long().clamp(min=0)
    if st.q8:
        code, scale = _q8_parts(pool, st.page, st.d)
        x = code[t].float() * scale[t][..., None]
    else:
        x = pool[t].float()
    return x.transpose(1, 2).flatten(2, 3)


def _place(st):
    """Row j of request r among the packed rows, [requests, max_rows], and whether there is one."""
    j = torch.arange(st.max_rows, device="cuda")
    place = st.start[:-1, None].long() + j
    return place.clamp(max=st.n - 1), place < st.start[1:, None]


def _attend(st, q):
    place, there = _place(st)
    n = st.case["len_hi"] + st.case["rows_hi"]
    k = _rows(st, st.k_pool, n)
    gq, slots = st.hq // st.hkv, torch.arange(k.shape[2], device="cuda")
    t = slots[None] - st.len[:, None].long()                                 # [requests, slots]: number among the drafted
    own_rows = (st.start[1:] - st.start[:-1])[:, None]
    if st.mask is None:
        seen = t[:, None] <= torch.arange(st.max_rows, device="cuda")[:, None]
    else:
        bit = t.clamp(0, st.max_rows - 1)[:, None].expand(-1, st.max_rows, -1)
        seen = (st.mask[place].gather(2, bit >> 5) >> (bit & 31)) & 1 > 0
    seen = (t < 0)[:, None] | (seen & (t >= 0)[:, None] & (t < own_rows)[:, None])      # [requests, rows, slots]
    x = q[place].float().view(*place.shape, st.hkv, gq, st.d).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s = torch.matmul(x, k.transpose(-1, -2)) / math.sqrt(st.d)
    s = s.masked_fill(~seen.repeat_interleave(gq, 1)[:, None], float("-inf"))
    e = (s - s.amax(-1, keepdim=True)).exp()
    o = torch.matmul(e, _rows(st, st.v_pool, n)) / e.sum(-1, keepdim=True)
    o = o.unflatten(2, (st.max_rows, gq)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return o[there].to(st.dt)


def _order(x):
    """Larger value, then lower index, as one whole number that is larger."""
    bits = (x.float() + 0.0).view(torch.int32).long()
    return (torch.where(bits < 0, -(bits & 0x7fffffff), bits) << 32) - torch.arange(x.shape[-1], device="cuda")


def _follow(st):
    place, there = _place(st)
    picked = (-_order(st.logits).amax(-1) & 0xffffffff).int()
    parent, rows = st.parent[place].long(), torch.arange(st.max_rows, device="cuda")
    agreed = (st.tokens[place] == picked[place.gather(1, parent.clamp(min=0))]) | (rows == 0)
    # a row is accepted where it and all its ancestors agree: doubling the reach, 64 rows at most
    ok, up = agreed & there, torch.where(parent < 0, rows, parent)
    for _ in range(6):
        ok, up = ok & ok.gather(1, up), up.gather(1, up)
    path = torch.where(ok, rows, st.max_rows).sort(-1).values[:, :st.max_path]
    count = ok.sum(-1).clamp(max=st.max_path)
    path = torch.where(path < st.max_rows, path, -1).int()
    last = path.gather(1, count[:, None] - 1).long()
    m = torch.arange(st.max_path, device="cuda")
    return dict(picked=picked, count=count.int(), path=path, next=picked[place.gather(1, last)[:, 0]],
                src_slot=torch.where(path >= 0, path + st.len[:, None], -1).int(),
                dst_slot=torch.where(path >= 0, m + st.len[:, None], -1).int())


def _moved(st):
    o = torch.arange(st.max_slots, device="cuda")
    on = o < st.slots[..., None]                                             # [sets, moves, slots]

    def where(req, first):
        slot = (first[..., None] + o)[on].long()
        return st.table[req[..., None].expand_as(on)[on].long(), slot // st.page].long(), slot % st.page

    (p, a), (to_p, to_a) = where(st.src_req, st.src_slot), where(st.dst_req, st.dst_slot)
    for pool in (st.k_pool, st.v_pool):
        pool[:, to_p, :, to_a] = pool[:, p, :, a]
    return dict(k=st.k_pool, v=st.v_pool)


def _best(st):
    # sums over the vocabulary and what they decide in 64 bits: continuations of two beams may be that close
    n, b, vocab, best = (st.case[k] for k in ("requests", "beams", "vocab", "best"))
    top = -(-_order(st.logits)).topk(min(best, vocab), -1, largest=False).values     # best first, equal ones by their index
    token = -top & 0xffffffff
    m = st.logits.amax(-1, keepdim=True).double()
    z = (st.logits.double() - m).exp_().sum(-1, keepdim=True)
    total = st.score.double()[:, None] + (st.logits.gather(1, token).double() - m - z.log())
    if st.done is not None:
        first = torch.arange(token.shape[1], device="cuda") == 0
        ended = torch.where(first, st.score.double()[:, None], float("-inf"))
        total = torch.where(st.done[:, None] > 0, ended, total)
        token = torch.where(st.done[:, None] > 0, st.end, token)
    total, at = torch.sort(total.view(n, -1), dim=-1, descending=True, stable=True)
    total, at = total[:, :best], at[:, :best]
    row = torch.arange(n, device="cuda")[:, None] * b + at // token.shape[1]
    none = total == float("-inf")
    return dict(score=total.float(), row=torch.where(none, -1, row).int(), token=torch.where(none, -1, token.view(n, -1).gather(1, at)).int())


def run(st):
    if own:
        from paper_2511_17560_amd import api
    if st.kind in ("tree", "verify"):
        q, res = st.q, {}
        if st.kind == "verify":
            if own:
                api.a3_paged_append(st.pages, st.k, st.v, st.req, st.slot, st.pos, st.n, q=st.q, q_out=st.q_out)
                q = st.q_out
            else:
                q = _append(st)
            res = dict(k=st.k_pool, v=st.v_pool, q=q)
        if own:
            api.a3_tree_attention(st.pages, q, st.start, None, st.len, st.mask, st.n, st.max_rows, st.out, st.ws)
            res["out"] = st.out
        else:
            res["out"] = _attend(st, q)
        return res
    if st.kind == "accept":
        if not own:
            return _follow(st)
        r = api.a3_tree_accept(st.logits, st.tokens, st.parent, st.start, st.len, st.n, st.max_rows, st.out)
        return dict(picked=r.picked, count=r.count, path=r.path, next=r.next_token, src_slot=r.src_slot, dst_slot=r.dst_slot)
    if st.kind == "move":
        if not own:
            return _moved(st)
        api.a3_paged_move(st.layers, st.src_req, st.src_slot, st.dst_req, st.dst_slot, st.slots, st.max_slots, st.sets, st.size)
        return dict(k=st.k_pool, v=st.v_pool)
    if not own:
        return _best(st)
    r = api.a3_beam_select(st.logits, st.score, st.done, st.end, st.out)
    return dict(score=r.score, row=r.row, token=r.token)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    st = prepare(case, seed)
    own = was
    f64 = torch.float64
    if case["kind"] == "move":
        return None                                                          # copies: no computed numbers
    if case["kind"] == "accept":
        logits, tokens, parent, start = st.logits.float().cpu().numpy(), st.tokens.tolist(), st.parent.tolist(), st.start.tolist()
        picked = logits.argmax(1)
        res = dict(picked=picked.astype(np.int32), count=[], path=[], next=[], src_slot=[], dst_slot=[])
        for g, n in enumerate(st.len.tolist()):
            s, path = start[g], [0]
            more = True
            while more and len(path) < st.max_path:
                here = path[-1]
                child = [c for c in range(here + 1, start[g + 1] - s) if parent[s + c] == here and tokens[s + c] == picked[s + here]]
                path += child[:1]
                more = bool(child)
            none = [-1] * (st.max_path - len(path))
            res["count"].append(len(path))
            res["path"].append(path + none)
            res["next"].append(picked[s + path[-1]])
            res["src_slot"].append([n + p for p in path] + none)
            res["dst_slot"].append([n + m for m in range(len(path))] + none)
        return {k: torch.as_tensor(np.asarray(v, dtype=np.int32)) for k, v in res.items()}
    if case["kind"] == "beam":
        n, b, best = case["requests"], case["beams"], case["best"]
        out = [[], [], []]
        for g in range(n):
            lp = st.score[g * b:(g + 1) * b].to(f64)[:, None] + torch.log_softmax(st.logits[g * b:(g + 1) * b].to(f64), -1)
            if st.done is not None:
                ended = torch.full_like(lp, -math.inf)
                ended[:, st.end] = st.score[g * b:(g + 1) * b].to(f64)
                lp = torch.where(st.done[g * b:(g + 1) * b, None].bool(), ended, lp)
            value, at = torch.sort(lp.flatten(), descending=True, stable=True)
            value, at = value[:best], at[:best]
            gone = value.isneginf()
            for o, v in zip(out, (value, (g * b + at // case["vocab"]).masked_fill(gone, -1), (at % case["vocab"]).masked_fill(gone, -1))):
                o.append(v)
        score, row, token = (torch.stack(o) for o in out)
        return dict(score=score, row=row.int(), token=token.int())
    d, page, res, q = st.d, st.page, {}, st.q.to(f64)
    k_pool, v_pool = st.k_pool, st.v_pool
    if case["kind"] == "verify":
        z = torch.view_as_complex(st.cs.to(f64).contiguous())[st.pos.long()][:, None]      # cos + i sin

        def turned(x):
            pair = x.unflatten(-1, (2, d // 2)).transpose(-1, -2) if st.half else x.unflatten(-1, (d // 2, 2))
            y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
            return (y.transpose(-1, -2) if st.half else y).flatten(-2)

        to = st.table[st.req.long(), torch.div(st.slot, page, rounding_mode="floor").long()].long(), torch.remainder(st.slot, page).long()
        res["q"] = turned(q)
        pools = [p.to(f64) for p in (k_pool, v_pool)]
        for p, x in zip(pools, (turned(st.k.to(f64)), st.v.to(f64))):
            p[to[0], :, to[1]] = x
        res["k"], res["v"] = pools
        q, k_pool, v_pool = (x.to(st.dt) for x in (res["q"], *pools))                      # the attention gets the stored ones
    outs, at = [], 0
    for r, (n, t) in enumerate(_plan(case)):
        both, ids = [], st.table[r, :-(-(n + len(t)) // page)].long()
        for pool in (k_pool, v_pool):
            if st.q8:
                x = pool[ids][..., :page * d].unflatten(-1, (page, d)).to(f64)
                x = x * pool[ids][..., page * d:].contiguous().view(torch.float32).to(f64)[..., None]
            else:
                x = pool[ids].to(f64)
            both.append(x.permute(1, 0, 2, 3).reshape(st.hkv, -1, d)[:, :n + len(t)])
        hidden = torch.zeros((len(t), 1, n + len(t)), dtype=torch.bool, device="cuda")
        hidden[:, 0, n:] = torch.as_tensor(~_ancestors(t), device="cuda")
        x = q[at:at + len(t)].to(f64).view(len(t), st.hkv, -1, d)
        for h in range(st.hkv):
            s = torch.matmul(x[:, h].flatten(0, 1), both[0][h].t().contiguous()).view(len(t), -1, n + len(t)) * d ** -0.5
            w = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
            outs.append(torch.matmul(w.flatten(0, 1), both[1][h]).view(len(t), -1, d))
        outs[-st.hkv:] = [torch.stack(outs[-st.hkv:], 1).flatten(1, 2)]
        at += len(t)
    res["out"] = torch.cat(outs)
    return res


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    """Inputs read once, outputs written once; multiply-adds count two."""
    if case["kind"] == "accept":
        rows, requests = float(sum(len(t) for t in _trees(case))), float(case["requests"])
        return dict(bytes=rows * (case["vocab"] * {"f32": 4.0, "bf16": 2.0}[case["dtype"]] + 12) + requests * (16 + 12 * 16), flops=rows * case["vocab"])
    if case["kind"] == "beam":
        rows = float(case["requests"] * case["beams"])
        return dict(bytes=rows * (case["vocab"] * {"f32": 4.0, "bf16": 2.0}[case["dtype"]] + 8) + case["requests"] * case["best"] * 12.0,
                    flops=5.0 * rows * case["vocab"])
    type_, hq, hkv, d, _, _, _ = SHAPES[case["shape"]]
    e = {"f32": 4, "bf16": 2}[type_]
    if case["kind"] == "move":
        rows = sum(n for s in _moves(case) for a, i, b, j, n in s if (a, i) != (b, j))       # (what stays where it is need not be read)
        return dict(bytes=4.0 * rows * case["layers"] * hkv * d * e + 20.0 * case["requests"], flops=0.0)
    held = hkv * (d + 4.0 if case["q8"] else d * e)                # one token of one cache, bytes
    plan = _plan(case)
    rows = float(sum(len(t) for _, t in plan))
    w = dict(bytes=sum(n + len(t) for n, t in plan) * 2.0 * held + rows * 2.0 * hq * d * e,
             flops=sum(4.0 * hq * d * (n * len(t) + int(_ancestors(t).sum())) for n, t in plan))
    if case["kind"] == "verify":
        w["bytes"] += rows * (2.0 * (hkv * d * e + held) + 2.0 * hq * d * e + 4.0 * d)
        w["flops"] += rows * 3.0 * (hq + hkv) * d
    return w
