"""Several candidates as a run: prompt -> pages -> verified trees -> more tokens; beams over shared and own pages.

Tolerances: those of the stack's tests for the same number of blocks (tests/test_gpu_generate.py): fp32 1e-4, bf16 2e-2 of the tensor's
largest value."""
import numpy as np
import pytest
import torch

from oracle import candidates_oracle as cand
from oracle import generate_oracle as gen
from oracle import stack_oracle as st
import a3_synth as synth
from paper_2511_17560_amd import api, stack
from gpu_util import idev, max_abs_rel, to_dev, to_host
from paged_util import get, make_pages

pytestmark = pytest.mark.gpu

SHAPES = {"f32": synth.ModelShape("cand-f32", "f32", 256, 8, 2, 64, 1e4, synth.ROPE_INTERLEAVED, ffn=384),
          "bf16": synth.ModelShape("cand-bf16", "bf16", 512, 8, 2, 128, 5e5, synth.ROPE_HALF, ffn=768)}
VOCAB, N_LAYERS = 97, 3


class Model:
    """Weights, a table of embeddings and the vocabulary's, and the float64 oracle of whole texts."""

    def __init__(self, dtype, lens, seed=3):
        self.dtype, self.shape = dtype, SHAPES[dtype]
        rng = np.random.default_rng(seed)
        self.w = synth.custom(self.shape, [[n - 4] if n > 4 else [] for n in lens], [min(4, n) for n in lens], seed=seed)
        self.sw = synth.draw_stack_weights(self.w, N_LAYERS)
        self.layers = [{k: to_dev(v, dtype) for k, v in lw.items()} for lw in self.sw["layers"]]
        self.g = to_dev(self.sw["g_final"], dtype)
        h = self.shape.hidden
        self.table = synth.round_to_storage(rng.standard_normal((VOCAB, h), dtype=np.float32), dtype).astype(np.float64)
        self.vocab = synth.round_to_storage(0.3 * rng.standard_normal((VOCAB, h), dtype=np.float32), dtype).astype(np.float64)
        self.wv = to_dev(self.vocab, dtype)
        self.prompts = [rng.integers(0, VOCAB, n) for n in lens]
        self.tol = 1e-4 if dtype == "f32" else 2e-2

    def embed(self, tokens):
        return to_dev(self.table[np.asarray(tokens)], self.dtype)

    def logits(self, texts):
        """Float64 logits behind every token of whole texts (rounded where the path stores)."""
        s = self.shape
        lens = [len(t) for t in texts]
        sd = dict(n_q_heads=s.n_q_heads, n_kv_heads=s.n_kv_heads, head_dim=s.head_dim, base=s.rope_base, layout=s.rope_layout,
                  sm_scale=s.head_dim ** -0.5, eps=s.rms_eps)
        layers = [{k: v.astype(np.float64) for k, v in lw.items()} for lw in self.sw["layers"]]
        r = st.full_prefill_stack(self.table[np.concatenate(texts)], np.concatenate([np.arange(n) for n in lens]), np.concatenate([[0], np.cumsum(lens)]),
                                  layers, self.sw["g_final"].astype(np.float64), sd, self.dtype)
        return np.split(r["hidden"] @ self.vocab.T, np.cumsum(lens)[:-1])

    def pages(self, lens, table=None, seed=0, page=32, q8=False):
        s = self.shape
        p = make_pages(lens, dtype=self.dtype, Hq=s.n_q_heads, Hkv=s.n_kv_heads, d=s.head_dim, page=page, base=s.rope_base, layout=s.rope_layout, seed=seed, q8=q8)
        pages = [p] + [p.sibling() for _ in range(N_LAYERS - 1)]
        for x in pages[1:]:
            x.k_pool.copy_(p.k_pool)
            x.v_pool.copy_(p.v_pool)
        return pages

    def prefill(self, pages):
        lay = api.Layout.from_workload(self.w)
        emb = np.concatenate([self.table[t] for t in self.prompts])
        return stack.prefill_stack(lay, self.shape, self.layers, self.g, to_dev(emb, self.dtype), pages=pages)

    def decode_layout(self, n):
        s = self.shape
        return api.Layout.decode(dtype=self.dtype, n_q_heads=s.n_q_heads, n_kv_heads=s.n_kv_heads, head_dim=s.head_dim, hidden=s.hidden,
                                 rope_base=s.rope_base, n_req=n)


TREES = [[-1, 0, 0, 1, 1, 3, 2], [-1], [-1, 0, 1, 2, 3], [-1, 0, 0, 0, 2, 4, 4, 5, 1, 8, 9, 6]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_verified_tree_is_its_branches_one_by_one(dtype):
    """Logits of every drafted token are those of the text of its branch; the accepted path, its cache and the tokens that follow are those of
    a text written token by token."""
    lens = [40, 1, 33, 90]
    m = Model(dtype, lens)
    pages = m.pages([n + 60 for n in lens])
    m.prefill(pages)
    layers = api.PageLayers(pages)
    rng = np.random.default_rng(5)
    n = sum(len(t) for t in TREES)
    lay = m.decode_layout(n)
    bufs = stack.DecodeBuffers(lay, m.shape, m.shape.ffn, pages, VOCAB, tree=(len(TREES), 12))
    out = api.TreeAccepted(len(TREES), n, 6, VOCAB)
    texts = [list(t) for t in m.prompts]
    next_token = rng.integers(0, VOCAB, len(TREES))
    for turn in range(3):
        # what the model says behind each branch, to draft one path that it agrees with
        tokens = [rng.integers(0, VOCAB, len(t)) for t in TREES]
        for g, t in enumerate(TREES):
            tokens[g][0] = next_token[g]
            at, text = 0, texts[g] + [next_token[g]]
            while True:
                children = [c for c in range(at + 1, len(t)) if t[c] == at]
                if not children or (turn == 1 and g == 3 and at == 2):
                    break
                at = int(rng.choice(children))
                tokens[g][at] = int(m.logits([np.array(text)])[0][-1].argmax())
                text.append(tokens[g][at])
        tree = stack.TreeRows(TREES, [len(t) for t in texts], np.concatenate(tokens), max_path=6)
        r = stack.verify_stack(lay, m.shape, m.layers, m.g, m.embed(np.concatenate(tokens)), layers, tree, bufs, m.wv, out)
        torch.cuda.synchronize()
        logits, picked = to_host(r["logits"]), out.picked.cpu().numpy()
        branches, rows, at = [], [], 0
        for g, t in enumerate(TREES):
            seen = cand.ancestors(t)
            for j in range(len(t)):
                branches.append(np.array(texts[g] + [int(tokens[g][i]) for i in np.nonzero(seen[j])[0]]))
        want = np.stack([x[-1] for x in m.logits(branches)])
        assert max_abs_rel(logits, want) <= m.tol
        assert np.array_equal(picked, gen.top(logits, 1)[:, 0])
        for g, t in enumerate(TREES):
            path = cand.follow(picked[at:at + len(t)], tokens[g], t, 6)
            assert out.count[g].item() == len(path) and out.path[g].tolist()[:len(path)] == path
            if len(t) > 1 and not (turn == 1 and g == 3):
                assert len(path) > 1                                     # the draft agrees (near ties may end a path early, not at once)
            texts[g] += [int(tokens[g][i]) for i in path]
            next_token[g] = out.next_token[g].item()
            assert next_token[g] == picked[at + path[-1]]
            at += len(t)
    # the caches are those of the texts: a plain prefill of them
    again = Model(dtype, [len(t) for t in texts])
    again.prompts, again.layers, again.g, again.sw, again.table, again.vocab = [np.array(t) for t in texts], m.layers, m.g, m.sw, m.table, m.vocab
    whole = again.pages([len(t) + 4 for t in texts], seed=9)
    again.prefill(whole)
    torch.cuda.synchronize()
    for a, b in zip(pages, whole):
        for g, t in enumerate(texts):
            for x, y in zip(get(a, g, 0, len(t)), get(b, g, 0, len(t))):
                assert max_abs_rel(x, y) <= m.tol
    # and one more token each goes on from them
    dlay = m.decode_layout(len(texts))
    slot = idev([len(t) for t in texts])
    r = stack.decode_stack(dlay, m.shape, m.layers, m.g, m.embed(next_token), pages, slot, slot, slot + 1,
                           stack.DecodeBuffers(dlay, m.shape, m.shape.ffn, pages, VOCAB), w_vocab=m.wv)
    want = np.stack([x[-1] for x in m.logits([np.array(t + [int(x)]) for t, x in zip(texts, next_token)])])
    assert max_abs_rel(to_host(r["logits"]), want) <= m.tol


@pytest.mark.parametrize("q8", [False, True])
def test_a_verification_step_captured(q8):
    """The step as one graph, replayed with the next trees, tokens and lengths, is the eager step, bit for bit; 8-bit pages too."""
    lens = [40, 9, 64]
    m = Model("bf16", lens)
    rng = np.random.default_rng(8)
    parents = [[-1, 0, 0, 1], [-1, 0, 1, 2], [-1, 0, 0, 0]]
    lay, runs = m.decode_layout(12), []
    steps = [(rng.permutation(3), rng.integers(0, VOCAB, 12)) for _ in range(4)]
    for captured in (False, True):
        pages = m.pages([n + 80 for n in lens], q8=q8)
        m.prefill(pages)
        layers = api.PageLayers(pages)
        bufs, out = stack.DecodeBuffers(lay, m.shape, m.shape.ffn, pages, VOCAB, tree=(3, 4)), api.TreeAccepted(3, 12, 4, VOCAB)
        tree = stack.TreeRows(parents, lens, np.zeros(12), max_path=4)
        resid = torch.zeros((12, m.shape.hidden), dtype=torch.bfloat16, device="cuda")
        step = lambda: stack.verify_stack(lay, m.shape, m.layers, m.g, resid, layers, tree, bufs, m.wv, out)
        if captured:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()                                                   # (the same rows are written again by the first replay)
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        now, got = list(lens), []
        for order, tokens in steps:
            fresh = stack.TreeRows([parents[i] for i in order], now, tokens, max_path=4)
            for name in ("tokens", "group_start", "group_req", "group_len", "parent", "mask", "path_req", "row_req", "row_slot", "row_pos"):
                getattr(tree, name).copy_(getattr(fresh, name))
            resid.copy_(m.embed(tokens))
            if captured:
                graph.replay()
            else:
                step()
            torch.cuda.synchronize()
            now = [n + c for n, c in zip(now, out.count.tolist())]
            got += [to_host(bufs.logits), out.path.cpu().numpy().copy(), out.next_token.cpu().numpy().copy()]
        for p in pages:
            for g in range(3):
                got += get(p, g, 0, now[g])
        runs.append(got)
    assert all(np.array_equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beam_search(dtype):
    """Six steps of three beams each over two prompts whose full pages the beams share: every beam's score is the float64 oracle's of its text,
    its cache that of its text, and at every step the best of all continuations were chosen."""
    lens, B, steps = [70, 45], 3, 6
    m = Model(dtype, lens)
    pages = m.pages([n + steps + 2 for n in lens for _ in range(B)], page=32)
    table = pages[0].page_table
    for g, n in enumerate(lens):
        table[g * B:g * B + B, :n // 32] = table[g * B, :n // 32]           # shared: the prompt's full pages
    # the prompts go to the first beam of each; its partial page to the others
    two = m.pages([n for n in lens], page=32, seed=1)
    pre = m.prefill(two)
    torch.cuda.synchronize()
    t2 = two[0].page_table.cpu().numpy()
    for a, b in zip(pages, two):
        for g, n in enumerate(lens):
            for j in range(-(-n // 32)):
                for x, y in ((a.k_pool, b.k_pool), (a.v_pool, b.v_pool)):
                    x[table[g * B, j].item()] = y[t2[g, j]]
    layers = api.PageLayers(pages)
    fork = [[g * B] * B for g in range(2)]
    full = [[n // 32 * 32] * B for n in lens]
    api.a3_paged_move(layers, idev(fork), idev(full), idev(np.arange(2 * B).reshape(2, B)), idev(full),
                      idev([[n % 32] * B for n in lens]), 32, 2, B)
    # the first choice: of the prompt's last logits, one beam alive
    last = np.cumsum(lens) - 1
    lg = torch.empty((2, VOCAB), device="cuda")
    api.a3_lm_head(api.Layout.from_workload(m.w), pre["hidden"], idev(last), 2, m.wv, lg)
    first = api.BeamChoice(2, 1, VOCAB, B)
    api.a3_beam_select(lg, torch.zeros(2, device="cuda"), None, 0, first)
    score, tokens = first.score.flatten().clone(), first.token.flatten().clone()
    texts = [list(m.prompts[g]) + [tokens[g * B + b].item()] for g in range(2) for b in range(B)]
    lay = m.decode_layout(2 * B)
    bufs = stack.DecodeBuffers(lay, m.shape, m.shape.ffn, pages, VOCAB)
    out = api.BeamChoice(2, B, VOCAB, B)
    row_len0 = idev([n for n in lens for _ in range(B)])
    own = idev([n // 32 * 32 for n in lens for _ in range(B)])
    for step in range(steps):
        slot = row_len0 + step
        r = stack.beam_stack(lay, m.shape, m.layers, m.g, m.embed(tokens.cpu().numpy()), layers, slot, slot, slot + 1, bufs, m.wv, score, own,
                             slot + 1 - own, 32 + steps, out)
        torch.cuda.synchronize()
        logits, before = to_host(r["logits"]), to_host(score)
        want = np.stack([x[-1] for x in m.logits([np.array(t) for t in texts])])
        assert max_abs_rel(logits, want) <= m.tol
        for g in range(2):
            s, b, t = cand.beams(logits[g * B:g * B + B], before[g * B:g * B + B], None, 0, B)
            assert np.abs(to_host(out.score)[g] - s).max() < 1e-4
            assert np.array_equal(out.row[g].cpu().numpy(), g * B + b) and np.array_equal(out.token[g].cpu().numpy(), t)
        texts = [texts[i] + [t] for i, t in zip(out.row.flatten().tolist(), out.token.flatten().tolist())]
        score, tokens = out.score.flatten().clone(), out.token.flatten().clone()
    lp = m.logits([np.array(t) for t in texts])
    for i, t in enumerate(texts):
        n = lens[i // B]
        total = sum(gen.log_probs(lp[i][p][None])[0, t[p + 1]] for p in range(n - 1, len(t) - 1))
        assert abs(total - float(score[i])) <= (steps + 1) * 10 * m.tol * max(1.0, np.abs(lp[i]).max())
    again = Model(dtype, [len(t) - 1 for t in texts])
    again.prompts, again.layers, again.g, again.sw, again.table = [np.array(t[:-1]) for t in texts], m.layers, m.g, m.sw, m.table
    whole = again.pages([len(t) for t in texts], seed=9)
    again.prefill(whole)
    torch.cuda.synchronize()
    for a, b in zip(pages, whole):
        for i, t in enumerate(texts):
            for x, y in zip(get(a, i, 0, len(t) - 1), get(b, i, 0, len(t) - 1)):
                assert max_abs_rel(x, y) <= m.tol


def test_what_steps_refuse():
    m = Model("bf16", [8, 8])
    pages = m.pages([40, 40])
    lay = m.decode_layout(4)
    bufs = stack.DecodeBuffers(lay, m.shape, m.shape.ffn, pages, VOCAB)
    tree = stack.TreeRows([[-1, 0], [-1, 0]], [8, 8], max_path=4)
    resid = torch.zeros((4, m.shape.hidden), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="without room for trees"):
        stack.verify_stack(lay, m.shape, m.layers, m.g, resid, api.PageLayers(pages), tree, bufs, m.wv, api.TreeAccepted(2, 4, 4, VOCAB))
    with pytest.raises(ValueError, match="paths of 5"):
        stack.verify_stack(lay, m.shape, m.layers, m.g, resid, api.PageLayers(pages), tree, bufs, m.wv, api.TreeAccepted(2, 4, 5, VOCAB))
    with pytest.raises(ValueError, match="parents stand in front"):
        stack.TreeRows([[-1, 1]], [8])
    with pytest.raises(ValueError, match="one page table"):
        api.PageLayers([pages[0], m.pages([40, 40])[0]])
    z = idev(np.zeros(4))
    with pytest.raises(ValueError, match="3 continuations for 2 beams"):
        stack.beam_stack(lay, m.shape, m.layers, m.g, resid, api.PageLayers(pages), z, z, z, bufs, m.wv, z.float(), z, z, 1, api.BeamChoice(2, 2, VOCAB, 3))
