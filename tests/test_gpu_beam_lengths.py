"""beam_stack over beams whose own runs differ in length (some have ended and hold fewer slots): the caches that go on are whole.

The blocks are left out (a step's logits are given): this is about what the selection and the moves make of them.  Values are copied, so equal."""
import numpy as np
import pytest
import torch

import a3_synth as synth
from oracle import candidates_oracle as cand
from paper_2511_17560_amd import api, stack
from gpu_util import idev
from paged_util import get, make_pages, put

pytestmark = pytest.mark.gpu
SHAPE, VOCAB, PAGE = synth.ModelShape("lengths", "bf16", 512, 8, 2, 128, 5e5, synth.ROPE_HALF, ffn=768), 61, 32


def _run(monkeypatch, how):
    """Steps of 2 groups of 4 beams; `how` runs the step.  The expected caches and the real ones, of every step."""
    rng = np.random.default_rng(12)
    B, n, first = 4, 8, [40, 25]
    pages = make_pages([140] * n, dtype="bf16", Hq=8, Hkv=2, d=128, page=PAGE, seed=4)
    pages = [pages, pages.sibling()]
    for p in pages[1:]:
        p.k_pool.fill_(float("nan"))
        p.v_pool.fill_(float("nan"))
    layers = api.PageLayers(pages)
    lay = api.Layout.decode(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=512, rope_base=5e5, n_req=n)
    bufs, out = stack.DecodeBuffers(lay, SHAPE, SHAPE.ffn, pages, VOCAB), api.BeamChoice(2, B, VOCAB, B)
    logits, score, done, runs = torch.zeros(n, VOCAB, device="cuda"), torch.zeros(n, device="cuda"), idev(np.zeros(n)), idev(np.zeros(n))
    own = idev(np.repeat(first, B))
    resid, z = torch.zeros((n, 512), dtype=torch.bfloat16, device="cuda"), idev(np.zeros(n))
    w = torch.zeros((VOCAB, 512), dtype=torch.bfloat16, device="cuda")
    monkeypatch.setattr(stack, "decode_stack", lambda *a, **k: dict(logits=logits))
    step = lambda stream=None: stack.beam_stack(lay, SHAPE, [], None, resid, layers, z, z, z, bufs, w, score, own, runs, 90, out, done=done, end_token=3,
                                                stream=stream)
    go = how(step)
    for turn in range(4):
        length = rng.integers(1, 80, n)
        over = (rng.random(n) < 0.4).astype(np.int32)
        if turn == 0:                                                    # the longest beam takes the place of the shortest, and the other way round
            length, over = np.array([3, 70, 5, 66, 1, 2, 79, 40]), np.array([0, 0, 1, 0, 0, 1, 0, 0])
        held = []
        for p in pages:
            for r in range(n):
                k, v = (rng.standard_normal((length[r], 2, 128)) for _ in range(2))
                put(p, r, first[r // B], k, v)
            held.append([get(p, r, first[r // B], first[r // B] + 80) for r in range(n)])
        x = rng.standard_normal((n, VOCAB)).astype(np.float32) * 2
        sc = (-5 * rng.random(n)).astype(np.float32)
        if turn == 0:
            sc[:] = [-30, 0, -0.5, -30, -30, -0.25, 0, -30]
        logits.copy_(torch.from_numpy(x))
        score.copy_(torch.from_numpy(sc))
        done.copy_(idev(over))
        runs.copy_(idev(length))
        torch.cuda.synchronize()
        go()
        torch.cuda.synchronize()
        rows = out.row.flatten().tolist()
        for g in range(2):
            part = slice(g * B, g * B + B)
            _, b, t = cand.beams(x[part].astype(np.float64), sc[part].astype(np.float64), over[part], 3, B)
            assert rows[part] == (g * B + b).tolist() and out.token[g].tolist() == t.tolist()
        for p, before in zip(pages, held):
            for j, i in enumerate(rows):
                at = first[j // B]
                for now, had, mine in zip(get(p, j, at, at + 80), before[i], before[j]):
                    want = mine.copy()                                   # (slots behind the source's run stay as they were)
                    want[:length[i]] = had[:length[i]]
                    assert np.array_equal(now, want, equal_nan=True), (turn, j, i)
        assert turn or any(length[i] != length[j] for j, i in enumerate(rows))   # targets take over runs of other lengths than their own


def test_eager(monkeypatch):
    _run(monkeypatch, lambda step: step)


def test_on_another_stream(monkeypatch):
    side = torch.cuda.Stream()
    _run(monkeypatch, lambda step: lambda: step(stream=side))


def test_captured(monkeypatch):
    def capture(step):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        return graph.replay
    _run(monkeypatch, capture)
