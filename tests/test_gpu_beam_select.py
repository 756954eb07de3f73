"""The best continuations of beams, against float64.

Rows and tokens are equal: the worths of two candidates here differ by far more than the kernel's error, or they are of one row and
equal, or exactly equal by construction.  Worths: score + (x - m) - log Z is rounded to float once (2^-24 of it), and log Z is off by
what float32 exponentials make of it: their argument's rounding and their own, relative 2^-24 * (|x - m| + 4) of each term, 64 at most
here, and sums of up to a few hundred terms in float32: 2^-24 * 400.  1e-4 leaves room for all of them at their worst."""
import numpy as np
import pytest
import torch

from oracle import candidates_oracle as cand
from paper_2511_17560_amd import api
from gpu_util import idev, to_host

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _select(x, score, n_beams, n_best, done=None, end=0, dtype="f32", ld=None, shift=0, out=None, stream=None):
    rows, vocab = x.shape
    wide = torch.full((rows, (ld or vocab) + shift), float("nan"), dtype=TYPES[dtype], device="cuda")
    part = wide[:, shift:shift + vocab]
    part.copy_(torch.from_numpy(x))
    n_groups = rows // n_beams
    out = api.BeamChoice(n_groups, n_beams, vocab, n_best) if out is None else out
    out.score.fill_(77.0)
    out.row.fill_(-77)
    out.ws.fill_(255)
    s = torch.tensor(np.asarray(score), dtype=torch.float32, device="cuda")
    torch.cuda.synchronize()
    api.a3_beam_select(part, s, None if done is None else idev(done), end, out, stream=stream)
    torch.cuda.synchronize()
    stored = part.double().cpu().numpy()
    return out, stored, s.double().cpu().numpy()


def _check(out, x, score, n_beams, n_best, done=None, end=0):
    for g in range(len(x) // n_beams):
        rows = slice(g * n_beams, (g + 1) * n_beams)
        s, b, t = cand.beams(x[rows], score[rows], None if done is None else np.asarray(done)[rows], end, n_best)
        got_s, got_r, got_t = (o[g].cpu().numpy() for o in (out.score, out.row, out.token))
        assert np.array_equal(got_r, np.where(b < 0, -1, g * n_beams + b)), g
        assert np.array_equal(got_t, t), g
        gone = b < 0
        assert np.isneginf(got_s[gone]).all()
        assert np.all(np.abs(got_s[~gone] - s[~gone]) <= 1e-4 + 2.0 ** -24 * np.abs(s[~gone])), g


def _logits(rng, rows, vocab):
    x = rng.standard_normal((rows, vocab)).astype(np.float32) * 2
    for r in range(rows):
        x[r, rng.integers(0, vocab, 4)] += rng.random(4) * 12
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,n_groups,n_beams,n_best", [(1, 2, 3, 5), (2, 1, 1, 1), (7, 3, 4, 64), (63, 1, 2, 4), (501, 5, 4, 8), (1000, 300, 4, 8), (4099, 2, 64, 64),
                                                           (8200, 3, 5, 10), (32003, 1, 8, 16), (32003, 20, 3, 6), (128256, 1, 4, 8), (152064, 2, 1, 2),
                                                           (170000, 1, 2, 64), (5001, 1100, 1, 2), (200003, 1, 1, 1)])
def test_best(vocab, n_groups, n_beams, n_best, dtype):
    rng = np.random.default_rng(vocab + n_best)
    rows = n_groups * n_beams
    score = -20 * rng.random(rows)
    out, x, s = _select(_logits(rng, rows, vocab), score, n_beams, n_best, dtype=dtype)
    _check(out, x, s, n_beams, n_best)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_start_anywhere(dtype):
    rng = np.random.default_rng(1)
    for shift in range(9):
        x, score = _logits(rng, 6, 3001), -3 * rng.random(6)
        out, stored, s = _select(x, score, 3, 7, dtype=dtype, ld=3001 + shift % 5, shift=shift)
        _check(out, stored, s, 3, 7)


def test_beams_that_have_ended_or_do_not_go_on():
    """Ended beams are one candidate each, and stay where they are in the order; beams at -inf, +inf or NaN, or without a distribution, give
    none; a beam that has ended needs no logits."""
    rng = np.random.default_rng(2)
    vocab, n_beams = 900, 6
    x = _logits(rng, 4 * n_beams, vocab)
    score = -2 * rng.random(4 * n_beams)
    done = (rng.random(4 * n_beams) < 0.4).astype(np.int32)
    done[0], score[0] = 1, 50.0
    done[1], score[1] = -3, -500.0                                       # any number but 0
    x[1] = np.nan
    done[2:6] = 0
    score[2], score[3], score[4] = -np.inf, np.nan, np.inf
    x[n_beams:2 * n_beams] = -np.inf                                     # a group of which only ended beams are left
    done[n_beams:2 * n_beams] = [0, 1, 0, 0, 1, 0]
    score[n_beams + 1] = score[n_beams + 4]                              # equal: the lower beam
    x[2 * n_beams, 5], x[2 * n_beams + 1, 7], x[2 * n_beams + 2] = np.nan, np.inf, -np.inf
    done[2 * n_beams:2 * n_beams + 3] = 0
    x[3 * n_beams:, 3:] = -np.inf                                        # three tokens a beam, fewer than are asked for
    done[3 * n_beams:] = 0
    for n_best in (1, 6, 30):
        for end in (0, 899, 2 ** 31 - 1):
            out, stored, s = _select(x, score, n_beams, n_best, done=done, end=end)
            _check(out, stored, s, n_beams, n_best, done=done, end=end)
    out, stored, s = _select(x, np.full(4 * n_beams, -np.inf), n_beams, 5)
    assert bool((out.row == -1).all()) and bool((out.token == -1).all()) and bool(torch.isneginf(out.score).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [3001, 32003, 140001])
def test_equal_candidates(vocab, dtype):
    """Equal logits: the lower token; beams that are the same in everything: the lower beam, wherever its row starts; constant rows; -0 and 0."""
    rng = np.random.default_rng(7)
    x = np.round(_logits(rng, 1, vocab) * 2) / 2
    x = np.repeat(x, 4, 0)
    out, stored, s = _select(x, [-1.0] * 4, 4, 16, dtype=dtype, ld=vocab + 1)
    want = np.lexsort((np.arange(vocab), -stored[0]))[:16]
    # every place of the order is taken by the four beams in turn, as far as it goes; equal logits of one beam come before the next beam's
    s0, b0, t0 = cand.beams(stored, s, None, 0, 16)
    assert np.array_equal(out.row[0].cpu().numpy(), b0) and np.array_equal(out.token[0].cpu().numpy(), t0) and set(t0) <= set(want)
    flat = np.zeros((4, vocab), np.float32)
    flat[1] = -0.0
    flat[2:, ::2] = -0.0
    out, stored, s = _select(flat, [-2.0, -1.0, -1.0, -1.0], 4, 9, dtype=dtype)
    assert out.row[0].tolist() == [1] * 9 and out.token[0].tolist() == list(range(9))
    lowest = float(torch.finfo(TYPES[dtype]).min)                        # a mask of the type's lowest value
    x = np.full((2, vocab), lowest, np.float32)
    x[0, [5, 90]], x[1, [vocab - 1]] = [1.0, 2.0], 3.0
    out, stored, s = _select(x, [0.0, -0.5], 2, 3, dtype=dtype)
    assert out.row[0].tolist() == [0, 1, 0] and out.token[0].tolist() == [90, vocab - 1, 5]
    assert np.abs(to_host(out.score)[0] - [-np.log1p(np.exp(-1.0)), -0.5, -1 - np.log1p(np.exp(-1.0))]).max() < 1e-5


def test_worths_close_together():
    """Two beams whose best continuations differ by 1e-5 in worth, either way round: the larger first."""
    vocab = 50000
    rng = np.random.default_rng(3)
    base = _logits(rng, 2, vocab)
    lp = base.astype(np.float64) - np.log(np.exp(base.astype(np.float64)).sum(-1, keepdims=True))
    best = lp.max(-1)
    for d in (1e-5, -1e-5):
        score = np.array([-best[0], -best[1] + d])
        out, stored, s = _select(base, score, 2, 2)
        total = (s + best)
        assert out.row[0].tolist()[0] == int(total[1] > total[0])
        _check(out, stored, s, 2, 2)


def test_adversarial_rows():
    """Values that rise or fall along the row, one thread's or one slice's far above all others, NaN-free but masked nearly everywhere."""
    vocab = 40003
    rise = np.linspace(-5, 5, vocab, dtype=np.float32)
    x = np.stack([rise, rise[::-1], np.where(np.arange(vocab) % 1024 == 3, rise + 9, rise), np.where((np.arange(vocab) > 3000) & (np.arange(vocab) < 3100), rise + 30, -9),
                  np.where(np.arange(vocab) == 12345, 0.0, -np.inf).astype(np.float32), np.where(np.arange(vocab) % 700 == 0, rise, -np.inf)]).astype(np.float32)
    for n_best in (1, 8, 64):
        out, stored, s = _select(x, [0.0, -0.1, -0.2, -3.0, -4.0, -5.0], 6, n_best)
        _check(out, stored, s, 6, n_best)
        out, stored, s = _select(x, [0.0] * 6, 1, n_best, dtype="bf16")
        _check(out, stored, s, 1, n_best)


def test_buffers_made_for_more_on_another_stream_and_captured():
    rng = np.random.default_rng(11)
    vocab, n_beams, n_best = 9001, 4, 8
    big, side = api.BeamChoice(9, n_beams, vocab, n_best), torch.cuda.Stream()
    x, score = _logits(rng, 8, vocab), -5 * rng.random(8)
    out, stored, s = _select(x, score, n_beams, n_best, out=big, stream=side)
    _check(out, stored, s, n_beams, n_best)
    assert bool((big.row[2:] == -77).all())
    xd, sd, dd = torch.empty((8, vocab), device="cuda"), torch.empty(8, device="cuda"), idev(np.zeros(8))
    xd.copy_(torch.from_numpy(x))
    sd.zero_()
    api.a3_beam_select(xd, sd, dd, 3, big)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.a3_beam_select(xd, sd, dd, 3, big)
    for i in range(4):
        x, score, done = _logits(rng, 8, vocab), (-5 * rng.random(8)).astype(np.float32), (rng.random(8) < 0.3).astype(np.int32)
        xd.copy_(torch.from_numpy(x))
        sd.copy_(torch.from_numpy(score))
        dd.copy_(idev(done))
        big.row.fill_(-77)
        g.replay()
        torch.cuda.synchronize()
        _check(big, x.astype(np.float64), score.astype(np.float64), n_beams, n_best, done=done, end=3)


def test_many_rows_of_more_than_4_gib():
    vocab, rows, n_beams = 140000, 8192, 4
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((rows, vocab), device="cuda", generator=g, dtype=torch.float32).to(torch.bfloat16).mul_(2)
    x[rows - 1, vocab - 1] = 30.0
    score = -0.5 * torch.rand(rows, device="cuda", generator=g)
    out = api.BeamChoice(rows // n_beams, n_beams, vocab, 4)
    api.a3_beam_select(x, score, None, 0, out)
    torch.cuda.synchronize()
    assert out.row[-1, 0].item() == rows - 1 and out.token[-1, 0].item() == vocab - 1
    for grp in (0, 1000, rows // n_beams - 1):
        part = slice(grp * n_beams, grp * n_beams + n_beams)
        s, b, t = cand.beams(x[part].double().cpu().numpy(), score[part].double().cpu().numpy(), None, 0, 4)
        assert np.array_equal(out.token[grp].cpu().numpy(), t) and np.array_equal(out.row[grp].cpu().numpy(), grp * n_beams + b)
