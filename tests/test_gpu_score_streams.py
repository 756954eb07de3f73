"""Rating tokens on every kind of stream argument that the library's calls take: none, a torch stream, a raw handle, the default stream's."""
import numpy as np
import pytest
import torch

from paper_2511_17560_amd import api, stack
from gpu_util import idev, to_dev

pytestmark = pytest.mark.gpu


def test_score_tokens_on_any_stream():
    n, h, vocab = 50, 64, 333
    rng = np.random.default_rng(3)
    lay = api.Layout.decode(dtype="f32", n_q_heads=1, n_kv_heads=1, head_dim=64, hidden=h, rope_base=1e4, n_req=n)
    x, w = to_dev(rng.standard_normal((n, h)), "f32"), to_dev(0.1 * rng.standard_normal((vocab, h)), "f32")
    tokens = idev(rng.integers(0, vocab, (n, 2)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    runs = []
    for stream in (None, side, side.cuda_stream, 0, torch.cuda.default_stream().cuda_stream):
        out = api.TokenLogprobs(n, vocab, 2, 3)
        for t in (out.logprob, out.entropy, out.top_logprob):
            t.fill_(9.0)
        torch.cuda.synchronize()
        before = torch.cuda.current_stream()
        assert stack.score_tokens(lay, x, None, n, w, tokens, out, rows_at_once=20, stream=stream) is out
        assert torch.cuda.current_stream() == before
        torch.cuda.synchronize()
        runs.append(out)
    for out in runs[1:]:
        for name in ("logprob", "entropy", "top_idx", "top_logprob"):
            assert torch.equal(getattr(out, name), getattr(runs[0], name))


def test_a_raw_handle_is_the_stream_it_names():
    """Calls queued on the handle come behind what is on the stream already."""
    side = torch.cuda.Stream()
    s = api.torch_stream(side.cuda_stream)
    assert s.cuda_stream == side.cuda_stream and api.torch_stream(side) is side
    assert api.torch_stream(0).cuda_stream == torch.cuda.default_stream().cuda_stream
    assert api.torch_stream(None).cuda_stream == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert api.torch_stream(None).cuda_stream == side.cuda_stream
