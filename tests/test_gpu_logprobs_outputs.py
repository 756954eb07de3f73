"""Outputs of log probabilities that do not hold what a call writes are refused, each of them; entropy may be None."""
import pytest
import torch

from paper_2511_17560_amd import api
from gpu_util import idev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,shape,dtype", [("logprob", (2, 2), torch.float32), ("logprob", (3, 2), torch.float64), ("entropy", (2,), torch.float32),
                                              ("top_idx", (2, 4), torch.int32), ("top_idx", (3, 4), torch.int64),
                                              ("top_logprob", (3, 3), torch.float32), ("ws", (1 << 20,), torch.float32)])
def test_outputs_that_are_too_small_or_of_another_type(name, shape, dtype):
    x, tok = torch.zeros((3, 50), device="cuda"), idev([[0, 1]] * 3)
    out = api.TokenLogprobs(3, 50, 2, 4)
    api.a3_token_logprobs(x, tok, out)
    for other in (torch.empty(shape, dtype=dtype, device="cuda"), getattr(out, name).cpu()):
        was = getattr(out, name)
        setattr(out, name, other)
        with pytest.raises(ValueError):
            api.a3_token_logprobs(x, tok, out)
        setattr(out, name, was)
    torch.cuda.synchronize()


def test_outputs_that_are_not_asked_for():
    x = torch.zeros((3, 50), device="cuda")
    out = api.TokenLogprobs(3, 50, 0, 0)
    out.entropy = out.logprob = out.top_idx = out.top_logprob = None
    api.a3_token_logprobs(x, None, out)
    torch.cuda.synchronize()
