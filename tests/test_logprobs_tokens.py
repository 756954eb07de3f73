"""Given tokens whose rows are not n_given apart are refused before anything else (no GPU needed)."""
import pytest
import torch

from paper_2511_17560_amd import api


def _out(n_given):
    out = object.__new__(api.TokenLogprobs)
    out.n_given, out.n_top, out.entropy = n_given, 0, torch.zeros(4)
    return out


@pytest.mark.parametrize("shape,n_given", [((4, 3), 2), ((4, 1), 2), ((4, 2), 1), ((8, 1), 2), ((1, 4), 1), ((2, 2, 3), 2), ((4, 2), 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_of_another_width_are_refused(shape, n_given, dtype):
    with pytest.raises(ValueError, match=rf"tokens are int32 \[4, {n_given}\]"):
        api.a3_token_logprobs(torch.zeros((4, 10), dtype=dtype), torch.zeros(shape, dtype=torch.int32), _out(n_given))


def test_missing_tokens_are_refused():
    with pytest.raises(ValueError, match=r"tokens are int32 \[4, 2\]"):
        api.a3_token_logprobs(torch.zeros((4, 10)), None, _out(2))


@pytest.mark.parametrize("shape,n_given", [((4, 2), 2), ((6, 2), 2), ((4,), 1), ((4, 1), 1)])
def test_rows_of_the_right_width_go_on_to_the_device_check(shape, n_given):
    """(the tensors here are on the CPU, which is what is refused then)"""
    with pytest.raises((ValueError, RuntimeError)) as e:
        api.a3_token_logprobs(torch.zeros((4, 10)), torch.zeros(shape, dtype=torch.int32), _out(n_given))
    assert "tokens are int32" not in str(e.value)
