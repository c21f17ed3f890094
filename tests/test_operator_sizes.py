"""Sizes travel to the library in 32 bits: a tensor of more rows than that is refused, not taken for one of what is left of the number.  No GPU is needed: the first thing looked at."""
import pytest


@pytest.fixture(scope="module")
def S():
    import paper_2507_16274_amd as S
    return S


@pytest.mark.parametrize("rows", [1 << 31, (1 << 32) + 4])
def test_rows(S, rows):
    import torch
    x = torch.zeros(1, 8).expand(rows, 8)
    one, w, q = torch.zeros(1).expand(rows), torch.zeros(8), torch.zeros(1, 1, 8).expand(rows, 1, 8)
    bounds = torch.zeros(2, dtype=torch.int32)
    calls = [lambda: S.stalloc_rms_norm(x, w), lambda: S.stalloc_rms_norm_backward(x, x, w, one), lambda: S.stalloc_token_logprobs(x, one),
             lambda: S.stalloc_token_logprobs_backward(x, one, one, one, one), lambda: S.stalloc_attention(q, q, q, bounds),
             lambda: S.stalloc_attention_backward(q, q, q, q, q, one, bounds), lambda: S.stalloc_attention(q[:4], q[:4], q[:4], torch.zeros(1).expand(rows + 1))]
    for call in calls:
        with pytest.raises(ValueError, match="2\\^31"):
            call()
