"""Gradients in place of what a call has yet to read are refused.  No GPU is needed."""
import ctypes

import pytest

INVALID = 1


@pytest.fixture(scope="module")
def S():
    import paper_2507_16274_amd as S
    return S


@pytest.mark.parametrize("stride,d_stride", [(100, 108), (108, 100), (0, 100)])
def test_gradient_of_logits(S, stride, d_stride):
    """In place of the logits only with the same distance between rows."""
    assert S.lib.stalloc_token_logprobs_backward(1, 4, 100, 512, stride, 256, 256, 256, 256, None, 512, d_stride, 256, None) == INVALID


@pytest.mark.parametrize("taken", ["d_o", "q", "o"])
def test_gradient_of_queries(S, taken):
    """The second kernel reads q and d_o again, and where results are not finite o, when dq is written."""
    shape, have = S._AttentionShape(1, 100, 2, 4, 2, 64, 0.125), ctypes.c_size_t(1 << 40)
    at = {name: 4096 * (i + 1) for i, name in enumerate(("d_o", "q", "k", "v", "o", "dq", "dk", "dv"))}
    at["dq"] = at[taken]
    t = {name: S._Heads(data, 512, 64) for name, data in at.items()}
    assert S.lib.stalloc_attention_backward(shape, t["d_o"], t["q"], t["k"], t["v"], t["o"], 256, 256, t["dq"], t["dk"], t["dv"], 256, 256, ctypes.byref(have), None) == INVALID
