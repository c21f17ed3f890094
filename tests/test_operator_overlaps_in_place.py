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
