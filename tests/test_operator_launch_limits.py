"""Shapes of more work than one launch takes (2^32 threads): refused on the host, when the workspace is asked for as well as in the call.  No GPU is needed."""
import ctypes

import pytest

TOO_LARGE = 9


@pytest.fixture(scope="module")
def S():
    import paper_2507_16274_amd as S
    return S


def _query(S, fn, count, **more):
    shape = S._AttentionShape(*{**dict(dtype=1, tokens=1 << 18, sequences=1 << 18, heads=64, kv_heads=64, head_dim=64, scale=0.125), **more}.values())
    need = ctypes.c_size_t(0)
    return fn(shape, *[None] * count, ctypes.byref(need), None)


def test_attention(S):
    """Workgroups of 256 threads: 2^24 of them are too many.  A batch has at most tokens / 128 + sequences + 1 pieces of every head."""
    for heads, kv_heads in ((64, 64), (64, 8)):
        assert _query(S, S.lib.stalloc_attention, 8, heads=heads, kv_heads=kv_heads) == TOO_LARGE
        assert _query(S, S.lib.stalloc_attention_backward, 12, heads=heads, kv_heads=kv_heads) == TOO_LARGE
    # 262144 pieces of 64 heads exactly, and one sequence less
    for sequences, want in (((1 << 18) - 2049, TOO_LARGE), ((1 << 18) - 2050, 0)):
        assert _query(S, S.lib.stalloc_attention, 8, sequences=sequences) == want
        assert _query(S, S.lib.stalloc_attention_backward, 12, sequences=sequences) == want
    t, have = S._Heads(256, 4096, 64), ctypes.c_size_t(1 << 40)
    shape = S._AttentionShape(1, 1 << 18, 1 << 18, 64, 64, 64, 0.125)
    assert S.lib.stalloc_attention(shape, t, t, t, 256, t, 256, 256, 256, ctypes.byref(have), None) == TOO_LARGE
    assert S.lib.stalloc_attention_backward(shape, t, t, t, t, t, 256, 256, t, t, t, 256, 256, ctypes.byref(have), None) == TOO_LARGE


def test_logprobs_backward(S):
    """A workgroup of 256 threads takes 8192 numbers of a row."""
    assert S.lib.stalloc_token_logprobs_backward(1, 1 << 23, 8193, 256, 8193, 256, 256, 256, 256, None, 256, 8193, 256, None) == TOO_LARGE
    assert S.lib.stalloc_token_logprobs_backward(1, (1 << 24) - 1, 8193, 256, 8193, 256, 256, 256, 256, None, 256, 8193, 256, None) == TOO_LARGE
