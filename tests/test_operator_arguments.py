"""What the operators of a training step refuse, before any HIP call: no GPU is needed."""
import ctypes

import pytest

INVALID, TOO_LARGE = 1, 9


@pytest.fixture(scope="module")
def S():
    import paper_2507_16274_amd as S
    return S


GOOD = dict(dtype=1, tokens=100, sequences=2, heads=4, kv_heads=2, head_dim=64, scale=0.125)


def _shape(S, **more):
    return S._AttentionShape(*{**GOOD, **more}.values())


def _attention(S, shape, tensors=None, bounds=256, lse=256, status=256, workspace=256, nbytes=1 << 40):
    t = tensors or [S._Heads(256, 512, 64) for _ in range(4)]
    have = ctypes.c_size_t(nbytes)
    return S.lib.stalloc_attention(shape, t[0], t[1], t[2], bounds, t[3], lse, status, workspace, ctypes.byref(have), None)


def _backward(S, shape, tensors=None, lse=256, bounds=256, status=256, workspace=256, nbytes=1 << 40):
    t = tensors or [S._Heads(256, 512, 64) for _ in range(8)]
    have = ctypes.c_size_t(nbytes)
    return S.lib.stalloc_attention_backward(shape, t[0], t[1], t[2], t[3], t[4], lse, bounds, t[5], t[6], t[7], status, workspace, ctypes.byref(have), None)


@pytest.mark.parametrize("more", [dict(dtype=0), dict(dtype=3), dict(tokens=0), dict(tokens=1 << 31), dict(sequences=0), dict(heads=0), dict(kv_heads=0),
                                  dict(heads=3), dict(kv_heads=8), dict(heads=1 << 17, kv_heads=1 << 17), dict(head_dim=0), dict(head_dim=12),
                                  dict(head_dim=136), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))], ids=str)
def test_attention_shapes(S, more):
    assert _attention(S, _shape(S, **more)) == INVALID and _backward(S, _shape(S, **more)) == INVALID
    assert _attention(S, _shape(S, **more), workspace=None) == INVALID and _backward(S, _shape(S, **more), workspace=None) == INVALID


def test_attention_tensors(S):
    shape = _shape(S)
    for call, count, written in ((_attention, 4, (3,)), (_backward, 8, (5, 6, 7))):
        for i in range(count):
            for bad in (S._Heads(None, 512, 64), S._Heads(264, 512, 64), S._Heads(256, 510, 64), S._Heads(256, 512, 63), S._Heads(256, 1 << 25, 64)):
                t = [S._Heads(256, 512, 64) for _ in range(count)]
                t[i] = bad
                assert call(S, shape, t) == INVALID
            if i in written:                                                     # outputs whose rows or heads would overlap
                for bad in (S._Heads(256, 0, 64), S._Heads(256, 512, 0)):
                    t = [S._Heads(256, 512, 64) for _ in range(count)]
                    t[i] = bad
                    assert call(S, shape, t) == INVALID
        for name in ("bounds", "lse", "status"):
            assert call(S, shape, **{name: None}) == INVALID
    assert _backward(S, shape, workspace=264) == INVALID and _backward(S, shape, nbytes=100) == INVALID
    assert _attention(S, _shape(S, tokens=(1 << 31) - 1, sequences=(1 << 31) - 1, heads=64)) == TOO_LARGE
    assert _attention(S, None) == INVALID


def test_attention_workspaces(S):
    """(a query looks at no memory, and needs no device) Row statistics always; sums of parts only where pieces are few."""
    for tokens in (1, 2, 100, 4096, 1 << 20):
        need = ctypes.c_size_t(0)
        assert S.lib.stalloc_attention_backward(_shape(S, tokens=tokens), *[None] * 12, ctypes.byref(need), None) == 0
        assert 8 * 4 * tokens <= need.value <= 8 * 4 * tokens + 16 * (tokens // 128 + 3) + 4096 + (1 << 28 if tokens < 1 << 20 else 0)
        assert S.lib.stalloc_attention(_shape(S, tokens=tokens), *[None] * 8, ctypes.byref(need), None) == 0
        assert 0 < need.value <= 1 << 28


def _norm(S, **more):
    a = {**dict(dtype=1, rows=4, width=100, x=256, x_stride=100, residual=256, residual_stride=100, weight=256, eps=1e-6, sum=256, y=256, q=None,
                scales=None, rstd=256), **more}
    return S.lib.stalloc_rms_norm(*a.values(), None)


@pytest.mark.parametrize("more", [dict(dtype=3), dict(rows=0), dict(rows=1 << 31), dict(width=0), dict(width=0x7ffff000), dict(x=None), dict(weight=None),
                                  dict(rstd=None), dict(eps=-1.0), dict(eps=float("nan")), dict(sum=None), dict(y=None), dict(q=256), dict(scales=256),
                                  dict(x=257), dict(weight=257), dict(residual=257), dict(sum=257), dict(y=257)], ids=str)
def test_norm(S, more):
    assert _norm(S, **more) == INVALID


@pytest.mark.parametrize("more", [dict(dtype=3), dict(rows=0), dict(width=0), dict(d_y=None), dict(sum=None), dict(weight=None), dict(rstd=None), dict(dx=None),
                                  dict(dweight=None), dict(workspace=264), dict(d_y=257), dict(dx=257), dict(d_sum=257)], ids=str)
def test_norm_backward(S, more):
    have = ctypes.c_size_t(1 << 40)
    a = {**dict(dtype=2, rows=4, width=100, d_y=256, stride=100, sum=256, weight=256, rstd=256, d_sum=None, dx=256, dweight=256, workspace=256), **more}
    assert S.lib.stalloc_rms_norm_backward(*a.values(), ctypes.byref(have), None) == INVALID
    small = ctypes.c_size_t(16)
    assert S.lib.stalloc_rms_norm_backward(2, 4, 100, 256, 100, 256, 256, 256, None, 256, 256, 256, ctypes.byref(small), None) == INVALID


@pytest.mark.parametrize("more", [dict(dtype=3), dict(rows=0), dict(rows=1 << 24), dict(vocabulary=0), dict(vocabulary=1 << 30), dict(logits=None), dict(logits=257),
                                  dict(tokens=None), dict(top=65), dict(top=101), dict(logprob=None), dict(entropy=None), dict(lse=None),
                                  dict(top_tokens=None), dict(top_logprobs=None), dict(status=None), dict(workspace=264)], ids=str)
def test_logprobs(S, more):
    have = ctypes.c_size_t(1 << 40)
    a = {**dict(dtype=1, rows=4, vocabulary=100, logits=256, stride=100, tokens=256, top=3, logprob=256, entropy=256, lse=256, top_tokens=256,
                top_logprobs=256, status=256, workspace=256), **more}
    assert S.lib.stalloc_token_logprobs(*a.values(), ctypes.byref(have), None) == INVALID


@pytest.mark.parametrize("more", [dict(dtype=3), dict(rows=0), dict(vocabulary=0), dict(logits=None), dict(tokens=None), dict(lse=None), dict(entropy=None),
                                  dict(d_logprob=None), dict(d_logits=None), dict(d_stride=99), dict(status=None), dict(d_logits=257)], ids=str)
def test_logprobs_backward(S, more):
    a = {**dict(dtype=1, rows=4, vocabulary=100, logits=256, stride=100, tokens=256, lse=256, entropy=256, d_logprob=256, d_entropy=256, d_logits=256,
                d_stride=100, status=256), **more}
    assert S.lib.stalloc_token_logprobs_backward(*a.values(), None) == INVALID


def test_clip(S):
    def call(entries, max_norm=1.0, k=None, norm=256, factor=256, workspace=256, nbytes=1 << 40):
        table = (S._Tensor * max(1, len(entries)))(*[S._Tensor(*e) for e in entries])
        have = ctypes.c_size_t(nbytes)
        return S.lib.stalloc_clip_gradients(table, len(entries) if k is None else k, max_norm, norm, factor, workspace, ctypes.byref(have), None)

    good = (256, 256, 10, 1)
    assert call([good], k=0) == INVALID
    for bad in ((256, 256, 10, 3), (None, 256, 10, 1), (257, 256, 10, 1), (256, 257, 10, 1), (256, 256, 1 << 42, 1)):
        assert call([good, bad]) == INVALID
    assert call([good], max_norm=-1.0) == INVALID and call([good], max_norm=float("nan")) == INVALID
    assert call([good], norm=None) == INVALID and call([good], factor=None) == INVALID
    assert call([good], workspace=264) == INVALID and call([good], nbytes=4) == INVALID
    assert call([good] * 300, workspace=None) == 0


def test_binding_refuses_what_is_not_on_the_gpu(S):
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    q = torch.zeros(4, 2, 8, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        S.stalloc_rms_norm(x, x[0])
    with pytest.raises(TypeError):
        S.stalloc_token_logprobs(x, i)
    with pytest.raises(TypeError):
        S.stalloc_attention(q, q, q, i)
    with pytest.raises(TypeError):
        S.stalloc_tensor_list([x])
    with pytest.raises(ValueError):
        S.stalloc_tensor_list([])
    with pytest.raises(ValueError):
        S.stalloc_token_logprobs(x, i, top=9)
