"""Attention of rows whose scores are infinite, or finite and so large that 32 bits of their sum say little: what the definition gives, or NaN where it gives none; never zeros."""
import numpy as np
import pytest

import plain_operators as plain
from test_gpu_attention import _bounds, _close, _inputs

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def S():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    return S


def _both(S, q, k, v, d_o, bounds):
    import torch
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    torch.cuda.synchronize()
    S.check_status(f)
    S.check_status(b)
    return f, b


SHAPES = [(4, 2, 64, [200]), (4, 2, 128, [70, 130]), (2, 1, 80, [150]), (1, 1, 128, [1300]), (3, 3, 80, [1025, 700])]      # (the last two: walks cut into parts)


@pytest.mark.parametrize("h,g,d,lengths", SHAPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("t", ["bfloat16", "float16"])
def test_an_infinity_in_a_query(S, t, sign, h, g, d, lengths):
    """Every score of the row is infinite: with one sign alone (the first token, which sees one key) as with both.  The row's output is NaN, and so is what it hands back; other rows are as
    they are without it."""
    import torch
    n = sum(lengths)
    q, k, v, d_o = _inputs(n + h, n, h, g, d, getattr(torch, t))
    bounds, cuts = _bounds(lengths), np.concatenate([[0], np.cumsum(lengths)])
    want, slack = plain.attention(q, k, v, cuts.tolist(), d ** -0.5, d_o)
    for at in (0, 1, 33, lengths[0] - 1):
        bad = q.clone()
        bad[at, 0, 3] = sign * INF * float(torch.sign(k[0, 0, 3]))            # (the first token's score has this sign)
        f, b = _both(S, bad, k, v, d_o, bounds)
        assert bool(torch.isnan(f["o"][at, 0]).all()) and not bool(torch.isfinite(f["lse"][0, at]))
        if at == 0 and sign < 0.0:
            assert float(f["lse"][0, 0]) == -INF
        assert bool(torch.isnan(b["dq"][at, 0]).all())
        assert bool(torch.isnan(b["dk"][: at + 1, 0]).all()) and bool(torch.isnan(b["dv"][: at + 1, 0]).all())
        rest = [i for i in range(n) if i != at]
        _close(f["o"][rest], want["o"][rest], slack["o"][rest], "o")
        _close(f["lse"][:, rest], want["lse"][:, rest], slack["lse"][:, rest], "lse")
        _close(b["dq"][rest], want["dq"][rest], slack["dq"][rest], "dq")
        for name in ("dk", "dv"):
            _close(b[name][at + 1:], want[name][at + 1:], slack[name][at + 1:], name)
            if g > 1:
                _close(b[name][:, 1:], want[name][:, 1:], slack[name][:, 1:], name)


def test_scores_that_are_all_minus_infinity(S):
    """Of every row: nothing is left of the whole sequence, and the one behind it is not concerned."""
    import torch
    q, k, v, d_o = _inputs(5, 190, 2, 1, 64, torch.bfloat16)
    q[:100, :, 0] = 1.0
    k[:100, :, 0] = -INF
    f, b = _both(S, q, k, v, d_o, _bounds([100, 90]))
    assert bool((f["lse"][:, :100] == -INF).all())
    for got in (f["o"], b["dq"], b["dk"], b["dv"]):
        assert bool(torch.isnan(got[:100]).all()) and bool(torch.isfinite(got[100:]).all())


def _definition(q, k, v, d_o, cuts, scale):
    """o, lse, dq, dk, dv and sum |p| |v| in 64 bits, one head."""
    import torch
    q, k, v, d_o = (x[:, 0].double().cpu() for x in (q, k, v, d_o))
    out = [torch.zeros_like(q), torch.zeros(q.shape[0], dtype=torch.float64)] + [torch.zeros_like(q) for _ in range(4)]
    for a, b in zip(cuts, cuts[1:]):
        s = (q[a:b] @ k[a:b].T * scale).masked_fill(torch.ones(b - a, b - a, dtype=torch.bool).triu(1), -INF)
        p = torch.softmax(s, -1)
        o = p @ v[a:b]
        ds = p * (d_o[a:b] @ v[a:b].T - (d_o[a:b] * o).sum(-1, keepdim=True)) * scale
        for x, y in zip(out, (o, torch.logsumexp(s, -1), ds @ k[a:b], ds.T @ q[a:b], p.T @ d_o[a:b], p @ v[a:b].abs())):
            x[a:b] = y
    return out


def _off(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("lengths", [[1], [150, 60], [1300]], ids=str)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("power", [24, 60, 100, 125])
def test_scores_beyond_everything(S, power, sign, lengths):
    """One column makes scores of 2^power and more, the rest of q is 0: weights are shared by the keys whose score is the largest, equal ones.  Scores are exact; weights are
    rounded to bfloat16 (u) and their sum's logarithm, about 8, kept to 2^-15."""
    import torch
    n, d, t = sum(lengths), 64, torch.bfloat16
    _, k, v, d_o = _inputs(power, n, 1, 1, d, t)
    q = torch.zeros(n, 1, d, dtype=t, device="cuda")
    q[:, 0, 0] = sign * 2.0 ** (power // 2)
    gen = torch.Generator().manual_seed(power)
    k[:, 0, 0] = (2.0 ** (power - power // 2) * torch.tensor([1.0, 1.0, 1.5, 1.75])[torch.randint(4, (n,), generator=gen)]).to(t).cuda()
    cuts = [0] + np.cumsum(lengths).tolist()
    o, lse, dq, dk, dv, size = _definition(q, k, v, d_o, cuts, d ** -0.5)
    f, b = _both(S, q, k, v, d_o, _bounds(lengths))
    u = plain.half(t)
    assert bool(((f["o"][:, 0].double().cpu() - o).abs() <= (2.1 * u + 2.0 ** -12) * size).all())
    assert bool(((f["lse"][0].double().cpu() - lse).abs() <= 2.0 ** -22 * lse.abs()).all())
    assert _off(b["dv"][:, 0], dv) <= 2 * u
    if n > 1:                                                    # (ds has no more than its own rounding and D's, from the rounded o; sum_j ds_ij is 0: column 0 of dq is all rounding)
        assert _off(b["dq"][:, 0, 1:], dq[:, 1:]) <= 4 * u
        assert _off(b["dk"][:, 0, 0], dk[:, 0]) <= 4 * u
    else:
        assert torch.equal(b["dv"], d_o) and torch.equal(f["o"], v)


@pytest.mark.parametrize("lengths", [[150, 60], [1300]], ids=str)
@pytest.mark.parametrize("large", [0, 2 ** 18, 2 ** 20, 2 ** 23])
@pytest.mark.parametrize("t", ["bfloat16", "float16"])
def test_a_constant_in_every_score(S, t, large, lengths):
    """It changes nothing but lse, and lse is what the backward pass has: whole numbers, so that scores are exact in 32 bits, the constant from one column.  Up to 2^16 (of the scaled
    score in units of log 2) weights carry the rounding of lse, 2^-23 of it; beyond that those of their own sum, 2^-15 of its logarithm."""
    import torch
    n, d, t = sum(lengths), 64, getattr(torch, t)
    gen = torch.Generator().manual_seed(3)
    q, k = ((torch.randint(-2, 3, (n, 1, d), generator=gen)).to(t).cuda() for _ in range(2))
    _, _, v, d_o = _inputs(7, n, 1, 1, d, t)
    q[:, 0, 0] = 2.0 ** 11 if large else 0.0
    k[:, 0, 0] = large / 2.0 ** 11
    cuts = [0] + np.cumsum(lengths).tolist()
    o, lse, dq, dk, dv, size = _definition(q, k, v, d_o, cuts, d ** -0.5)
    f, b = _both(S, q, k, v, d_o, _bounds(lengths))
    u, carried = plain.half(t), 2.0 ** -7 * 0.7
    assert bool(((f["o"][:, 0].double().cpu() - o).abs() <= (2.1 * u + 2.0 ** -12) * size).all())
    assert bool(((f["lse"][0].double().cpu() - lse).abs() <= 2.0 ** -22 * (1.0 + lse.abs())).all())
    assert _off(b["dv"][:, 0], dv) <= 2 * u + carried
    assert _off(b["dq"][:, 0, 1:], dq[:, 1:]) <= 4 * u + 2 * carried
    assert _off(b["dk"][:, 0, 1:], dk[:, 1:]) <= 4 * u + 2 * carried


def test_large_scores_beside_numbers_that_are_not_finite(S):
    """An infinity in the last value: the rows before it are walked pair by pair, with scores of 2^60 in a sum of their own."""
    import torch
    n, d, t = 180, 64, torch.bfloat16
    _, k, v, d_o = _inputs(2, n, 1, 1, d, t)
    q = torch.zeros(n, 1, d, dtype=t, device="cuda")
    q[:, 0, 0] = 2.0 ** 30
    k[:, 0, 0] = (2.0 ** 30 * (1.0 + torch.arange(n) % 3)).to(t).cuda()
    o, _, dq, _, _, size = _definition(q, k, v, d_o, [0, n], d ** -0.5)
    v[n - 1, 0, 5] = INF
    f, b = _both(S, q, k, v, d_o, _bounds([n]))
    u = plain.half(t)
    assert bool(((f["o"][: n - 1, 0].double().cpu() - o[: n - 1]).abs() <= (2.1 * u + 2.0 ** -12) * size[: n - 1]).all())
    assert _off(b["dq"][: n - 1, 0, 1:], dq[: n - 1, 1:]) <= 4 * u
