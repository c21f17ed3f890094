"""stalloc_token_logprobs and its backward pass against the definition in 64 bits.  Tolerances (32-bit sums): z is a sum of `vocabulary` positive
numbers, each good to a few roundings of its exponent's argument, so ln z is good to that many relative roundings of z; orders are exact."""
import pytest

import plain_operators as plain

pytestmark = pytest.mark.gpu
F32, INF = 2.0 ** -24, float("inf")


@pytest.fixture(scope="module")
def S():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    return S


def _inputs(seed, rows, vocabulary, t, spread=3.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, vocabulary, generator=gen) * spread).to(t)
    tokens = torch.randint(vocabulary, (rows,), generator=gen, dtype=torch.int32)
    return x, tokens, torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)


def _ln_z(vocabulary, away):
    """Relative error of z: additions in 32 bits in chains of at most vocabulary / 256 + 40, arguments of up to `away` rounded twice."""
    return (vocabulary / 256 + 40) * F32 + 4 * F32 * away


def _check(S, x, tokens, top, d_logprob=None, d_entropy=None, **more):
    import torch
    dev = x.cuda()
    got = S.stalloc_token_logprobs(dev, tokens.cuda(), top=top, **more)
    torch.cuda.synchronize()
    S.check_status(got)
    want = plain.token_logprobs(x, tokens, max(top, 1))
    finite = torch.where(torch.isfinite(x), x.double(), 0.0)
    away = float((finite.amax() - finite.amin()).abs()) if x.numel() else 0.0
    away = min(away, 120.0)                                       # (further off than that nothing is left of a term)
    rel = _ln_z(x.shape[1], away)

    def near(a, b, allowed):
        a = a.double().cpu()
        assert torch.equal(torch.isfinite(a), torch.isfinite(b)) and torch.equal(a[~torch.isfinite(a)], b[~torch.isfinite(b)])
        off = torch.where(torch.isfinite(b), (a - b).abs(), 0.0)
        assert bool((off <= allowed * (1.0 + b.abs().masked_fill(~torch.isfinite(b), 0.0)) ).all()), float(off.max())

    near(got["lse"], want[2], rel + 4 * F32)
    near(got["logprob"], want[0], rel + 4 * F32)
    near(got["entropy"], want[1], (2 * rel + 8 * F32) * (1.0 + away))
    if top:
        assert torch.equal(got["top_tokens"].long().cpu(), want[3])
        near(got["top_logprobs"], want[4], rel + 4 * F32)
    if d_logprob is not None:
        b = S.stalloc_token_logprobs_backward(dev, tokens.cuda(), got["lse"], got["entropy"], d_logprob.cuda(),
                                              None if d_entropy is None else d_entropy.cuda())
        torch.cuda.synchronize()
        S.check_status(b)
        d = plain.token_logprobs_backward(x, tokens, d_logprob, d_entropy)
        size = d_logprob.double().abs()[:, None] + (0.0 if d_entropy is None else d_entropy.double().abs()[:, None] * (1.0 + away + want[1][:, None]))
        m = x.double().amax(-1, keepdim=True)
        m = m.masked_fill(m == -INF, 0.0)
        p = torch.exp(x.double() - m)
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
        allowed = plain.half(x.dtype) * d.abs() * 1.01 + (2 * rel + 16 * F32 * (1 + away)) * size * (p + 1e-6) + torch.finfo(x.dtype).tiny * 2 * plain.half(x.dtype)
        allowed = allowed + 4 * F32 * d.abs()
        off = (b["d_logits"].double().cpu() - d).abs()
        assert bool((off <= allowed).all()), float((off - allowed).max())
    return got


SHAPES = [(1, 1), (2, 2), (3, 7), (1, 8), (4, 100), (2, 2047), (2, 2048), (3, 2049), (5, 4097), (2, 8192), (1, 50257), (3, 70001), (300, 997), (2100, 260)]


@pytest.mark.parametrize("rows,vocabulary", SHAPES)
@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
def test_forward_and_backward(S, rows, vocabulary, t):
    import torch
    x, tokens, g, h = _inputs(rows * vocabulary, rows, vocabulary, getattr(torch, t))
    if rows > 2:
        tokens[1] = -1
    _check(S, x, tokens, min(vocabulary, 9), g, h)
    _check(S, x, tokens, 0, g, None)


@pytest.mark.parametrize("top", [1, 2, 31, 64])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_top(S, rows, top):
    import torch
    x, tokens, _, _ = _inputs(top, rows, 9001, torch.bfloat16)       # (thousands of ties among 9001 numbers of 8 bits)
    _check(S, x, tokens, top)


def test_ties_and_orders(S):
    """All equal; ascending; descending; the best ones next to each other; the best ones a workgroup's stride apart."""
    import torch
    v = 20000
    x = torch.zeros(6, v)
    x[1] = torch.arange(v) * 0.01
    x[2] = -torch.arange(v) * 0.01
    x[3, 8000:8064] = 5.0
    x[4, 5::2048] = 7.0
    x[5, 3] = -0.0                                                   # equals the zeros around it
    tokens = torch.tensor([0, v - 1, 0, 8010, 5, 3], dtype=torch.int32)
    for t in (torch.float32, torch.float16):
        _check(S, x.to(t), tokens, 64)


@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
def test_masked_numbers(S, t):
    """-infinity, the type's lowest value, rows of nothing else, a single number left, targets that are masked."""
    import torch
    t = getattr(torch, t)
    x, tokens, g, h = _inputs(9, 8, 5000, t)
    low = torch.finfo(t).min
    x[0, 100:] = -INF
    x[1, :] = -INF
    x[2, :] = low
    x[3, 1:] = low
    x[4, :] = -INF
    x[4, 4321] = 2.0
    x[5, :2500] = low
    x[6, :] = -INF
    x[6, 7] = low
    x[6, 4000] = low
    tokens = torch.tensor([5, 3, 8, 0, 4321, 3000, 7, 1], dtype=torch.int32)
    _check(S, x, tokens, 5, g, h)
    tokens[0] = 4000                                                 # cannot occur
    got = S.stalloc_token_logprobs(x.cuda(), tokens.cuda(), top=5)
    assert float(got["logprob"][0]) == -INF and float(got["logprob"][1]) == -INF and float(got["entropy"][1]) == 0.0


def test_numbers_that_are_not_numbers_stay_in_their_row(S):
    import torch
    x, tokens, g, h = _inputs(4, 5, 3001, torch.float32)
    clean = S.stalloc_token_logprobs(x.cuda(), tokens.cuda(), top=4)
    y = x.clone()
    y[1, 17] = float("nan")
    y[3, 2900] = INF
    got = S.stalloc_token_logprobs(y.cuda(), tokens.cuda(), top=4)
    for name in ("logprob", "entropy", "lse", "top_tokens"):
        assert torch.equal(got[name][[0, 2, 4]], clean[name][[0, 2, 4]])
    assert bool(torch.isnan(got["lse"][1])) and not bool(torch.isfinite(got["lse"][3]))
    back = S.stalloc_token_logprobs_backward(y.cuda(), tokens.cuda(), got["lse"], got["entropy"], g.cuda(), h.cuda())["d_logits"]
    assert bool(torch.isnan(back[1]).all()) and bool(torch.isfinite(back[[0, 2, 4]]).all())


def test_strided_rows_and_gradients_in_place(S):
    import torch
    rows, v = 40, 5003
    x, tokens, g, h = (z.cuda() for z in _inputs(12, rows, v, torch.bfloat16))
    f = S.stalloc_token_logprobs(x, tokens, top=3)
    want = S.stalloc_token_logprobs_backward(x, tokens, f["lse"], f["entropy"], g, h)["d_logits"]
    wide = torch.full((rows, v + 29), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = wide[:, :v]
    view.copy_(x)
    got = S.stalloc_token_logprobs(view, tokens, top=3)
    assert all(torch.equal(got[name], f[name]) for name in ("logprob", "entropy", "lse", "top_tokens", "top_logprobs"))
    back = S.stalloc_token_logprobs_backward(view, tokens, f["lse"], f["entropy"], g, h, out={"d_logits": view})["d_logits"]
    assert back is view and torch.equal(view, want) and bool(torch.isnan(wide[:, v:]).all())


def test_tokens_beyond_the_vocabulary_are_reported(S):
    import torch
    for rows in (1, 7, 3000):
        x, tokens, g, _ = (z.cuda() for z in _inputs(2, rows, 300, torch.float16))
        tokens[rows - 1] = 300
        f = S.stalloc_token_logprobs(x, tokens)
        b = S.stalloc_token_logprobs_backward(x, tokens, f["lse"], f["entropy"], g)
        torch.cuda.synchronize()
        assert int(f["status"].item()) == 11 and int(b["status"].item()) == 11
    with pytest.raises(S.StallocError, match="STALLOC_ERR_BAD_TOKEN"):
        S.check_status(f)


def test_gradient_against_differences(S):
    import torch
    x, tokens, g, h = _inputs(21, 6, 50, torch.float32, spread=1.0)
    f = S.stalloc_token_logprobs(x.cuda(), tokens.cuda())
    b = S.stalloc_token_logprobs_backward(x.cuda(), tokens.cuda(), f["lse"], f["entropy"], g.cuda(), h.cuda())
    way, step = torch.randn(x.shape, generator=torch.Generator().manual_seed(1), dtype=torch.float64), 1e-6

    def loss(z):
        lp, entropy = plain.token_logprobs(z, tokens, 1)[:2]
        return float((lp * g.double()).sum() + (entropy * h.double()).sum())

    slope = (loss(x.double() + step * way) - loss(x.double() - step * way)) / (2 * step)
    assert abs(float((b["d_logits"].double().cpu() * way).sum()) - slope) <= 1e-4 * (1.0 + abs(slope))


def test_logits_beyond_the_caches(S):
    """256 MiB and more go past the caches, in rows of an odd number of elements: rows spread over the tensor against the definition, and a
    gradient in place of the logits."""
    import torch
    rows, v = 1400, 100003
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(rows, v, device="cuda", dtype=torch.bfloat16).normal_(0.0, 2.0, generator=gen)
    tokens = torch.randint(v, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.randn(rows, device="cuda", generator=gen)
    some = torch.tensor([0, 1, 700, 1398, 1399])
    f = S.stalloc_token_logprobs(x, tokens, top=3)
    kept = x[some.cuda()].cpu()
    small = _check(S, kept, tokens.cpu()[some], 3, g.cpu()[some])
    for name in ("logprob", "entropy", "lse", "top_tokens", "top_logprobs"):
        a, b = f[name][some.cuda()].double().cpu(), small[name].double().cpu()
        assert bool(((a - b).abs() <= 2e-6 * (1.0 + b.abs())).all())           # (rows that are few are cut into parts: another order of sums)
    want = S.stalloc_token_logprobs_backward(x[some.cuda()], tokens[some.cuda()], f["lse"][some.cuda()], f["entropy"][some.cuda()], g[some.cuda()])["d_logits"]
    back = S.stalloc_token_logprobs_backward(x, tokens, f["lse"], f["entropy"], g, out={"d_logits": x})["d_logits"]
    assert torch.equal(back[some.cuda()], want)
