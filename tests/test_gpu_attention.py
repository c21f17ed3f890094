"""stalloc_attention and its backward pass against the definition in 64 bits; tolerances are bounds on the kernels' roundings
(plain_operators.attention)."""
import numpy as np
import pytest

import plain_operators as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    return S


def _inputs(seed, n, h, g, d, t, spread=1.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(n, (h + 2 * g) * d, generator=gen) * spread).to(t).cuda()
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split((h * d, g * d, g * d), dim=1))      # views into one projection
    d_o = torch.randn(n, h, d, generator=gen).to(t).cuda()
    return q, k, v, d_o


def _bounds(lengths):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()


def _close(got, want, slack, what):
    import torch
    got = got.double().cpu()
    if not got.numel():
        return
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine], want[~fine]), what
    over = ((got - want).abs() - slack).masked_fill(~fine, 0.0)
    assert float(over.max()) <= 0.0, (what, float(over.max()), float((got - want).abs().masked_fill(~fine, 0.0).max()))


def _check(S, q, k, v, d_o, bounds, scale=None, **more):
    import torch
    f = S.stalloc_attention(q, k, v, bounds, scale=scale, **more)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds, scale=scale, **more)
    torch.cuda.synchronize()
    S.check_status(f, "attention")
    S.check_status(b, "attention backward")
    cuts = bounds.cpu().tolist()
    want, slack = plain.attention(q, k, v, cuts, q.shape[2] ** -0.5 if scale is None else scale, d_o)
    for name in ("o", "lse"):
        _close(f[name], want[name], slack[name], name)
    for name in ("dq", "dk", "dv"):
        _close(b[name], want[name], slack[name], name)
    return f, b


LENGTHS = {
    "one_token": [1],
    "empty_ones": [0, 1, 0, 0, 5, 0],
    "around_32": [31, 32, 33],
    "around_64": [63, 64, 65, 1],
    "around_128": [127, 128, 129],
    "ragged": [3, 300, 1, 0, 77, 130],
    "long": [700],
    "many": [2, 0, 9, 1, 30] * 30,
}


@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(S, lengths, t, d):
    import torch
    lengths = LENGTHS[lengths]
    q, k, v, d_o = _inputs(len(lengths) + d, sum(lengths), 4, 2, d, getattr(torch, t))
    _check(S, q, k, v, d_o, _bounds(lengths))


@pytest.mark.parametrize("h,g,d", [(1, 1, 8), (3, 3, 16), (5, 1, 40), (8, 4, 56), (8, 1, 72), (6, 3, 80), (2, 2, 96), (9, 3, 120), (64, 8, 128)])
def test_heads(S, h, g, d):
    import torch
    q, k, v, d_o = _inputs(h * d, 150, h, g, d, torch.bfloat16)
    _check(S, q, k, v, d_o, _bounds([1, 149]))


@pytest.mark.parametrize("padding", [1, 64, 129, 300])
def test_padding_behind_the_last_sequence(S, padding):
    import torch
    q, k, v, d_o = _inputs(padding, 140 + padding, 4, 2, 64, torch.float16)
    for x in (q, k, v):
        x[140:] = float("nan")                                # what is there must not matter
    f, b = _check(S, q, k, v, d_o, _bounds([40, 100]))
    assert float(f["o"][140:].abs().max()) == 0.0 and bool((f["lse"][:, 140:] == -float("inf")).all())
    for name in ("dq", "dk", "dv"):
        assert float(b[name][140:].abs().max()) == 0.0
    nothing = _bounds([0, 0])                                 # no sequence has a token at all
    f, b = _check(S, q, k, v, d_o, nothing)
    assert float(f["o"].abs().max()) == 0.0 and float(b["dk"].abs().max()) == 0.0


def test_other_sequences_do_not_matter(S):
    """NaN and infinities in one sequence stay there."""
    import torch
    q, k, v, d_o = _inputs(3, 300, 4, 2, 64, torch.bfloat16)
    bounds = _bounds([100, 50, 150])
    for i, x in enumerate((q, k, v, d_o)):
        x[100 + i] = (float("nan"), float("inf"), float("-inf"), float("nan"))[i]
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    torch.cuda.synchronize()
    clean = [x.clone() for x in (q, k, v, d_o)]
    for x in clean:
        x[100:150] = 0.0
    want, slack = plain.attention(*clean[:3], [0, 100, 150, 300], 64 ** -0.5, clean[3])
    for name, got in (("o", f["o"]), ("dq", b["dq"]), ("dk", b["dk"]), ("dv", b["dv"])):
        for part in (slice(0, 100), slice(150, 300)):
            _close(got[part], want[name][part], slack[name][part], name)


def test_scores_that_grow_and_large_ones(S):
    """Keys in ascending order of their scores (the running maximum is raised again and again), scores of several hundred."""
    import torch
    q, k, v, d_o = _inputs(17, 400, 2, 1, 64, torch.float16)
    k.mul_(torch.linspace(0.0, 6.0, 400).view(-1, 1, 1).cuda().half())
    q.copy_(torch.where(q < 0, -q, q))
    k.copy_(torch.where(k < 0, -k, k))
    _check(S, q, k, v, d_o, _bounds([400]))
    _check(S, q, k, v, d_o, _bounds([130, 270]), scale=1.5)
    _check(S, q, k, v, d_o, _bounds([400]), scale=1e-3)


def test_layouts(S):
    """Heads before tokens, key heads that are one tensor expanded, outputs into views of a fused gradient."""
    import torch
    n, h, g, d = 200, 4, 2, 64
    q, k, v, d_o = _inputs(5, n, h, g, d, torch.bfloat16)
    bounds = _bounds([150, 50])
    by_head = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, d_o)]
    fused = torch.full((n, (h + 2 * g) * d), 7.0, dtype=torch.bfloat16, device="cuda")
    views = [x.unflatten(1, (-1, d)) for x in fused.split((h * d, g * d, g * d), dim=1)]
    f = S.stalloc_attention(*by_head[:3], bounds, out={"o": torch.empty(h, n, d, dtype=torch.bfloat16, device="cuda").transpose(0, 1)})
    b = S.stalloc_attention_backward(by_head[3], *by_head[:3], f["o"], f["lse"], bounds, out=dict(zip(("dq", "dk", "dv"), views)))
    torch.cuda.synchronize()
    want_f, want_b = _check(S, q, k, v, d_o, bounds)
    assert torch.equal(f["o"], want_f["o"]) and torch.equal(f["lse"], want_f["lse"])
    for name, view in zip(("dq", "dk", "dv"), views):
        assert b[name] is view and torch.equal(view, want_b[name])
    one = k[:, :1].expand(n, g, d)
    _check(S, q, one, v, d_o, bounds)


def test_offsets_beyond_32_bits(S):
    """Rows 12 M numbers apart: the last ones lie 2.4 G numbers behind the first."""
    import torch
    n, d, far = 200, 64, 12 << 20
    q, k, v, d_o = _inputs(6, n, 2, 1, d, torch.bfloat16)
    wide = torch.empty(n * far, dtype=torch.bfloat16, device="cuda")
    strided = [wide.as_strided((n, x.shape[1], d), (far, d, 1), i * 1024) for i, x in enumerate((q, k, v, d_o, q, q, k, v))]
    for to, x in zip(strided, (q, k, v, d_o)):
        to.copy_(x)
    bounds = _bounds([n])
    f = S.stalloc_attention(*strided[:3], bounds, out={"o": strided[4]})
    b = S.stalloc_attention_backward(strided[3], *strided[:3], f["o"], f["lse"], bounds, out=dict(zip(("dq", "dk", "dv"), strided[5:])))
    want_f, want_b = _check(S, q, k, v, d_o, bounds)
    assert torch.equal(f["o"], want_f["o"])
    for name in ("dq", "dk", "dv"):
        assert torch.equal(b[name], want_b[name])


def test_same_result_every_time_on_any_stream(S):
    import torch
    q, k, v, d_o = _inputs(8, 500, 8, 2, 64, torch.bfloat16)
    bounds = _bounds([260, 3, 237])
    first, grads = _check(S, q, k, v, d_o, bounds)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        f = S.stalloc_attention(q, k, v, bounds, stream=stream)
        b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds, stream=stream)
        stream.synchronize()
        assert torch.equal(f["o"], first["o"]) and torch.equal(f["lse"], first["lse"])
        assert all(torch.equal(b[name], grads[name]) for name in ("dq", "dk", "dv"))


def test_gradient_against_differences(S):
    """The loss sum(o * d_o) moved along a random direction, differences in 64 bits: the directional derivative within what the
    gradient's own roundings allow."""
    import torch
    n, h, g, d = 90, 4, 2, 32
    q, k, v, d_o = _inputs(11, n, h, g, d, torch.float16)
    bounds = _bounds([50, 40])
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    _, slack = plain.attention(q, k, v, [0, 50, 90], d ** -0.5, d_o)
    gen = torch.Generator().manual_seed(1)
    host = [x.double().cpu() for x in (q, k, v)]
    up, step = d_o.double().cpu(), 1e-5

    def loss(x):
        o, _ = plain.attention(*x, [0, 50, 90], d ** -0.5)
        return float((o["o"] * up).sum())

    for i, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(host[i].shape, generator=gen, dtype=torch.float64)
        moved = [[x + s * step * way if j == i else x for j, x in enumerate(host)] for s in (1.0, -1.0)]
        slope = (loss(moved[0]) - loss(moved[1])) / (2 * step)
        got = float((b[name].double().cpu() * way).sum())
        allowed = float((slack[name] * way.abs()).sum()) + 1e-5 * abs(slope) + 1e-4        # (and the differences' own error)
        assert abs(got - slope) <= allowed, (name, got, slope, allowed)


@pytest.mark.parametrize("cuts", [[1, 20, 60], [0, 40, 20], [0, 20, 61], [0, 1 << 30, 60], [-1, 20, 60], [0, -5, 60]])
def test_bad_bounds_are_reported(S, cuts):
    import torch
    q, k, v, d_o = _inputs(1, 60, 2, 1, 64, torch.bfloat16)
    bounds = torch.tensor(cuts, dtype=torch.int32).cuda()
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    torch.cuda.synchronize()
    assert int(f["status"].item()) == 10 and int(b["status"].item()) == 10
    with pytest.raises(S.StallocError, match="STALLOC_ERR_BAD_BOUNDS"):
        S.check_status(f)


def _lengths(seed, count, most):
    rng = np.random.default_rng(seed)
    return [int(n) for n in np.exp(rng.uniform(0.0, np.log(most), count))]


@pytest.mark.parametrize("seed,count,most,pad", [(1, 40, 900, 0), (2, 700, 60, 130), (3, 3000, 3, 1)])
def test_batches_whose_pieces_are_listed(S, seed, count, most, pad):
    """Enough pieces and heads for the list that puts the longest walks first (more sequences than a workgroup looks at in one go
    among them): sequences from all over the batch against the definition."""
    import torch
    lengths = _lengths(seed, count, most)
    lengths[3:5] = [0, 0]
    n, h, g, d = sum(lengths) + pad, 64, 4, 64
    q, k, v, d_o = _inputs(seed, n, h, g, d, torch.bfloat16)
    bounds = _bounds(lengths)
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    torch.cuda.synchronize()
    S.check_status(f)
    S.check_status(b)
    assert f["workspace"].numel() > 256                       # (the list is in it: 16 bytes a piece)
    cuts = bounds.cpu().tolist()
    for s in range(0, count, max(1, count // 9)):
        lo, hi = cuts[s], cuts[s + 1]
        if lo == hi:
            continue
        want, slack = plain.attention(q[lo:hi], k[lo:hi], v[lo:hi], [0, hi - lo], d ** -0.5, d_o[lo:hi])
        _close(f["o"][lo:hi], want["o"], slack["o"], "o")
        _close(f["lse"][:, lo:hi], want["lse"], slack["lse"], "lse")
        for name in ("dq", "dk", "dv"):
            _close(b[name][lo:hi], want[name], slack[name], name)
    if pad:
        assert float(f["o"][n - pad:].abs().max()) == 0.0 and float(b["dk"][n - pad:].abs().max()) == 0.0
    cuts[2] = n + 5
    bad = torch.tensor(cuts, dtype=torch.int32).cuda()
    assert int(S.stalloc_attention(q, k, v, bad)["status"].item()) == 10


@pytest.mark.parametrize("d", [64, 128, 80])
@pytest.mark.parametrize("at", [0, 1, 31, 32, 70, 127, 128, 199])
def test_later_tokens_do_not_matter(S, d, at):
    """NaN and infinities in what a later token stands for reach neither the output nor the gradients of earlier ones: rows that do not see
    the token at `at`, and keys that it does not see, are what they are without it."""
    import torch
    n, h, g = 200, 4, 2
    t = torch.float16 if at % 2 else torch.bfloat16
    q, k, v, d_o = _inputs(at + d, n, h, g, d, t)
    bounds = _bounds([n])
    _, clean = _check(S, q, k, v, d_o, bounds)
    want, slack = plain.attention(q, k, v, [0, n], d ** -0.5, d_o)
    for which, bad in ((1, float("nan")), (2, float("inf")), (2, float("-inf")), (2, float("nan")), (3, float("nan")), (3, float("inf")), (0, float("nan"))):
        x = [y.clone() for y in (q, k, v, d_o)]
        x[which][at, 0, 3] = bad
        f = S.stalloc_attention(*x[:3], bounds)
        b = S.stalloc_attention_backward(x[3], *x[:3], f["o"], f["lse"], bounds)
        torch.cuda.synchronize()
        if which in (1, 2):                                    # k or v of token `at`: rows before it do not see it
            _close(f["o"][:at], want["o"][:at], slack["o"][:at], "o")
            _close(b["dq"][:at], want["dq"][:at], slack["dq"][:at], "dq")
            if which == 2:                                     # v: rows that see it have it where it is, as it is
                seen = f["o"][at:, :h // g].float().cpu()      # (the heads that read key head 0)
                assert bool((torch.isnan(seen[:, :, 3]) if bad != bad else seen[:, :, 3] == bad).all())
                assert bool(torch.isfinite(seen[:, :, [0, 1, 2, 4, 5]]).all()) and bool(torch.isfinite(f["o"][:, h // g:]).all())
            else:
                assert bool(torch.isnan(f["o"][at:, :h // g]).all())
        else:                                                  # q or d_o of row `at`: keys behind it are not seen by it
            for name in ("dk", "dv"):
                _close(b[name][at + 1:], want[name][at + 1:], slack[name][at + 1:], name)
            _close(b["dq"][:at], want["dq"][:at], slack["dq"][:at], "dq")
            if which == 3:                                     # d_o: keys that the row sees have it in dv
                got = b["dv"][:at + 1, 0, 3].float().cpu()
                assert bool((torch.isnan(got) if bad != bad else got == bad).all())
        assert bool(torch.isfinite(b["dk"][:, 1:]).all()) and bool(torch.isfinite(b["dq"][:, h // g:]).all())      # the other key head


@pytest.mark.parametrize("h,g,d,lengths", [(1, 1, 128, [1300]), (2, 1, 64, [2100]), (3, 3, 80, [1025, 700]), (4, 1, 128, [900, 0, 40, 1100]), (8, 1, 64, [600])])
def test_walks_cut_into_parts(S, h, g, d, lengths):
    """Few heads and long sequences: walks over keys and rows are cut into parts, some of them empty, padding behind them; with infinities and
    NaN in later tokens, which earlier ones do not see, in any part."""
    import torch
    n = sum(lengths) + 130
    q, k, v, d_o = _inputs(n, n, h, g, d, torch.bfloat16)
    bounds = _bounds(lengths)
    f, b = _check(S, q, k, v, d_o, bounds)
    assert f["workspace"].numel() >= (8 * n * h * d if lengths[0] > 1200 else 0) and b["workspace"].numel() > 4 * n * h * d     # (parts' sums are in it)
    again = S.stalloc_attention(q, k, v, bounds)
    assert torch.equal(again["o"], f["o"])
    want, slack = plain.attention(q, k, v, bounds.cpu().tolist(), d ** -0.5, d_o)
    at = lengths[0] - 3
    for x in (k, v):
        x[at, 0, 1] = float("nan")
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    for name, got in (("o", f["o"]), ("dq", b["dq"])):
        _close(got[:at], want[name][:at], slack[name][:at], name)
        _close(got[lengths[0]:], want[name][lengths[0]:], slack[name][lengths[0]:], name)
