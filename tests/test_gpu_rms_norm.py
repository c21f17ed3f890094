"""stalloc_rms_norm and its backward pass against the definition in 64 bits.  Tolerances: y is rounded once to its type; before that the sum
of squares has at most `width` additions in 32 bits (relative to a sum of positive numbers), a root, a division and three products."""
import pytest

import plain_operators as plain

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -24


@pytest.fixture(scope="module")
def S():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    return S


def _inputs(seed, rows, width, t, spread=1.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    make = lambda *shape: (torch.randn(*shape, generator=gen) * spread).to(t)                # noqa: E731
    return make(rows, width), make(rows, width), (1.0 + 0.3 * torch.randn(width, generator=gen)).to(t), make(rows, width), make(rows, width)


def _rel(width):
    return (width + 8) * F32 / 2 + 8 * F32


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 127), (2, 128), (9, 129), (70, 512), (4, 1000), (6, 1024), (5, 1025), (33, 2048), (3, 4095), (4, 4096),
          (2, 8192), (2, 8193), (2, 20000), (2, 32768), (3, 32769), (1, 50000)]


@pytest.mark.parametrize("rows,width", SHAPES)
@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
def test_forward(S, rows, width, t):
    import torch
    t = getattr(torch, t)
    x, r, w, _, _ = _inputs(rows + width, rows, width, t)
    for residual in (None, r):
        want_sum, want_rstd, want_y = plain.rms_norm(x, residual, w, 1e-5)
        got = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=None if residual is None else r.cuda(), eps=1e-5)
        assert torch.equal(got["sum"].cpu(), want_sum)
        assert float(((got["rstd"].double().cpu() - want_rstd).abs() / want_rstd).max()) <= _rel(width)
        allowed = (plain.half(t) + _rel(width) + 2 * F32) * want_y.abs() + torch.finfo(t).tiny * 2 * plain.half(t)
        assert float(((got["y"].double().cpu() - want_y).abs() - allowed).max()) <= 0.0


@pytest.mark.parametrize("rows,width", SHAPES)
@pytest.mark.parametrize("t", ["float32", "bfloat16"])
def test_eight_bits(S, rows, width, t):
    """Scales to 32-bit accuracy; every number within half a step of e4m3 (2^-4 relative, 2^-10 absolute below its normal range)."""
    import torch
    t = getattr(torch, t)
    x, r, w, _, _ = _inputs(rows * 3 + width, rows, width, t)
    if rows > 1:
        x[1, : min(width, 128)] = 0.0
        r[1, : min(width, 128)] = 0.0                             # a block of zeros
    _, _, y = plain.rms_norm(x, r, w, 1e-5)
    want = plain.eight_bits(y)
    got = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), eps=1e-5, eight_bits=True)
    assert "y" not in got
    scales, q = got["scales"].double().cpu(), got["q"].cpu().double()
    rel = _rel(width) + 8 * F32
    assert float(((scales - want).abs() / want).max()) <= rel
    spread = scales.repeat_interleave(128, 1)[:, :width]
    allowed = (2.0 ** -4 * (1 + 2.0 ** -4) + rel) * y.abs() + 2.0 ** -10 * spread
    assert float(((q * spread - y).abs() - allowed).max()) <= 0.0
    both = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), eps=1e-5, eight_bits=True, out={"y": torch.empty(rows, width, dtype=t, device="cuda")})
    assert torch.equal(both["q"].view(torch.uint8), got["q"].view(torch.uint8))
    assert torch.equal(both["y"], S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), eps=1e-5)["y"])


def test_eight_bits_of_numbers_that_are_not_finite(S):
    """They mark their block of 128 columns (and, since they are in its norm, the row's every number) and no other row."""
    import torch
    x, r, w, _, _ = _inputs(1, 4, 300, torch.float32)
    x[1, 5] = float("nan")
    x[2, 200] = float("inf")
    w[299] = float("inf")                                         # the last block of every row: infinite there
    got = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), eight_bits=True)
    value = got["q"].cpu().float() * got["scales"].cpu().repeat_interleave(128, 1)[:, :300]
    assert bool(torch.isfinite(value[0, :256]).all()) and bool(torch.isnan(value[0, 256:]).all())
    assert bool(torch.isnan(value[1]).all()) and bool(torch.isfinite(value[3, :256]).all())


def test_strided_rows_and_sums_in_place(S):
    import torch
    rows, width, t = 37, 1000, torch.bfloat16
    x, r, w, _, _ = _inputs(4, rows, width, t)
    want = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda())
    for pad in (1, 8, 13):
        wide = torch.full((rows, width + pad), float("nan"), dtype=t, device="cuda")
        wide[:, :width] = x.cuda()
        stream = r.cuda()
        got = S.stalloc_rms_norm(wide[:, :width], w.cuda(), residual=stream, out={"sum": stream})
        assert got["sum"] is stream and torch.equal(stream, want["sum"]) and torch.equal(got["y"], want["y"])
    shifted = torch.empty(rows * width + 1, dtype=t, device="cuda")[1:].view(rows, width)     # rows at odd multiples of two bytes
    shifted.copy_(x)
    assert torch.equal(S.stalloc_rms_norm(shifted, w.cuda(), residual=r.cuda())["y"], want["y"])


@pytest.mark.parametrize("rows,width", SHAPES + [(3000, 512), (1500, 1100), (300, 9000), (70, 40000)])
@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
def test_backward(S, rows, width, t):
    """dx: three terms, each with the relative errors of rstd and of c (a sum of `width` products, relative to the sum of their magnitudes).
    dweight: a sum over the rows, in 32 bits."""
    import torch
    t = getattr(torch, t)
    x, r, w, d_y, d_sum = _inputs(rows + 7 * width, rows, width, t)
    f = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda())
    s, rstd = f["sum"].cpu(), f["rstd"].double().cpu()
    exact = 1.0 / torch.sqrt((s.double() ** 2).mean(-1) + 1e-6)
    for through in (None, d_sum):
        want, want_w = plain.rms_norm_backward(d_y, s, w, exact, through)
        b = S.stalloc_rms_norm_backward(d_y.cuda(), f["sum"], w.cuda(), f["rstd"], d_sum=None if through is None else through.cuda())
        g, q = (w.double() * d_y.double()), exact[:, None]
        c_abs = (g * s.double()).abs().mean(-1, keepdim=True)
        rel = _rel(width) * 4 + (width + 8) * F32
        parts = q * g.abs() + q ** 3 * s.double().abs() * c_abs
        allowed = (rel * parts + plain.half(t) * want.abs()) * (1 + plain.half(t)) + 4 * F32 * (parts + want.abs()) + torch.finfo(t).tiny * 2 * plain.half(t)
        assert float(((b["dx"].double().cpu() - want).abs() - allowed).max()) <= 0.0
        allowed = (rows * F32 + _rel(width) + 4 * F32) * (d_y.double() * s.double() * q).abs().sum(0)
        assert float(((b["dweight"].double().cpu() - want_w).abs() - allowed).max()) <= 0.0


def test_backward_in_place_and_repeated(S):
    import torch
    rows, width = 900, 2000
    x, r, w, d_y, d_sum = (z.cuda() for z in _inputs(3, rows, width, torch.bfloat16))
    f = S.stalloc_rms_norm(x, w, residual=r)
    want = S.stalloc_rms_norm_backward(d_y, f["sum"], w, f["rstd"], d_sum=d_sum)
    for place in ("d_y", "d_sum"):
        a, b = d_y.clone(), d_sum.clone()
        got = S.stalloc_rms_norm_backward(a, f["sum"], w, f["rstd"], d_sum=b, out={"dx": a if place == "d_y" else b})
        assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dweight"], want["dweight"])
    wide = torch.zeros(rows, width + 5, dtype=torch.bfloat16, device="cuda")
    wide[:, :width] = d_y
    got = S.stalloc_rms_norm_backward(wide[:, :width], f["sum"], w, f["rstd"], d_sum=d_sum)
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dweight"], want["dweight"])


def test_gradient_against_differences(S):
    import torch
    rows, width = 5, 60
    x, r, w, d_y, _ = _inputs(2, rows, width, torch.float32)
    f = S.stalloc_rms_norm(x.cuda(), w.cuda())
    b = S.stalloc_rms_norm_backward(d_y.cuda(), x.cuda(), w.cuda(), f["rstd"])
    gen = torch.Generator().manual_seed(5)

    def loss(x, w):
        s = x.double()
        return float((s / torch.sqrt((s ** 2).mean(-1, keepdim=True) + 1e-6) * w.double() * d_y.double()).sum())

    for name in ("dx", "dweight"):
        at = x if name == "dx" else w
        way, step = torch.randn(at.shape, generator=gen, dtype=torch.float64), 1e-6
        moved = [(at.double() + k * step * way) for k in (1, -1)]
        slope = [loss(m, w) if name == "dx" else loss(x, m) for m in moved]
        slope = (slope[0] - slope[1]) / (2 * step)
        assert abs(float((b[name].double().cpu() * way).sum()) - slope) <= 1e-5 * (1.0 + abs(slope)) + 1e-4
