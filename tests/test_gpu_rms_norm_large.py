"""stalloc_rms_norm and its backward pass on tensors of 64 MiB and more, whose inputs go past the caches: the same bounds as for small ones, the
reference in 64 bits on the GPU."""
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


def _rel(width):
    return (width + 8) * F32 / 2 + 8 * F32


# a wave a row with one group and with two, a workgroup a row with few and with many threads (odd widths: rows begin anywhere), and four groups a thread
SHAPES = [("float32", 34000, 500), ("bfloat16", 41000, 1000), ("float16", 6200, 5501), ("bfloat16", 3000, 12007), ("bfloat16", 1700, 20000)]


@pytest.mark.parametrize("t,rows,width", SHAPES)
def test_both_passes(S, t, rows, width):
    import torch
    t = getattr(torch, t)
    assert rows * width * t.itemsize >= 64 << 20
    gen = torch.Generator(device="cuda").manual_seed(rows)
    make = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(t)            # noqa: E731
    x, r, d_y, d_sum, w = make(rows, width), make(rows, width), make(rows, width), make(rows, width), make(width)
    want_sum, want_rstd, want_y = plain.rms_norm(x, r, w, 1e-6)
    f = S.stalloc_rms_norm(x, w, residual=r)
    assert torch.equal(f["sum"], want_sum)
    assert float(((f["rstd"].double() - want_rstd).abs() / want_rstd).max()) <= _rel(width)
    least = torch.finfo(t).tiny * 2 * plain.half(t)
    assert float(((f["y"].double() - want_y).abs() - (plain.half(t) + _rel(width) + 2 * F32) * want_y.abs() - least).max()) <= 0.0
    del want_y
    eight = S.stalloc_rms_norm(x, w, residual=r, eight_bits=True)
    few = slice(rows // 2, rows // 2 + 3)                            # (a small call goes through the caches)
    small = S.stalloc_rms_norm(x[few].contiguous(), w, residual=r[few].contiguous(), eight_bits=True)
    assert torch.equal(eight["q"][few].view(torch.uint8), small["q"].view(torch.uint8)) and torch.equal(eight["scales"][few], small["scales"])
    want, want_w = plain.rms_norm_backward(d_y, want_sum, w, want_rstd, d_sum)
    b = S.stalloc_rms_norm_backward(d_y, f["sum"], w, f["rstd"], d_sum=d_sum)
    s, q = want_sum.double(), want_rstd[:, None]
    g = w.double() * d_y.double()
    parts = q * g.abs() + q ** 3 * s.abs() * (g * s).abs().mean(-1, keepdim=True)
    rel = _rel(width) * 4 + (width + 8) * F32
    allowed = (rel * parts + plain.half(t) * want.abs()) * (1 + plain.half(t)) + 4 * F32 * (parts + want.abs()) + least
    assert float(((b["dx"].double() - want).abs() - allowed).max()) <= 0.0
    allowed = (rows * F32 + _rel(width) + 4 * F32) * (d_y.double() * s * q).abs().sum(0)
    assert float(((b["dweight"].double() - want_w).abs() - allowed).max()) <= 0.0
    a, c = d_y.clone(), d_sum.clone()
    for at in (a, c):
        got = S.stalloc_rms_norm_backward(a, f["sum"], w, f["rstd"], d_sum=c, out={"dx": at})
        assert torch.equal(got["dx"], b["dx"]) and torch.equal(got["dweight"], b["dweight"])
        a, c = d_y.clone(), d_sum.clone()
