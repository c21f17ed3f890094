"""Gradients of attention in half precision whatever the size of d_o: they lose their own rounding to the type (which is large where they lie below its normal numbers), and the rounding of
weights and of their gradients for the second products, each within the type's normal range.

u is half a step of the type.  A rounding to nearest is off by at most 0.58 u in the root mean square, relative to the norm of many numbers; rounded weights' gradients are multiplied by
keys and queries of both signs and independent of them, so a sum of such products is off by as much of its norm as they are.  So: sqrt(r^2 + (0.58 u)^2), r what the exact result loses by
rounding, and a tenth for chance, sums in 32 bits and D, which comes from the rounded output (1 / sqrt(row) of that rounding reaches ds)."""
import pytest

import plain_operators as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    return S


def _exact(q, k, v, d_o, bounds):
    """dq, dk, dv in 64 bits on the GPU, products in two dimensions."""
    import torch
    q, k, v, d_o = (x.double() for x in (q, k, v, d_o))
    scale = q.shape[2] ** -0.5
    out = [torch.zeros_like(x) for x in (q, k, v)]
    for a, b in zip(bounds, bounds[1:]):
        later = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
        for h in range(q.shape[1]):
            g = h * k.shape[1] // q.shape[1]
            x, y, z, up = q[a:b, h].contiguous(), k[a:b, g].contiguous(), v[a:b, g].contiguous(), d_o[a:b, h].contiguous()
            p = torch.softmax((x @ y.T * scale).masked_fill(later, -float("inf")), -1)
            ds = p * (up @ z.T - (up * (p @ z)).sum(-1, keepdim=True)) * scale
            out[0][a:b, h] = ds @ y
            out[1][a:b, g] += ds.T @ x
            out[2][a:b, g] += p.T @ up
    return out


def _check(S, q, k, v, d_o, cuts, where=slice(None)):
    import torch
    bounds = torch.tensor(cuts, dtype=torch.int32).cuda()
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    torch.cuda.synchronize()
    S.check_status(b)
    u = plain.half(torch.float16)
    for name, want in zip(("dq", "dk", "dv"), _exact(q, k, v, d_o, cuts)):
        got, want = b[name][where].double(), want[where]
        size = float(want.norm())
        rounding = float((want.half().double() - want).norm()) / size
        assert float((got - want).norm()) / size <= 1.1 * (rounding ** 2 + (0.58 * u) ** 2) ** 0.5, name


def _inputs(seed, n, h, g, d, size, of_v=1.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda heads, scale: (torch.randn(n, heads, d, generator=gen, device="cuda") * scale).half()      # noqa: E731
    return make(h, 1.0), make(g, 1.0), make(g, of_v), make(h, size)


@pytest.mark.parametrize("n,h,g,d,cuts", [(2048, 2, 1, 128, [0, 2048]), (4096, 1, 1, 64, [0, 4096]), (2500, 6, 3, 80, [0, 900, 2500]), (3000, 32, 16, 64, [0, 1900, 1911, 3000]),
                                          (2300, 16, 16, 128, [0, 2300])])      # (walks cut into parts, and not)
@pytest.mark.parametrize("size", [1e-5, 1e-4, 1e-3, 1.0, 1e4])
def test_any_size(S, size, n, h, g, d, cuts):
    if size == 1e4 and h // g * n > 5000:
        size = 3e3                                               # (dv, a sum over the heads of a group, has to fit the type itself)
    _check(S, *_inputs(n + h, n, h, g, d, size), cuts)


@pytest.mark.parametrize("of_v", [1e-3, 30.0])
def test_values_of_any_size(S, of_v):
    _check(S, *_inputs(9, 2048, 2, 2, 64, 1e-2 / of_v, of_v), [0, 2048])


def test_a_long_row(S):
    """Weights of 1 / 16384 and less."""
    _check(S, *_inputs(4, 16384, 1, 1, 64, 1e-2), [0, 16384])


@pytest.mark.parametrize("falling", [True, False])
def test_sizes_that_change_along_the_sequence(S, falling):
    """d_o falls or grows by 10^6 from one end to the other: rows and keys where it is small have gradients of their own size."""
    import torch
    q, k, v, d_o = _inputs(5, 2048, 2, 2, 64, 1.0)
    slope = torch.logspace(1, -5, 2048, device="cuda").view(-1, 1, 1)
    d_o = (d_o.float() * (slope if falling else slope.flip(0))).half()
    for at in range(0, 2048, 512):
        _check(S, q, k, v, d_o, [0, 2048], slice(at, at + 512))
