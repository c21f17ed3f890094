"""The output of stalloc_rms_norm in 8 bits: the nearest 8-bit number to y / scale, as a division gives it, and half precision against the definition in 64 bits."""
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


def _quotients(y, scales):
    """y / scale in 32 bits, rounded to nearest, then to e4m3."""
    import torch
    spread = scales.cpu().repeat_interleave(128, 1)[:, :y.shape[1]]
    return (y.cpu() / spread).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def test_numbers_between_two_of_the_type(S):
    """Rows whose numbers lie, up to the last bits of 32, half way between two 8-bit ones: all odd multiples of half a step, of many row maxima.  y in 32 bits is what is
    divided, so the quotient is known."""
    import torch
    rows = 4096
    gen = torch.Generator().manual_seed(1)
    half_way = (torch.arange(17, 32, 2) / 16.0).view(1, -1) * 2.0 ** torch.arange(-5, 8).view(-1, 1)       # 1 + odd / 16 in every binade of the type's normal numbers
    half_way = half_way.flatten()[:127]
    most = 0.5 + torch.rand(rows, 1, generator=gen)
    x = torch.cat([torch.full((rows, 1), 448.0), half_way[half_way < 440.0].expand(rows, -1)], 1) * most
    x[:, 1::2] *= -1.0
    got = S.stalloc_rms_norm(x.cuda(), torch.ones(x.shape[1], device="cuda"), eight_bits=True, out={"y": torch.empty(x.shape, device="cuda")})
    torch.cuda.synchronize()
    want = _quotients(got["y"], got["scales"])
    assert torch.equal(got["q"].cpu().view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("rows,width", [(5, 127), (70, 512), (33, 2048), (3, 4095), (2, 20000), (2, 40000)])
def test_as_a_division(S, rows, width):
    import torch
    gen = torch.Generator().manual_seed(width)
    x, r, w = torch.randn(rows, width, generator=gen), torch.randn(rows, width, generator=gen), 1.0 + 0.3 * torch.randn(width, generator=gen)
    x[0, 3] = r[0, 3] = -0.0
    got = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), eight_bits=True, out={"y": torch.empty(rows, width, device="cuda")})
    torch.cuda.synchronize()
    assert torch.equal(got["q"].cpu().view(torch.uint8), _quotients(got["y"], got["scales"]).view(torch.uint8))


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 127), (2, 128), (9, 129), (70, 512), (4, 1000), (6, 1024), (5, 1025), (33, 2048), (3, 4095), (2, 8193), (2, 20000), (3, 32769)]


@pytest.mark.parametrize("rows,width", SHAPES)
def test_half_precision(S, rows, width):
    """Scales to 32-bit accuracy; every number within half a step of e4m3 (2^-4 relative, 2^-10 of the scale below its normal range)."""
    import torch
    gen = torch.Generator().manual_seed(rows * 3 + width)
    make = lambda *shape: torch.randn(*shape, generator=gen).to(torch.float16)               # noqa: E731
    x, r, w = make(rows, width), make(rows, width), (1.0 + 0.3 * torch.randn(width, generator=gen)).to(torch.float16)
    if rows > 1:
        x[1, : min(width, 128)] = 0.0
        r[1, : min(width, 128)] = 0.0                             # a block of zeros
    _, _, y = plain.rms_norm(x, r, w, 1e-5)
    want = plain.eight_bits(y)
    got = S.stalloc_rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), eps=1e-5, eight_bits=True)
    torch.cuda.synchronize()
    rel = (width + 8) * F32 / 2 + 16 * F32                        # rstd (a sum of `width` squares), two products, the scale's division
    assert float(((got["scales"].double().cpu() - want).abs() / want).max()) <= rel
    spread = got["scales"].double().cpu().repeat_interleave(128, 1)[:, :width]
    allowed = (2.0 ** -4 * (1 + 2.0 ** -4) + rel) * y.abs() + 2.0 ** -10 * spread
    assert float(((got["q"].cpu().double() * spread - y).abs() - allowed).max()) <= 0.0
