"""Norms of more rows, or of wider ones, than one launch takes threads for: norms per head of a long batch, a norm over a whole tensor."""
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


@pytest.mark.parametrize("rows,width,eight_bits", [((1 << 26) + 5, 3, False), ((1 << 26) - 3, 8, True), ((1 << 25) + 7, 1025, False)])
def test_many_rows(S, rows, width, eight_bits):
    """Every row against the definition, in 32 bits on the GPU: rows of the second launch are not those of the first."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(width)
    x = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w = torch.ones(width, dtype=torch.bfloat16, device="cuda")
    got = S.stalloc_rms_norm(x, w, eight_bits=eight_bits, out={"y": torch.empty_like(x)})
    torch.cuda.synchronize()
    step, rel = 1 << 22, (width + 8) * F32
    for at in list(range(0, rows, step))[:: max(1, width // 40)] + [rows - 5]:       # (of wide rows some; the last ones always)
        part = slice(at, min(rows, at + (step if width < 100 else 4096)))
        s = x[part].float()
        rstd = 1.0 / torch.sqrt(s.square().mean(-1) + 1e-6)
        assert bool(((got["rstd"][part] - rstd).abs() <= 2 * rel * rstd).all())
        y = s * rstd[:, None]
        assert bool(((got["y"][part].float() - y).abs() <= (plain.half(torch.bfloat16) * 1.01 + 2 * rel) * y.abs()).all())
        if eight_bits:
            scale = y.abs().amax(-1, keepdim=True).clamp(min=448 * 2.0 ** -126) / 448
            assert bool(((got["scales"][part] - scale).abs() <= 3 * rel * scale).all())
            assert bool(((got["q"][part].float() * scale - y).abs() <= (2.0 ** -4 + 4 * rel) * 1.07 * y.abs() + 2.0 ** -10 * scale).all())


def test_backward_of_one_wide_row(S):
    import torch
    width = (1 << 28) + 1000
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, d_y = (torch.empty(1, width, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    w = torch.ones(width, dtype=torch.bfloat16, device="cuda")
    rstd = torch.full((1,), 1.25, device="cuda")
    dweight = torch.full((width,), float("nan"), device="cuda")
    got = S.stalloc_rms_norm_backward(d_y, x, w, rstd, out={"dweight": dweight})
    torch.cuda.synchronize()
    want = d_y[0].float() * x[0].float() * 1.25
    assert bool(((got["dweight"] - want).abs() <= 4 * F32 * want.abs()).all())


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    import torch
    torch.cuda.empty_cache()
