"""The most likely tokens of rows that hold NaN of either sign: their order is unspecified, but every place is written, with tokens of the vocabulary that are all different."""
import pytest

pytestmark = pytest.mark.gpu
BITS = {"float32": ("int32", 0x7fc00000, -0x400000), "bfloat16": ("int16", 0x7fc0, -0x40), "float16": ("int16", 0x7e00, -0x200)}      # NaN, and NaN with the sign bit


@pytest.mark.parametrize("rows,vocabulary,top", [(5, 4000, 16), (5, 300, 64), (5, 64, 64), (5, 70001, 5), (5, 70001, 64), (2100, 260, 9), (5, 33000, 17)])
@pytest.mark.parametrize("t", list(BITS))
def test_every_place_is_a_token(t, rows, vocabulary, top):
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    word, plus, minus = BITS[t]
    x = torch.randn(rows, vocabulary, generator=torch.Generator().manual_seed(top)).to(getattr(torch, t))
    clean = x.clone()
    bits = x.view(getattr(torch, word))
    bits[0, :] = minus
    bits[1, ::2] = minus
    bits[2, :] = plus
    bits[3, vocabulary // 2:] = minus
    x[3, : vocabulary // 2] = -float("inf")
    assert bool(torch.isnan(x[0]).all()) and bool((bits[0] < 0).all())
    tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    out = {"top_tokens": torch.full((rows, top), -77, dtype=torch.int32, device="cuda"), "top_logprobs": torch.full((rows, top), 77.0, device="cuda")}
    got = S.stalloc_token_logprobs(x.cuda(), tokens, top=top, out=out)
    torch.cuda.synchronize()
    S.check_status(got)
    found, values = got["top_tokens"].cpu(), got["top_logprobs"].cpu()
    assert int(found.min()) >= 0 and int(found.max()) < vocabulary
    assert bool((found.sort(-1).values.diff(dim=-1) > 0).all())
    assert bool(torch.isnan(values[:4]).all()) and bool(torch.isnan(got["lse"][:4]).all())
    want = S.stalloc_token_logprobs(clean.cuda(), tokens, top=top)
    assert torch.equal(found[4:], want["top_tokens"][4:].cpu()) and torch.equal(values[4:], want["top_logprobs"][4:].cpu())
