"""Steps whose numbers have overflowed throughout: everything that sees them is NaN, and calls with finite numbers behind them on the same workspace are as they were."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128, 40])
@pytest.mark.parametrize("which", [1, 2, 3])
def test_everything_is_nan(which, d):
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    n, h, g = 700, 4, 2
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = [torch.randn(n, heads, d, generator=gen, device="cuda").to(torch.float16) for heads in (h, g, g, h)]
    bounds = torch.tensor([0, 300, 301, 690], dtype=torch.int32).cuda()
    keep = {}

    def both(x):
        f = S.stalloc_attention(*x[:3], bounds, workspace_cache=keep)
        b = S.stalloc_attention_backward(x[3], *x[:3], f["o"], f["lse"], bounds, workspace_cache=keep)
        return [f["o"], b["dq"], b["dk"], b["dv"]]

    want = both(x)
    bad = list(x)
    bad[which] = torch.full_like(x[which], float("nan"))
    o, dq, dk, dv = both(bad)
    for name, got in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        # (v has no part in dv, nor d_o in the output; a NaN in k is in every weight)
        if (name, which) in (("o", 3), ("dv", 2)):
            assert bool(torch.isfinite(got).all()), name
        else:
            assert bool(torch.isnan(got[:690]).all()), name
        assert not bool(got[690:].any()), name                       # (padding)
    for got, w in zip(both(x), want):
        assert torch.equal(got, w)
