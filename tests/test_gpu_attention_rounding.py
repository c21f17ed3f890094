"""What roundings cost the gradients of rows that see few keys: dq and dk of sequences of at most 128 tokens lose their own rounding to the type and no more.

A rounding to nearest of x = m 2^e, 1 <= m < 2, is off by at most u |x| / m, u half a step of the type, and by u |x| / (m sqrt 3) in the root mean square: relative to the norm of a large
tensor at most u / sqrt 3, 0.58 u.  Everything else is held in 32 bits, but for what is left of ds behind two roundings (2^-16 of it in bfloat16); 5 % are for these and for chance
(10^5 numbers and more).  With D from the rounded o and ds rounded once the three errors add up to 0.7 to 0.8 u."""
import pytest

import plain_operators as plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("h,g,d", [(8, 8, 64), (8, 2, 128), (6, 3, 80)])
def test_short_sequences(t, h, g, d):
    import numpy as np
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    t = getattr(torch, t)
    cuts = [0] + list(np.cumsum([128, 127, 33, 5, 64, 97, 2, 20, 1, 80]))
    n, gen = int(cuts[-1]), torch.Generator().manual_seed(d)
    q, k, v, d_o = (torch.randn(n, heads, d, generator=gen).to(t) for heads in (h, g, g, h))
    scale = d ** -0.5
    want, _ = plain.attention(q, k, v, [int(c) for c in cuts], scale, d_o)
    bounds = torch.tensor(cuts, dtype=torch.int32).cuda()
    q, k, v, d_o = (x.cuda() for x in (q, k, v, d_o))
    f = S.stalloc_attention(q, k, v, bounds)
    b = S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds)
    for name in ("dq", "dk"):
        off = b[name].double().cpu() - want[name]
        assert float(off.norm() / want[name].norm()) <= 1.05 * plain.half(t) / 3 ** 0.5, name
