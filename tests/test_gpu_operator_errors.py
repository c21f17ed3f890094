"""An error that some other call of the thread left behind is not an operator's: it is called once, succeeds, and what it does in place is done once."""
import ctypes
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    return S


def _hip():
    """The runtime that this process has loaded."""
    with open("/proc/self/maps") as f:
        (path,) = {line.split()[-1] for line in f if "libamdhip64.so" in line}
    return ctypes.CDLL(path)


def _leave_an_error():
    assert _hip().hipSetDevice(4096) != 0                        # no such device: refused on the host, and remembered


def test_in_place_calls_work_once(S):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    grads = [torch.randn(n, generator=gen, device="cuda") for n in (1000, 70_000)]
    kept, cache = [g.clone() for g in grads], {}
    todo = S.stalloc_tensor_list(grads, grads)
    S.stalloc_clip_gradients(todo, math.inf, workspace_cache=cache)                          # (makes the workspace; changes nothing)
    torch.cuda.synchronize()
    _leave_an_error()
    f = S.stalloc_clip_gradients(todo, 1.0, workspace_cache=cache)
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in kept))
    assert abs(float(f["norm"]) - want) <= 2.0 ** -22 * want

    rows, width = 64, 2000
    x, w, d_y, d_sum = (torch.randn(*s, generator=gen, device="cuda").bfloat16() for s in ((rows, width), (width,), (rows, width), (rows, width)))
    n, cache = S.stalloc_rms_norm(x, w), {}
    want = S.stalloc_rms_norm_backward(d_y, x, w, n["rstd"], d_sum=d_sum, workspace_cache=cache)
    torch.cuda.synchronize()
    for place in ("d_y", "d_sum"):
        a, b = d_y.clone(), d_sum.clone()
        torch.cuda.synchronize()
        _leave_an_error()
        got = S.stalloc_rms_norm_backward(a, x, w, n["rstd"], d_sum=b, out={"dx": a if place == "d_y" else b}, workspace_cache=cache)
        torch.cuda.synchronize()
        assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dweight"], want["dweight"])


def test_every_entry_point(S):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, d_o = (torch.randn(40, 4, 64, generator=gen, device="cuda").half() for _ in range(2))
    bounds = torch.tensor([0, 40], dtype=torch.int32).cuda()
    x, w, tokens, one = (torch.randn(5, 100, generator=gen, device="cuda"), torch.ones(100, device="cuda"), torch.arange(5, device="cuda").int(),
                         torch.ones(5, device="cuda"))
    f, n, p = S.stalloc_attention(q, q, q, bounds), S.stalloc_rms_norm(x, w), S.stalloc_token_logprobs(x, tokens)
    calls = [lambda: S.stalloc_attention(q, q, q, bounds), lambda: S.stalloc_attention_backward(d_o, q, q, q, f["o"], f["lse"], bounds),
             lambda: S.stalloc_rms_norm(x, w), lambda: S.stalloc_rms_norm_backward(x, x, w, n["rstd"]), lambda: S.stalloc_token_logprobs(x, tokens, top=3),
             lambda: S.stalloc_token_logprobs_backward(x, tokens, p["lse"], p["entropy"], one), lambda: S.stalloc_clip_gradients(S.stalloc_tensor_list([x]), 1.0)]
    torch.cuda.synchronize()
    keep = []
    for call in calls:
        _leave_an_error()
        keep.append(call())
    torch.cuda.synchronize()
