"""The operators of a training step allocate nothing and work on the caller's stream only: captured in a graph, with outputs and workspaces that
stay, every replay gives what eager calls give on the same inputs, eager work and synchronizations in between."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2507_16274_amd as S
    return S


def _attention(S, n, h, g, d, lengths):
    import torch
    cuts = [0]
    for x in lengths:
        cuts.append(cuts[-1] + x)
    bounds = torch.tensor(cuts, dtype=torch.int32).cuda()
    shapes = [(n, h, d), (n, g, d), (n, g, d), (n, h, d)]
    f, b, c1, c2 = {}, {}, {}, {}

    def call(q, k, v, d_o):
        f.update(S.stalloc_attention(q, k, v, bounds, out=f, workspace_cache=c1))
        b.update(S.stalloc_attention_backward(d_o, q, k, v, f["o"], f["lse"], bounds, out=b, workspace_cache=c2))
        return [f["o"], f["lse"], b["dq"], b["dk"], b["dv"], f["status"], b["status"]]
    return shapes, torch.bfloat16, call


def _norm(S, rows, width):
    import torch
    f, b, c = {}, {}, {}
    weight = torch.ones(width, dtype=torch.bfloat16, device="cuda")

    def call(x, r, d_y):
        f.update(S.stalloc_rms_norm(x, weight, residual=r, eight_bits=True, out={**f, "y": f.get("y", torch.empty_like(x))}))
        b.update(S.stalloc_rms_norm_backward(d_y, f["sum"], weight, f["rstd"], d_sum=r, out=b, workspace_cache=c))
        return [f["sum"], f["y"], f["q"].view(torch.uint8), f["scales"], b["dx"], b["dweight"]]
    return [(rows, width)] * 3, torch.bfloat16, call


def _logprobs(S, rows, vocabulary):
    import torch
    f, b, c = {}, {}, {}
    tokens = (torch.arange(rows, device="cuda") * 7 % vocabulary).int()

    def call(x, g):
        f.update(S.stalloc_token_logprobs(x, tokens, top=5, out=f, workspace_cache=c))
        b.update(S.stalloc_token_logprobs_backward(x, tokens, f["lse"], f["entropy"], g, g, out=b))
        return [f["logprob"], f["entropy"], f["lse"], f["top_tokens"], f["top_logprobs"], b["d_logits"], f["status"], b["status"]]
    return [(rows, vocabulary), (rows,)], torch.float32, call


def _clip(S, sizes):
    import torch
    outs, c, f, held = [], {}, {}, {}

    def call(*grads):
        if "list" not in held:
            outs.extend(torch.empty_like(g) for g in grads)
            held["list"] = S.stalloc_tensor_list(grads, outs)
        f.update(S.stalloc_clip_gradients(held["list"], 1.0, out=f, workspace_cache=c))
        return [f["norm"], f["factor"], *outs]
    return [(n,) for n in sizes], torch.float32, call


CASES = {
    "attention_short": lambda S: _attention(S, 100, 4, 2, 64, [30, 0, 70]),
    "attention_listed": lambda S: _attention(S, 5000, 64, 8, 64, [700, 20, 1500, 3, 2700]),
    "attention_parts": lambda S: _attention(S, 1500, 2, 1, 128, [1400]),
    "norm": lambda S: _norm(S, 70, 3000),
    "logprobs_parts": lambda S: _logprobs(S, 3, 20000),
    "logprobs_rows": lambda S: _logprobs(S, 2100, 300),
    "clip": lambda S: _clip(S, [70_000, 3, 9000] + [11] * 150),
}


@pytest.mark.parametrize("name", CASES)
def test_replays_match_eager_calls(S, name):
    import torch
    shapes, dtype, call = CASES[name](S)
    gen = torch.Generator(device="cuda").manual_seed(1)
    sets = [[torch.randn(s, generator=gen, device="cuda").to(dtype) for s in shapes] for _ in range(2)]
    inputs = [x.clone() for x in sets[0]]
    want = []
    for values in sets:                                              # eager: also sizes the workspaces and makes the outputs
        for x, value in zip(inputs, values):
            x.copy_(value)
        out = call(*inputs)
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(*inputs)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            captured = call(*inputs)
    torch.cuda.synchronize()
    for which in (0, 1, 0, 0, 1):
        for x, value in zip(inputs, sets[which]):
            x.copy_(value)
        for t in captured:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(captured, want[which]):
            assert torch.equal(got, w)
