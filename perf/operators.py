"""Operators of a training step that write where a plan says, as cases that can be timed and compared.

A case names one operator (`op`), whether it is the forward call alone or a training pass (`train`: forward and
backward), a type and sizes.  `run` computes it in elementary torch operations or, where `own` is true, with the
package's entry points, into outputs and a workspace that the caller keeps, as a step at planned addresses does.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E4M3_MAX, BLOCK, LEAST_SCALE = 448.0, 128, 2.0 ** -126
EPS = 1e-6
BUCKET = 25 * 2 ** 20                          # bytes of a gradient bucket


def _attention(name, **more):
    return {**({"name": name} if name else {}), "op": "attention", "train": False, "type": "bf16", "tokens": 4096, "sequences": 1, "cut": 0,
            "pad": 0, "heads": 32, "kv_heads": 32, "head_dim": 128, **more}


def _norm(name, **more):
    return {**({"name": name} if name else {}), "op": "norm", "train": False, "type": "bf16", "rows": 4096, "width": 4096, "eight_bits": False, **more}


def _logprobs(name, **more):
    return {**({"name": name} if name else {}), "op": "logprobs", "train": False, "type": "bf16", "rows": 4096, "vocabulary": 32000, "padded": 0,
            "top": 0, **more}


def _clip(name, **more):
    return {**({"name": name} if name else {}), "op": "clip", "type": "f32", "buckets": 1, "bucket": BUCKET // 4, "small": 0, "small_width": 4096,
            **more}


def listed():
    return [
        # a few short texts through the two-layer model of a test: launches are all there is
        _attention("attention_few", tokens=187, sequences=5, cut=1, heads=8, kv_heads=2, head_dim=64),
        # documents of very different lengths packed to one row of a batch, padding at its end, four heads to a key head
        _attention("attention_packed", type="f16", tokens=8000, sequences=23, cut=2, pad=61, heads=32, kv_heads=8),
        # one long text on the widest configuration (hidden 8192, sequence 8192)
        _attention("attention_long", tokens=8192, heads=64, kv_heads=8),
        # a layer of a pipeline stage in training (hidden 4096, sequence 4096): what its backward phase recomputes and derives
        _attention("attention_train", train=True),
        # the same over packed documents with small heads
        _attention("attention_train_packed", train=True, type="f16", tokens=5003, sequences=17, cut=3, pad=3, heads=16, kv_heads=4, head_dim=64),
        # the norm before a projection in 8 bits, for a handful of tokens
        _norm("norm_few", type="f16", rows=7, width=4096, eight_bits=True),
        # the same for a whole micro-batch of the widest configuration
        _norm("norm_eight_bits", rows=8192, width=8192, eight_bits=True),
        # a training pass of the norm of a stage, width no power of two
        _norm("norm_train", train=True, rows=8192, width=5120),
        # scoring a few sampled tokens, alternatives shown
        _logprobs("logprobs_few", type="f32", rows=16, vocabulary=50257, top=16),
        # the loss of a micro-batch: its logits are the largest buffer of the last stage
        _logprobs("logprobs_train", train=True, vocabulary=131072, padded=53, top=4),
        # gradients of a model of test size: many small tensors
        _clip("clip_few", type="bf16", buckets=6, bucket=512 * 512, small=20, small_width=509),
        # the gradient buckets of an interleaved stage
        _clip("clip_buckets", buckets=48, small=13, small_width=8191),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "norm", "norm", "logprobs", "logprobs", "clip"))
    if op == "attention":
        train = rng.random() < 0.5
        kv_heads = rng.choice((1, 2, 3, 4, 8, 8))
        heads = kv_heads * rng.choice((1, 2, 4, 5, 8))
        most = int(math.sqrt((32 * 4096 ** 2 if train else 64 * 8192 ** 2) / heads))
        tokens = _spread(rng, 1, min(most, 16384))
        sequences = rng.choice((1, 1, 1 + tokens // 100, _spread(rng, 1, 64)))
        if train:                              # (the gradient of a sequence of one token is zero: its weight is 1 whatever its score is)
            tokens = max(tokens, 16)
            sequences = min(sequences, tokens // 4)
        return _attention(None, train=train, type=rng.choice(("bf16", "bf16", "f16")), tokens=tokens, sequences=sequences,
                          cut=rng.randrange(1 << 20), pad=rng.choice((0, 0, min(tokens // 2, 37))), heads=heads, kv_heads=kv_heads,
                          head_dim=rng.choice((64, 128, 128, 80, 96, 32)))
    if op == "norm":
        rows, width = _spread(rng, 1, 16384), rng.choice((512, 1000, 2048, 4096, 5120, 8192, 777))
        return _norm(None, train=rng.random() < 0.5, type=rng.choice(("bf16", "f16", "f32")), rows=max(1, min(rows, 8192 * 8192 // width)),
                     width=width, eight_bits=rng.random() < 0.4)
    if op == "logprobs":
        vocabulary = rng.choice((32000, 50257, 65536, 100003, 131072, 997))
        rows = max(1, min(_spread(rng, 1, 8192), 4096 * 131072 // vocabulary))
        return _logprobs(None, train=rng.random() < 0.5, type=rng.choice(("bf16", "bf16", "f16", "f32")), rows=rows, vocabulary=vocabulary,
                         padded=rng.choice((0, 0, 3, 53)), top=rng.choice((0, 1, 5, 16)))
    return _clip(None, type=rng.choice(("f32", "bf16", "f16")), buckets=rng.randint(1, 40), bucket=_spread(rng, 1000, BUCKET // 4),
                 small=rng.randint(0, 20), small_width=rng.choice((512, 4096, 8191, 1)))


def _bounds(c):
    """Boundaries of the packed sequences: lengths spread over two orders of magnitude, one of them empty where there are several."""
    live = c["tokens"] - c["pad"]
    rng = random.Random(c["cut"])
    share = [math.exp(rng.uniform(0.0, 4.6)) for _ in range(c["sequences"])]
    if c["sequences"] > 3:
        share[rng.randrange(c["sequences"])] = 0.0
    total, at, cuts = sum(share), 0.0, [0]
    for s in share[:-1]:
        at += s
        cuts.append(max(cuts[-1], int(live * at / total)))
    return cuts + [live]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[c["type"]]

    def normal(*shape, scale=1.0, to=t):
        x = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, scale, generator=gen)
        return x.to(to)

    s = {"case": c, "keep": {}}                # `keep`: outputs and workspace of a program that calls the operator again and again
    if c["op"] == "attention":
        n, h, g, d = c["tokens"], c["heads"], c["kv_heads"], c["head_dim"]
        qkv = normal(n, (h + 2 * g) * d)       # as the projection leaves them: one row per token
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split((h * d, g * d, g * d), dim=1))
        s["bounds"] = torch.tensor(_bounds(c), dtype=torch.int32, device="cuda")
        if c["train"]:
            s["d_o"] = normal(n, h, d, scale=0.1)
    elif c["op"] == "norm":
        n, w = c["rows"], c["width"]
        s["x"], s["residual"] = normal(n, w), normal(n, w, scale=3.0)
        s["weight"] = (1.0 + normal(w, scale=0.2, to=torch.float32)).to(t)
        if c["train"]:
            s["d_y"], s["d_sum"] = normal(n, w, scale=0.1), normal(n, w, scale=0.1)
    elif c["op"] == "logprobs":
        n, v = c["rows"], c["vocabulary"]
        s["logits"] = normal(n, v, scale=2.0)
        s["tokens"] = torch.randint(v - c["padded"], (n,), generator=gen, device="cuda", dtype=torch.int32)
        sure = torch.rand(n, generator=gen, device="cuda") < 0.6      # what a trained model gives: most tokens are expected
        s["logits"][torch.arange(n, device="cuda"), s["tokens"].long()] += (12.0 * sure).to(t)
        if c["padded"]:
            s["logits"][:, v - c["padded"]:] = float("-inf")          # columns that only round the vocabulary up
        if n > 4:
            s["tokens"][n // 3] = -1                                  # a position without a target
        if c["train"]:
            s["d_logprob"] = normal(n, scale=1.0 / n, to=torch.float32)
            s["d_entropy"] = normal(n, scale=0.01 / n, to=torch.float32)
    else:
        sizes = [c["bucket"] + 3 * i for i in range(c["buckets"])] + [c["small_width"]] * c["small"]
        s["grads"] = [normal(m, scale=0.02) for m in sizes]
        s["max_norm"] = 1.0
    return s


# ---------------------------------------------------------------------------------------------
# plain forms

def _seen(c, bounds):
    """[tokens, tokens] which keys a token sees, and by token whether it belongs to a sequence."""
    at = torch.arange(c["tokens"], device=bounds.device)
    which = torch.searchsorted(bounds[1:].contiguous(), at.to(torch.int32), right=True)
    lives = at < bounds[-1]
    return (which[:, None] == which[None, :]) & (at[None, :] <= at[:, None]) & lives[:, None], lives


def _plain_attention(s):
    c = s["case"]
    n, h, g, d = c["tokens"], c["heads"], c["kv_heads"], c["head_dim"]
    scale = 1.0 / math.sqrt(d)
    q, k, v = (s[x].float().transpose(0, 1).contiguous() for x in ("q", "k", "v"))
    q = q.view(g, h // g * n, d)
    seen, lives = _seen(c, s["bounds"])
    p = torch.matmul(q, k.transpose(1, 2).contiguous()).view(g, h // g, n, n)
    p.mul_(scale).masked_fill_(~seen, float("-inf"))
    top = p.amax(-1, keepdim=True).masked_fill_(~lives[:, None], 0.0)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).view(h, n)
    p.div_(total.masked_fill(~lives[:, None], 1.0))
    o = torch.matmul(p.view(g, -1, n), v).view(h, n, d).transpose(0, 1)
    out = {"o": o.to(TYPES[c["type"]]), "lse": lse}
    if c["train"]:
        d_o = s["d_o"].float().transpose(0, 1).reshape(g, -1, d)
        dot = (d_o * o.transpose(0, 1).reshape(g, -1, d)).sum(-1).view(g, h // g, n, 1)
        out["dv"] = torch.matmul(p.view(g, -1, n).transpose(1, 2).contiguous(), d_o)
        ds = torch.matmul(d_o, v.transpose(1, 2).contiguous()).view_as(p)
        ds.sub_(dot).mul_(p).mul_(scale)
        ds = ds.view(g, -1, n)
        out["dq"] = torch.matmul(ds, k).view(h, n, d)
        out["dk"] = torch.matmul(ds.transpose(1, 2).contiguous(), q)
        for_tokens = {x: out[x].transpose(0, 1).to(TYPES[c["type"]]) for x in ("dq", "dk", "dv")}
        out.update(for_tokens)
    return out


def _eight_bits(y):
    """y as e4m3 numbers and a scale for every row and 128 columns."""
    n, w = y.shape
    cols = -(-w // BLOCK)
    y = torch.nn.functional.pad(y, (0, cols * BLOCK - w)).view(n, cols, BLOCK)
    scales = y.abs().amax(-1).clamp(min=E4M3_MAX * LEAST_SCALE) / E4M3_MAX
    q = (y / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).view(n, -1)[:, :w].to(torch.float32).to(torch.float8_e4m3fn)
    return q, scales


def _plain_norm(s):
    c = s["case"]
    t = TYPES[c["type"]]
    total = (s["x"].float() + s["residual"].float()).to(t)            # the sum is kept in the inputs' type, and what is kept is normed
    x, w = total.float(), s["weight"].float()
    rstd = torch.rsqrt(x.square().mean(-1) + EPS)
    y = x * rstd[:, None] * w
    out = {"sum": total, "rstd": rstd}
    if c["eight_bits"]:
        out["q"], out["scales"] = _eight_bits(y)
    else:
        out["y"] = y.to(t)
    if c["train"]:
        d_y = s["d_y"].float()
        wdy = w * d_y
        mean = (wdy * x).mean(-1, keepdim=True)
        r = rstd[:, None]
        out["dx"] = (r * (wdy - x * (r * r * mean)) + s["d_sum"].float()).to(t)
        out["dweight"] = (d_y * x * r).sum(0)
    return out


def _plain_logprobs(s):
    c = s["case"]
    x, tokens = s["logits"].float(), s["tokens"].long()
    aimed = tokens >= 0
    at = tokens.clamp(min=0)[:, None]
    top = x.amax(-1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(-1, keepdim=True)
    lse = top + total.log()
    away = (x - top).masked_fill_(e == 0, 0.0)
    entropy = total.log() - (e * away).sum(-1, keepdim=True) / total
    out = {"logprob": torch.where(aimed, (x.gather(1, at) - lse)[:, 0], 0.0), "entropy": entropy[:, 0], "lse": lse[:, 0]}
    if c["top"]:
        bits = (x + 0.0).view(torch.int32)
        rank = (bits ^ ((bits >> 31) & 0x7fffffff)).long() << 32      # larger numbers first, then the lower index
        rank += 0xffffffff - torch.arange(c["vocabulary"], device=x.device)
        best = 0xffffffff - (rank.topk(c["top"], dim=-1).values & 0xffffffff)
        out["top_tokens"] = best.to(torch.int32)
        out["top_logprobs"] = x.gather(1, best) - lse
    if c["train"]:
        p = e.div_(total)
        g = torch.where(aimed, s["d_logprob"], 0.0)[:, None]
        away = (away + (top - lse)).masked_fill_(p == 0, 0.0)
        d = -p * (g + s["d_entropy"][:, None] * (away + entropy))
        d.scatter_add_(1, at, g)
        out["d_logits"] = d.to(TYPES[c["type"]])
    return out


def _plain_clip(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = (s["max_norm"] / norm).clamp(max=1.0).float()
    return {"norm": norm.float(), "clipped": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


# ---------------------------------------------------------------------------------------------
# the package's entry points

def _own_attention(s):
    import paper_2507_16274_amd as S
    keep = s["keep"]
    f = S.stalloc_attention(s["q"], s["k"], s["v"], s["bounds"], out=keep.get("f"), workspace_cache=keep)
    keep["f"] = f
    if not s["case"]["train"]:
        return {"o": f["o"], "lse": f["lse"]}
    b = S.stalloc_attention_backward(s["d_o"], s["q"], s["k"], s["v"], f["o"], f["lse"], s["bounds"], out=keep.get("b"), workspace_cache=keep)
    keep["b"] = b
    return {"o": f["o"], "lse": f["lse"], "dq": b["dq"], "dk": b["dk"], "dv": b["dv"]}


def _own_norm(s):
    import paper_2507_16274_amd as S
    keep, c = s["keep"], s["case"]
    f = S.stalloc_rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, eight_bits=c["eight_bits"], out=keep.get("f"))
    keep["f"] = f
    out = {"sum": f["sum"], "rstd": f["rstd"]}
    out.update({"q": f["q"], "scales": f["scales"]} if c["eight_bits"] else {"y": f["y"]})
    if c["train"]:
        b = S.stalloc_rms_norm_backward(s["d_y"], f["sum"], s["weight"], f["rstd"], d_sum=s["d_sum"], out=keep.get("b"), workspace_cache=keep)
        keep["b"] = b
        out.update({"dx": b["dx"], "dweight": b["dweight"]})
    return out


def _own_logprobs(s):
    import paper_2507_16274_amd as S
    keep, c = s["keep"], s["case"]
    f = S.stalloc_token_logprobs(s["logits"], s["tokens"], top=c["top"], out=keep.get("f"), workspace_cache=keep)
    keep["f"] = f
    out = {x: f[x] for x in ("logprob", "entropy", "lse")}
    if c["top"]:
        out.update({"top_tokens": f["top_tokens"], "top_logprobs": f["top_logprobs"]})
    if c["train"]:
        b = S.stalloc_token_logprobs_backward(s["logits"], s["tokens"], f["lse"], f["entropy"], s["d_logprob"], s["d_entropy"], out=keep.get("b"))
        keep["b"] = b
        out["d_logits"] = b["d_logits"]
    return out


def _own_clip(s):
    import paper_2507_16274_amd as S
    keep = s["keep"]
    if "list" not in keep:                     # made once by a program whose gradients stay where they are
        keep["clipped"] = [torch.empty_like(g) for g in s["grads"]]
        keep["list"] = S.stalloc_tensor_list(s["grads"], keep["clipped"])
    f = S.stalloc_clip_gradients(keep["list"], s["max_norm"], out=keep.get("f"), workspace_cache=keep)
    keep["f"] = f
    return {"norm": f["norm"][0], "clipped": keep["clipped"]}


PLAIN = {"attention": _plain_attention, "norm": _plain_norm, "logprobs": _plain_logprobs, "clip": _plain_clip}
OWN = {"attention": _own_attention, "norm": _own_norm, "logprobs": _own_logprobs, "clip": _own_clip}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


def work(case):
    c = case
    size = {"f32": 4, "bf16": 2, "f16": 2}[c.get("type", "f32")]
    if c["op"] == "attention":
        cuts = _bounds(c)
        pairs = c["heads"] * sum((b - a) * (b - a + 1) // 2 for a, b in zip(cuts, cuts[1:]))
        q, kv = c["tokens"] * c["heads"] * c["head_dim"] * size, c["tokens"] * c["kv_heads"] * c["head_dim"] * size
        nbytes = 2 * q + 2 * kv + 4 * c["tokens"] * c["heads"]
        if c["train"]:
            nbytes += 2 * q + 2 * kv           # the gradient of the output read, three gradients written
        return {"bytes": nbytes, "flops": pairs * c["head_dim"] * (14 if c["train"] else 4)}
    if c["op"] == "norm":
        each = c["rows"] * c["width"]
        nbytes = 3 * each * size + 4 * c["rows"]
        nbytes += each + 4 * c["rows"] * -(-c["width"] // BLOCK) if c["eight_bits"] else each * size
        return {"bytes": nbytes + (3 * each * size if c["train"] else 0), "flops": each * (14 if c["train"] else 6)}
    if c["op"] == "logprobs":
        each = c["rows"] * c["vocabulary"]
        return {"bytes": each * size * (2 if c["train"] else 1) + c["rows"] * (16 + 8 * c["top"]), "flops": each * (10 if c["train"] else 5)}
    each = sum(c["bucket"] + 3 * i for i in range(c["buckets"])) + c["small_width"] * c["small"]
    return {"bytes": 2 * each * size, "flops": 3 * each}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_attention(s):
    c, cuts = s["case"], _bounds(s["case"])
    n, h, g, d = c["tokens"], c["heads"], c["kv_heads"], c["head_dim"]
    q, k, v = (s[x].double() for x in ("q", "k", "v"))
    zero = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")                     # noqa: E731
    out = {"o": zero(n, h, d), "lse": zero(h, n) - float("inf")}
    if c["train"]:
        d_o = s["d_o"].double()
        out.update({"dq": zero(n, h, d), "dk": zero(n, g, d), "dv": zero(n, g, d)})
    for a, b in zip(cuts, cuts[1:]):
        if a == b:
            continue
        later = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
        for head in range(h):
            kv = head * g // h
            x = (q[a:b, head] @ k[a:b, kv].T) / math.sqrt(d)
            x[later] = -float("inf")
            lse = torch.logsumexp(x, -1)
            x = torch.exp(x - lse[:, None])
            out["o"][a:b, head] = x @ v[a:b, kv]
            out["lse"][head, a:b] = lse
            if c["train"]:
                up = d_o[a:b, head]
                out["dv"][a:b, kv] += x.T @ up
                y = x * (up @ v[a:b, kv].T - (up * out["o"][a:b, head]).sum(-1)[:, None]) / math.sqrt(d)
                out["dq"][a:b, head] = y @ k[a:b, kv]
                out["dk"][a:b, kv] += y.T @ q[a:b, head]
    return out


def _exact_norm(s):
    c = s["case"]
    x = (s["x"].double() + s["residual"].double()).to(TYPES[c["type"]]).double()
    w = s["weight"].double()
    inverse = 1.0 / torch.sqrt((x ** 2).sum(-1) / c["width"] + EPS)
    y = w * x * inverse[:, None]
    out = {"sum": x, "rstd": inverse}
    if c["eight_bits"]:
        cols = -(-c["width"] // BLOCK)
        scales, q = torch.empty(c["rows"], cols, dtype=torch.float64, device="cuda"), torch.empty_like(y)
        for j in range(cols):
            part = y[:, j * BLOCK:(j + 1) * BLOCK]
            scales[:, j] = torch.clamp(part.abs().max(-1).values / E4M3_MAX, min=LEAST_SCALE)
            q[:, j * BLOCK:(j + 1) * BLOCK] = part / scales[:, j:j + 1]
        out["q"], out["scales"] = q.float().clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scales
    else:
        out["y"] = y
    if c["train"]:
        d_y = s["d_y"].double()
        normed = x * inverse[:, None]
        through = (w * d_y - normed * (w * d_y * normed).mean(-1, keepdim=True)) * inverse[:, None]
        out["dx"], out["dweight"] = through + s["d_sum"].double(), (d_y * normed).sum(0)
    return out


def _exact_logprobs(s):
    c = s["case"]
    n, v = c["rows"], c["vocabulary"]
    got = []
    for a in range(0, n, 512):
        x, tokens = s["logits"][a:a + 512].double(), s["tokens"][a:a + 512].long()
        log_p = torch.log_softmax(x, -1)
        p = torch.exp(log_p)
        safe = torch.where(p > 0, log_p, 0.0)
        entropy = -(p * safe).sum(-1)
        aimed = tokens >= 0
        part = {"logprob": torch.where(aimed, log_p.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0), "entropy": entropy,
                "lse": torch.logsumexp(x, -1)}
        if c["top"]:
            part["top_logprobs"] = log_p.sort(-1, descending=True).values[:, :c["top"]]
        if c["train"]:
            g = torch.where(aimed, s["d_logprob"][a:a + 512].double(), 0.0)
            hot = torch.zeros_like(p)
            hot[torch.arange(p.shape[0], device="cuda"), tokens.clamp(min=0)] = aimed.double()
            part["d_logits"] = (hot - p) * g[:, None] - s["d_entropy"][a:a + 512].double()[:, None] * p * (safe + entropy[:, None])
        got.append(part)
    out = {x: torch.cat([part[x] for part in got]) for x in got[0]}
    if c["top"]:
        out["top_tokens"] = None
    return out


def _exact_clip(s):
    total = sum(float((g.double() ** 2).sum()) for g in s["grads"])
    norm = math.sqrt(total)
    factor = min(1.0, s["max_norm"] / norm)
    return {"norm": norm, "clipped": [g.double() * factor for g in s["grads"]]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "norm": _exact_norm, "logprobs": _exact_logprobs, "clip": _exact_clip}[case["op"]](s)
