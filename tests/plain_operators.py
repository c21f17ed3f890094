"""Operators of a training step from their definitions, in 64 bits on the CPU, with bounds on what the kernels' roundings may
change.  A rounding to type t is off by at most half(t) of the value."""
import math

import torch

INF = float("inf")


def half(t):
    """Half a step of the type, relative to the value."""
    return torch.finfo(t).eps / 2


def attention(q, k, v, bounds, scale, d_o=None):
    """o, lse and, for d_o, dq, dk, dv of packed causal attention; `slack`: for every output, what the kernel's roundings can
    change at most: weights and their gradients are rounded to the inputs' type t for the second products, outputs once more;
    the stored o that the backward pass starts from is off by its own bound; scores are sums of head_dim products in 32 bits."""
    t, f32 = q.dtype, 2.0 ** -24
    q, k, v = (x.double().cpu() for x in (q, k, v))
    d_o = None if d_o is None else d_o.double().cpu()
    n, h, d = q.shape
    g = k.shape[1]
    u = half(t)
    out = {"o": torch.zeros_like(q), "lse": torch.full((h, n), -INF, dtype=torch.float64)}
    slack = {"o": torch.zeros_like(q), "lse": torch.zeros(h, n, dtype=torch.float64)}
    if d_o is not None:
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            out[name], slack[name] = torch.zeros_like(like), torch.zeros_like(like)
    for a, b in zip(bounds, bounds[1:]):
        if a >= b:
            continue
        seen = torch.ones(b - a, b - a, dtype=torch.bool).tril()
        for head in range(h):
            kv = head * g // h
            qs, ks, vs = q[a:b, head], k[a:b, kv], v[a:b, kv]
            s = (qs @ ks.T * scale).masked_fill(~seen, -INF)
            lse = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[:, None])
            # scores: head_dim + 2 roundings of partial sums, the shift and the exponential a few more of |s|; twice: weight and sum
            ds_ = ((d + 2) * f32 * (qs.abs() @ ks.T.abs()) * scale + 8 * f32 * s.masked_fill(~seen, 0.0).abs()).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
            rel = 2 * ds_ + 16 * f32
            o = p @ vs
            p_abs = p @ vs.abs()
            out["o"][a:b, head], out["lse"][head, a:b] = o, lse
            slack["o"][a:b, head] = (u + rel + (b - a) * f32) * p_abs * (1 + u) + u * o.abs()
            slack["lse"][head, a:b] = ds_[:, 0] + (8 + math.log2(b - a + 1)) * f32 * (1 + lse.abs())
            if d_o is None:
                continue
            up = d_o[a:b, head]
            dp = up @ vs.T
            dots = (up * o).sum(-1, keepdim=True)
            ds = p * (dp - dots) * scale
            off_dots = (up.abs() * slack["o"][a:b, head]).sum(-1, keepdim=True) + (d + 2) * f32 * (up.abs() * o.abs()).sum(-1, keepdim=True)
            off_ds = (u + rel + 8 * f32) * ds.abs() + p * scale * (off_dots + (d + 2) * f32 * (up.abs() @ vs.T.abs()) + 4 * f32 * (dp.abs() + dots.abs()))
            m = (b - a) * f32
            if t == torch.float16:           # (numbers below the type's smallest normal are rounded to multiples of its smallest one)
                off_ds = off_ds + 2.0 ** -25 * seen
            dq, dk, dv = ds @ ks, ds.T @ qs, p.T @ up
            out["dq"][a:b, head] = dq
            out["dk"][a:b, kv] += dk
            out["dv"][a:b, kv] += dv
            slack["dq"][a:b, head] = off_ds @ ks.abs() + m * (ds.abs() @ ks.abs())
            slack["dk"][a:b, kv] += off_ds.T @ qs.abs() + m * (ds.abs().T @ qs.abs())
            slack["dv"][a:b, kv] += ((u + m + rel) * p).T @ up.abs() + (2.0 ** -25 if t == torch.float16 else 0.0) * (seen.double().T @ up.abs())
    least = torch.finfo(t).tiny * u * 2
    for name in slack:
        if name not in ("o", "lse"):
            slack[name] = slack[name] * (1 + u) + u * out[name].abs()
        if name != "lse":
            slack[name] = slack[name] + least
    return out, slack


def rms_norm(x, residual, weight, eps):
    """sum (rounded as it is kept), rstd, y."""
    t = x.dtype
    total = x if residual is None else (x.double() + residual.double()).float().to(t)
    s = total.double()
    rstd = 1.0 / torch.sqrt((s ** 2).mean(-1) + eps)
    return total, rstd, s * rstd[:, None] * weight.double()


def eight_bits(y):
    """Scales of every row's blocks of 128 columns."""
    rows, width = y.shape
    cols = -(-width // 128)
    padded = torch.zeros(rows, cols * 128, dtype=y.dtype)
    padded[:, :width] = y
    return padded.view(rows, cols, 128).abs().amax(-1).clamp(min=448 * 2.0 ** -126) / 448


def rms_norm_backward(d_y, s, weight, rstd, d_sum):
    s, d_y, w = s.double(), d_y.double(), weight.double()
    r = rstd.double()[:, None]
    g = w * d_y
    dx = r * (g - s * r * r * (g * s).mean(-1, keepdim=True))
    return dx if d_sum is None else dx + d_sum.double(), (d_y * s * r).sum(0)


def token_logprobs(x, tokens, top):
    """logprob, entropy, lse, top_tokens, top_logprobs."""
    x = x.double()
    m = x.amax(-1, keepdim=True)
    empty = m == -INF
    e = torch.exp(x - m.masked_fill(empty, 0.0))
    z = e.sum(-1, keepdim=True)
    lse = m + torch.log(z)
    log_p = torch.where(empty, -INF, (x - m.masked_fill(empty, 0.0)) - torch.log(z))    # (x - lse would lose ln z next to lowest values)
    p = torch.exp(log_p)
    entropy = -(p * log_p.masked_fill(p == 0, 0.0)).sum(-1)
    picked = log_p.gather(1, tokens.long().clamp(min=0)[:, None])[:, 0]
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :top]
    return torch.where(tokens >= 0, picked, 0.0), entropy, lse[:, 0], order, log_p.gather(1, order)


def token_logprobs_backward(x, tokens, d_logprob, d_entropy):
    _, entropy, lse, _, _ = token_logprobs(x, tokens, 1)
    empty = (lse == -INF)[:, None]
    m = x.double().amax(-1, keepdim=True).masked_fill(empty, 0.0)
    log_p = torch.where(empty, -INF, (x.double() - m) - torch.log(torch.exp(x.double() - m).sum(-1, keepdim=True)))
    p = torch.exp(log_p)
    aimed = (tokens >= 0)[:, None] & ~empty
    g = torch.where(aimed, d_logprob.double()[:, None], 0.0)
    hot = torch.zeros_like(p).scatter_(1, tokens.long().clamp(min=0)[:, None], 1.0)
    d = g * (hot - p)
    if d_entropy is not None:
        d = d - d_entropy.double()[:, None] * p * (log_p.masked_fill(p == 0, 0.0) + entropy[:, None])
    return d.masked_fill(empty, 0.0)
