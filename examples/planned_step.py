"""A training step that runs at the addresses of a plan.

A step of a small causal language model (packed sequences, grouped heads, norms with residual, log probabilities of the
targets, all gradients, clipping, update) takes every buffer from a `Memory`.  The first step is profiled: every buffer is a tensor
of its own, and what it asks for becomes an allocation trace.  stalloc_plan places the trace; from then on the step runs inside one
pool, at the planned addresses; besides there are only the weights and a few words.  What it computes stays the same to the last bit.

    python examples/planned_step.py [--layers 4 --hidden 1024 --tokens 4096 ...]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
from types import SimpleNamespace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_16274_amd as S  # noqa: E402

ROUND = 512                                    # sizes are rounded up to this many bytes, as in the other traces


class Memory:
    """Where the buffers of a step are.  Profiling: tensors of their own, every request and release noted.  Planned: views of one pool at the
    addresses given for the requests, in their order."""

    def __init__(self, pool=None, offsets=None):
        self.pool, self.offsets = pool, offsets
        self.begin()

    def begin(self):
        self.count, self.clock, self.live = 0, 0, {}
        self.size, self.t_alloc, self.t_free = [], [], []

    def take(self, *shape, dtype=torch.bfloat16):
        nbytes = math.prod(shape) * dtype.itemsize
        if self.pool is None:
            t = torch.empty(shape, dtype=dtype, device="cuda")
            self._note(t, nbytes)
        else:
            at = self.offsets[self.count]
            t = self.pool[at:at + nbytes].view(dtype).view(shape)
            self.count += 1
        return t

    def give(self, *tensors):
        """These buffers are not needed any more."""
        if self.pool is None:
            for t in tensors:
                self.t_free[self.live.pop(t.data_ptr())] = self.clock
                self.clock += 1

    def call(self, fn, *args, **more):
        """A call that needs a workspace: it is a request like the others, over when the call is."""
        if self.pool is None:
            out = fn(*args, workspace_cache={}, **more)
            self._note(out["workspace"], out["workspace"].numel())
            self.give(out["workspace"])
            return out
        at = self.offsets[self.count]
        planned = self.pool[at:at + self.sizes[self.count]]
        self.count += 1
        out = fn(*args, workspace_cache={"ws": planned}, **more)
        if out["workspace"].data_ptr() != planned.data_ptr():
            raise MemoryError("a workspace is larger than what was planned for it")
        return out

    def _note(self, t, nbytes):
        self.live[t.data_ptr()] = self.count
        self.count += 1
        self.size.append(max(1, -(-nbytes // ROUND)) * ROUND)
        self.t_alloc.append(self.clock)
        self.t_free.append(-1)
        self.clock += 1

    def trace(self):
        assert not self.live, "a buffer of the step was never given back"
        return SimpleNamespace(size=np.array(self.size, np.uint64), t_alloc=np.array(self.t_alloc, np.uint32),
                               t_free=np.array(self.t_free, np.uint32), t_end=self.clock)


def plan_of(trace, orders=64):
    """(addresses, extent, lower bound) of the best of `orders` placement orders."""
    size, ta, tf = S.trace_to_device(trace)
    made = S.stalloc_make_orders(size, ta, tf, trace.t_end, orders)
    plan = S.stalloc_plan(size, ta, tf, trace.t_end, made["orders"], want_offsets=False)
    check = S.stalloc_validate(size, ta, tf, trace.t_end, plan["best_offsets"].view(1, -1))
    bound = S.stalloc_lower_bound(size, ta, tf, trace.t_end)
    for out in (made, plan, check, bound):
        S.check_status(out)
    assert int(check["conflicts"].item()) == 0
    return plan["best_offsets"].tolist(), int(plan["peaks"].min()), int(bound["lower_bound"].item())


def planned(trace, orders=64):
    """A Memory for steps like the one that was profiled, and what the plan says."""
    offsets, extent, bound = plan_of(trace, orders)
    memory = Memory(torch.empty(extent, dtype=torch.uint8, device="cuda"), offsets)
    memory.sizes = [int(s) for s in trace.size]
    return memory, extent, bound


# ---------------------------------------------------------------------------------------------
# the model

def make_model(c, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def weight(rows, cols):
        return (torch.randn(rows, cols, generator=gen, device="cuda") / math.sqrt(cols)).to(torch.bfloat16)

    layers = [{"norm": torch.ones(c.hidden, dtype=torch.bfloat16, device="cuda"), "norm2": torch.ones(c.hidden, dtype=torch.bfloat16, device="cuda"),
               "qkv": weight((c.heads + 2 * c.kv_heads) * c.head_dim, c.hidden), "out": weight(c.hidden, c.heads * c.head_dim),
               "up": weight(4 * c.hidden, c.hidden), "down": weight(c.hidden, 4 * c.hidden)} for _ in range(c.layers)]
    return {"layers": layers, "norm": torch.ones(c.hidden, dtype=torch.bfloat16, device="cuda"), "vocabulary": weight(c.vocabulary, c.hidden),
            "embedding": weight(c.vocabulary, c.hidden).mul_(math.sqrt(c.hidden))}           # (the embedding is not trained)


def make_batch(c, seed=1):
    """Tokens of packed sequences, each token's target the next one of its sequence, none for a sequence's last."""
    rng = np.random.default_rng(seed)
    cuts = np.sort(rng.choice(np.arange(1, c.tokens), c.sequences - 1, replace=False)) if c.sequences > 1 else np.array([], int)
    bounds = np.concatenate([[0], cuts, [c.tokens]]).astype(np.int32)
    tokens = (rng.integers(0, c.vocabulary, c.tokens) % 97).astype(np.int32)
    targets = np.roll(tokens, -1)
    targets[bounds[1:] - 1] = -1
    dev = lambda x: torch.from_numpy(x).cuda()                                               # noqa: E731
    return {"tokens": dev(tokens).long(), "targets": dev(targets), "bounds": dev(bounds), "count": int((targets >= 0).sum())}


def step(c, model, batch, mem, lr=0.05, max_norm=1.0):
    """One training step; returns the loss and the gradients' norm (device tensors)."""
    n, w = c.tokens, c.hidden
    take, give = mem.take, mem.give
    mem.begin()
    split = lambda t: [x.unflatten(1, (-1, c.head_dim)) for x in t.split((c.heads * c.head_dim, c.kv_heads * c.head_dim, c.kv_heads * c.head_dim), dim=1)]  # noqa: E731
    norm = lambda x, weight, residual: S.stalloc_rms_norm(x, weight, residual=residual, out={"sum": residual, "y": take(n, w), "rstd": take(n, dtype=torch.float32)})  # noqa: E731

    def product(a, b, rows, cols):
        return torch.mm(a, b, out=take(rows, cols))

    # Forward.  What a layer passes on is added to the stream by the next norm, in place; norms keep what the stream was.
    stream = torch.index_select(model["embedding"], 0, batch["tokens"], out=take(n, w))
    fresh, saved = take(n, w).zero_(), []
    for layer in model["layers"]:
        k = {}
        for half, (weight, first) in enumerate((("norm", "qkv"), ("norm2", "up"))):
            f = norm(fresh, layer[weight], stream)
            give(fresh)
            k[half] = {"sum": take(n, w).copy_(stream), "y": f["y"], "rstd": f["rstd"]}
            k[first] = product(f["y"], layer[first].t(), n, layer[first].shape[0])
            if half == 0:
                q, key, v = split(k["qkv"])
                k["o"], k["lse"] = take(n, c.heads, c.head_dim), take(c.heads, n, dtype=torch.float32)
                mem.call(S.stalloc_attention, q, key, v, batch["bounds"], out={"o": k["o"], "lse": k["lse"], "status": c.status})
                fresh = product(k["o"].flatten(1), layer["out"].t(), n, w)
            else:
                torch.clamp(k["up"], min=0.0, out=k["up"])
                fresh = product(k["up"], layer["down"].t(), n, w)
        saved.append(k)
    last = norm(fresh, model["norm"], stream)
    give(fresh)
    logits = product(last["y"], model["vocabulary"].t(), n, c.vocabulary)
    one = {name: take(n, dtype=torch.float32) for name in ("logprob", "entropy", "lse")}
    mem.call(S.stalloc_token_logprobs, logits, batch["targets"], out={**one, "status": c.token_status})
    loss = one["logprob"].sum() / -batch["count"]

    # Backward.  The gradient of the logits takes their place; `through` is the gradient of the stream.
    grads = []

    def weight_gradient(param, d_out, x):
        g = torch.mm(d_out.t(), x, out=take(*param.shape))
        grads.append((param, g))

    def norm_backward(d_y, total, weight, rstd, through):
        g = take(w, dtype=torch.float32)
        out = {"dx": d_y, "dweight": g}
        mem.call(S.stalloc_rms_norm_backward, d_y, total, weight, rstd, d_sum=through, out=out)
        grads.append((weight, g))
        return d_y

    d_logprob = take(n, dtype=torch.float32).fill_(-1.0 / batch["count"])
    S.stalloc_token_logprobs_backward(logits, batch["targets"], one["lse"], one["entropy"], d_logprob, out={"d_logits": logits, "status": c.token_status})
    weight_gradient(model["vocabulary"], logits, last["y"])
    d_y = product(logits, model["vocabulary"], n, w)
    give(logits, d_logprob, *one.values())
    through = norm_backward(d_y, stream, model["norm"], last["rstd"], None)
    give(last["y"], last["rstd"], stream)
    for layer, k in zip(reversed(model["layers"]), reversed(saved)):
        weight_gradient(layer["down"], through, k["up"])
        d_up = product(through, layer["down"], n, 4 * w)
        d_up.mul_(torch.sign(k["up"], out=k["up"]))
        give(k["up"])
        weight_gradient(layer["up"], d_up, k[1]["y"])
        d_y = product(d_up, layer["up"], n, w)
        give(d_up, k[1]["y"])
        before, through = through, norm_backward(d_y, k[1]["sum"], layer["norm2"], k[1]["rstd"], through)
        give(before, k[1]["sum"], k[1]["rstd"])
        weight_gradient(layer["out"], through, k["o"].flatten(1))
        d_o = product(through, layer["out"], n, c.heads * c.head_dim)
        d_qkv = take(n, (c.heads + 2 * c.kv_heads) * c.head_dim)
        q, key, v = split(k["qkv"])
        mem.call(S.stalloc_attention_backward, d_o.unflatten(1, (-1, c.head_dim)), q, key, v, k["o"], k["lse"], batch["bounds"],
                 out={**dict(zip(("dq", "dk", "dv"), split(d_qkv))), "status": c.status})
        give(d_o, k["qkv"], k["o"], k["lse"])
        weight_gradient(layer["qkv"], d_qkv, k[0]["y"])
        d_y = product(d_qkv, layer["qkv"], n, w)
        give(d_qkv, k[0]["y"])
        before, through = through, norm_backward(d_y, k[0]["sum"], layer["norm"], k[0]["rstd"], through)
        give(before, k[0]["sum"], k[0]["rstd"])
    give(through)

    # All gradients to a norm of at most max_norm, in place; then the update.
    tensors = [g for _, g in grads]
    clipped = mem.call(S.stalloc_clip_gradients, S.stalloc_tensor_list(tensors, tensors), max_norm, out={"norm": c.norm, "factor": c.factor})
    for param, g in grads:
        param.add_(g.to(param.dtype) if g.dtype != param.dtype else g, alpha=-lr)
    give(*tensors)
    return loss, clipped["norm"].clone()


def config(**more):
    c = {"layers": 4, "hidden": 1024, "heads": 8, "kv_heads": 2, "head_dim": 128, "vocabulary": 32000, "tokens": 4096, "sequences": 7, **more}
    c = SimpleNamespace(**c)
    # (A call overwrites its status, so calls that can go wrong in different ways have words of their own.)
    c.status, c.token_status = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    c.norm, c.factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    return c


def run(c, steps=3, orders=64, batch=None):
    """Profiles a step, plans it, runs `steps` of them both ways.  Returns a report."""
    batch = batch or make_batch(c)
    apart, pooled = make_model(c), make_model(c)
    profiler = Memory()
    results = [[], []]
    results[0].append(step(c, apart, batch, profiler))
    trace = profiler.trace()
    memory, extent, bound = planned(trace, orders)
    for _ in range(steps - 1):
        results[0].append(step(c, apart, batch, profiler))
    for _ in range(steps):
        results[1].append(step(c, pooled, batch, memory))
    torch.cuda.synchronize()
    for status in (c.status, c.token_status):
        S.check_status({"status": status})
    weights = [[m["vocabulary"], m["norm"]] + [x for layer in m["layers"] for x in layer.values()] for m in (apart, pooled)]
    return {"requests": len(trace.size), "sum": int(trace.size.sum()), "bound": bound, "extent": extent,
            "losses": [[float(loss) for loss, _ in r] for r in results], "norms": [[float(norm) for _, norm in r] for r in results],
            "same": all(torch.equal(a, b) for a, b in zip(*weights))}


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("layers", 4), ("hidden", 1024), ("heads", 8), ("kv_heads", 2), ("head_dim", 128), ("vocabulary", 32000), ("tokens", 4096), ("sequences", 7)):
        ap.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    ap.add_argument("--steps", type=int, default=3)
    a = vars(ap.parse_args())
    steps = a.pop("steps")
    r = run(config(**a), steps)
    mib = lambda b: "%.1f MiB" % (b / 2 ** 20)                                               # noqa: E731
    print("%d requests, %s if none shared its place; most alive at once %s; plan %s" % (r["requests"], mib(r["sum"]), mib(r["bound"]), mib(r["extent"])))
    print("losses with buffers of their own: %s" % r["losses"][0])
    print("losses at the planned addresses:  %s" % r["losses"][1])
    print("weights after %d steps: %s" % (steps, "the same" if r["same"] else "DIFFERENT"))
    return 0 if r["same"] else 1


if __name__ == "__main__":
    sys.exit(main())
