"""Timed cases of the layer operators: what a program that trains n worker
replicas on one GPU calls between two local steps.

Every worker's parameters are one row of the [n, ld] buffers; a call takes the
token rows of all workers, packed one worker after the other, and each worker
uses the weights at a given column of its own row.  Gradients of weights are
written into the rows [n, ld] of fp32 gradients that the local step reads.

Fields of a case:
  pass      "embedding", "embedding_grad", "norm", "norm_grad", "linear",
            "linear_input" (gradient of the input), "linear_weight" (of the
            weight)
  n         workers
  rows      token rows of all workers together
  split     how they are spread: "even", "ragged" (a worker's share is random)
            or "gaps" (ragged, every third worker has none)
  act       type of activations ("f32" or "bf16")
  params    type of parameters (likewise)
  vocab     rows of the embedding table (embedding passes)
  width     its columns, or the norm's
  n_in, n_out  the features of a linear layer
  shift     columns of the worker's row in front of the weights
"""
import math
import random

import torch

own = False

EPS = 1e-5
SCALE = 0.5
PASSES = ("embedding", "embedding_grad", "norm", "norm_grad", "linear", "linear_input", "linear_weight")
MOST_BYTES = 2_000_000_000   # of a drawn case, below the largest listed one
MOST_FLOPS = 200_000_000_000


def listed():
    return [
        # the smallest call: one token per worker, latency only
        dict(name="embedding-n4-1token", **_table("embedding", 4, 4, 512, 64, "f32", "f32")),
        # a batch of 16 workers, two sequences of 2048 tokens each, 32K vocabulary
        dict(name="embedding-n16-64k", **_table("embedding", 16, 65_536, 32_000, 1024, "bf16", "f32")),
        # odd sizes, workers without tokens, fp32 throughout, weights that start at an odd column
        dict(name="embedding_grad-n5-odd", **_table("embedding_grad", 5, 3001, 1237, 321, "f32", "f32", "gaps", 3)),
        # the dense gradient of the 32K table for every one of 16 workers
        dict(name="embedding_grad-n16-64k", **_table("embedding_grad", 16, 65_536, 32_000, 1024, "bf16", "f32")),
        # the norms of a batch, forward and backward
        dict(name="norm-n16-64k", **_norm("norm", 16, 65_536, 1024, "bf16", "f32")),
        dict(name="norm_grad-n16-64k", **_norm("norm_grad", 16, 65_536, 1024, "bf16", "f32")),
        dict(name="norm_grad-n7-odd", **_norm("norm_grad", 7, 5003, 1023, "f32", "f32", "ragged", 5)),
        # one token of every worker through one layer: reading the weights is all there is
        dict(name="linear-n16-1row", **_linear("linear", 16, 16, 2048, 2048, "bf16", "f32")),
        # a batch through a widening layer, bf16 replicas
        dict(name="linear-n16-32k", **_linear("linear", 16, 32_768, 1024, 4096, "bf16", "bf16")),
        # the way back through a square layer, fp32 replicas under bf16 activations
        dict(name="linear_input-n16-32k", **_linear("linear_input", 16, 32_768, 2048, 2048, "bf16", "f32")),
        # the weight's gradient of a ragged batch
        dict(name="linear_weight-n8-ragged", **_linear("linear_weight", 8, 30_011, 2048, 2048, "bf16", "f32", "ragged")),
        # fp32 throughout, odd features and rows
        dict(name="linear_weight-n3-odd", **_linear("linear_weight", 3, 1111, 257, 513, "f32", "f32", "ragged", 1)),
    ]


def _table(kind, n, rows, vocab, width, act, params, split="even", shift=0):
    return {"pass": kind, "n": n, "rows": rows, "vocab": vocab, "width": width, "act": act, "params": params,
            "split": split, "shift": shift}


def _norm(kind, n, rows, width, act, params, split="even", shift=0):
    return {"pass": kind, "n": n, "rows": rows, "width": width, "act": act, "params": params, "split": split,
            "shift": shift}


def _linear(kind, n, rows, n_in, n_out, act, params, split="even", shift=0):
    return {"pass": kind, "n": n, "rows": rows, "n_in": n_in, "n_out": n_out, "act": act, "params": params,
            "split": split, "shift": shift}


def _between(rng, low, high):
    """Spread over the logarithm; a third of the values are rounded to a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 1 / 3 and v >= 64:
        v = v // 64 * 64
    return max(low, min(high, v))


def draw(rng):
    while True:
        kind = rng.choice(PASSES)
        act, params = rng.choice((("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")))
        n = _between(rng, 1, 32)
        rows = _between(rng, n, 65_536)
        split = rng.choice(("even", "even", "ragged", "gaps"))
        shift = rng.choice((0, 0, 64, 1, 6))
        if kind.startswith("embedding"):
            c = _table(kind, n, rows, _between(rng, 16, 50_000), _between(rng, 16, 4096), act, params, split, shift)
        elif kind.startswith("norm"):
            c = _norm(kind, n, rows, _between(rng, 16, 8192), act, params, split, shift)
        else:
            c = _linear(kind, n, rows, _between(rng, 16, 4096), _between(rng, 16, 4096), act, params, split, shift)
        w = work(c)
        most = MOST_FLOPS if act == "bf16" else MOST_FLOPS // 8
        if w["bytes"] <= MOST_BYTES and w["flops"] <= most and _columns(c) * n <= 600_000_000:
            return c


def _row_ptr(c):
    """Where each worker's rows begin (n + 1 numbers), from the case alone."""
    n, rows = c["n"], c["rows"]
    if c["split"] == "even":
        return [rows * i // n for i in range(n + 1)]
    rng = random.Random(rows * 64 + n)
    share = [rng.random() for _ in range(n)]
    if c["split"] == "gaps" and n > 1:
        share = [0.0 if i % 3 == 1 else s for i, s in enumerate(share)]
    total, at, out = sum(share), 0.0, [0]
    for s in share:
        at += s
        out.append(int(rows * at / total))
    out[-1] = rows
    if c["split"] == "gaps" and n > 1 and (n - 1) % 3 == 1:
        out[-2] = rows  # the last worker is one of those without rows
    return out


def _columns(c):
    """Parameters of one worker: those in front of the weights, then the weights."""
    if "vocab" in c:
        return c["shift"] + c["vocab"] * c["width"]
    if "n_in" in c:
        return c["shift"] + c["n_in"] * c["n_out"]
    return c["shift"] + 2 * c["width"]


_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _distinct(c):
    """How many table rows are looked up, on average, with the tokens of prepare()."""
    v, ptr = c["vocab"], _row_ptr(c)
    edge = (torch.arange(v + 1, dtype=torch.float64) / v) ** (1 / 3)
    p = edge[1:] - edge[:-1]
    counts, total = {}, 0.0
    for a, b in zip(ptr, ptr[1:]):
        counts[b - a] = counts.get(b - a, 0) + 1
    for rows, times in counts.items():
        total += times * float((1 - (1 - p) ** rows).sum())
    return total


def work(c):
    n, rows, sa, sp = c["n"], c["rows"], _BYTES[c["act"]], _BYTES[c["params"]]
    kind = c["pass"]
    if kind == "embedding":
        return {"bytes": 4 * rows + _distinct(c) * c["width"] * sp + rows * c["width"] * sa, "flops": rows * c["width"]}
    if kind == "embedding_grad":
        return {"bytes": 4 * rows + rows * c["width"] * sa + n * c["vocab"] * c["width"] * 4,
                "flops": 2 * rows * c["width"]}
    busy = sum(1 for a, b in zip(_row_ptr(c), _row_ptr(c)[1:]) if b > a)
    if kind == "norm":
        return {"bytes": 2 * rows * c["width"] * sa + 8 * rows + 2 * busy * c["width"] * sp,
                "flops": 8 * rows * c["width"]}
    if kind == "norm_grad":
        return {"bytes": 3 * rows * c["width"] * sa + 8 * rows + busy * c["width"] * sp + 2 * n * c["width"] * 4,
                "flops": 14 * rows * c["width"]}
    size = c["n_in"] * c["n_out"]
    flops = 2 * rows * size
    if kind == "linear_weight":
        return {"bytes": rows * (c["n_in"] + c["n_out"]) * sa + n * size * 4, "flops": flops}
    return {"bytes": rows * (c["n_in"] + c["n_out"]) * sa + busy * size * sp, "flops": flops}


def _normal(gen, shape, dtype, scale=1.0, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, scale, generator=gen).to(dtype)


def _inputs(c, seed):
    """The parameters [n, columns] and what the call takes, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, rows, kind = c["n"], c["rows"], c["pass"]
    act, par = _TYPE[c["act"]], _TYPE[c["params"]]
    s = {"c": c, "ptr": _row_ptr(c)}
    cols = _columns(c)
    if kind.startswith("embedding"):
        s["params"] = _normal(gen, (n, cols), par, 0.02)
        u = torch.empty(rows, dtype=torch.float64, device="cuda").uniform_(generator=gen)
        # frequent tokens first, as in a vocabulary sorted by frequency
        s["tokens"] = (u ** 3 * c["vocab"]).to(torch.int32).clamp_(max=c["vocab"] - 1)
        if kind == "embedding_grad":
            s["d"] = _normal(gen, (rows, c["width"]), act)
    elif kind.startswith("norm"):
        w = c["width"]
        s["params"] = _normal(gen, (n, cols), par, 0.1)
        s["params"][:, c["shift"]:c["shift"] + w] += 1  # gains near 1, biases near 0
        x = _normal(gen, (rows, w), torch.float32)
        scale = torch.empty((rows, 1), device="cuda").uniform_(0.5, 4.0, generator=gen)
        shift = torch.empty((rows, 1), device="cuda").normal_(0.0, 0.5, generator=gen)
        s["x"] = (x * scale + shift).to(act)  # a residual stream: rows of different size, off centre
        if kind == "norm_grad":
            s["d"] = _normal(gen, (rows, w), act)
            x = s["x"].double()
            mean = x.mean(1)
            s["stats"] = torch.stack((mean, ((x - mean[:, None]).square().mean(1) + EPS).rsqrt()), 1).float()
    else:
        k, m = c["n_in"], c["n_out"]
        s["params"] = _normal(gen, (n, cols), par, k ** -0.5)
        if kind != "linear_input":
            s["x"] = _normal(gen, (rows, k), act)
        if kind != "linear":
            s["d"] = _normal(gen, (rows, m), act)
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    if own:
        import numpy as np

        import paper_2606_11081_amd as g

        # the context of the workers; the outer state plays no part in these passes
        s["run"] = g.GASLoC(c["n"], _columns(c), param_dtype=c["params"], outer_momentum=0.0, consensus_momentum=0.0)
        s["run"].x[:, :_columns(c)].copy_(s.pop("params"))
        s["ptr"] = np.asarray(s["ptr"], dtype=np.int64)
        if c["pass"] in ("embedding_grad", "norm_grad", "linear_weight"):
            s["grads"] = torch.empty((c["n"], s["run"].ld), dtype=torch.float32, device="cuda")
    return s


def _run_own(s):
    c, run, ptr = s["c"], s["run"], s["ptr"]
    kind, at = c["pass"], c["shift"]
    if kind == "embedding":
        return run.embedding(at, c["vocab"], c["width"], s["tokens"], ptr, scale=SCALE, dtype=c["act"])
    if kind == "embedding_grad":
        run.embedding_grad(at, c["vocab"], c["width"], s["tokens"], ptr, s["d"], s["grads"], scale=SCALE)
        return s["grads"][:, at:at + c["vocab"] * c["width"]]
    if kind == "norm":
        return run.layer_norm(at, at + c["width"], c["width"], s["x"], ptr, eps=EPS)
    if kind == "norm_grad":
        dx = run.layer_norm_grad(at, at + c["width"], c["width"], s["x"], ptr, s["stats"], s["d"], s["grads"])
        return dx, s["grads"][:, at:at + 2 * c["width"]]
    if kind == "linear":
        return run.linear(at, c["n_out"], c["n_in"], s["x"], ptr)
    if kind == "linear_input":
        return run.linear_grad_input(at, c["n_out"], c["n_in"], s["d"], ptr)
    run.linear_grad_weight(at, c["n_out"], c["n_in"], s["x"], s["d"], ptr, s["grads"])
    return s["grads"][:, at:at + c["n_out"] * c["n_in"]]


def _run_plain(s):
    """Worker by worker, in fp32; weights meet bf16 activations rounded to bf16, as in a mixed-precision step."""
    c, params, at = s["c"], s["params"], s["c"]["shift"]
    kind, act, n = c["pass"], _TYPE[c["act"]], c["n"]
    spans = list(zip(s["ptr"], s["ptr"][1:]))
    if kind == "embedding":
        out = torch.empty((c["rows"], c["width"]), dtype=act, device="cuda")
        for i, (a, b) in enumerate(spans):
            table = params[i, at:].view(c["vocab"], c["width"])
            out[a:b] = (table[s["tokens"][a:b].long()].float() * SCALE).to(act)
        return out
    if kind == "embedding_grad":
        grads = torch.zeros((n, c["vocab"], c["width"]), dtype=torch.float32, device="cuda")
        for i, (a, b) in enumerate(spans):
            grads[i].index_add_(0, s["tokens"][a:b].long(), s["d"][a:b].float())
        return (grads * SCALE).view(n, -1)
    if kind in ("norm", "norm_grad"):
        w = c["width"]
        x = s["x"].float()
        if kind == "norm":
            mean = x.mean(1, keepdim=True)
            rstd = ((x - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
            out = torch.empty_like(s["x"])
            for i, (a, b) in enumerate(spans):
                gain, bias = params[i, at:at + w].float(), params[i, at + w:at + 2 * w].float()
                out[a:b] = ((x[a:b] - mean[a:b]) * rstd[a:b] * gain + bias).to(act)
            return out, torch.cat((mean, rstd), 1)
        mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
        hat, d = (x - mean) * rstd, s["d"].float()
        dx = torch.empty_like(s["x"])
        grads = torch.zeros((n, 2 * w), dtype=torch.float32, device="cuda")
        for i, (a, b) in enumerate(spans):
            h = d[a:b] * params[i, at:at + w].float()
            dx[a:b] = (rstd[a:b] * (h - h.mean(1, keepdim=True)
                                    - hat[a:b] * (h * hat[a:b]).mean(1, keepdim=True))).to(act)
            grads[i, :w] = (d[a:b] * hat[a:b]).sum(0)
            grads[i, w:] = d[a:b].sum(0)
        return dx, grads
    k, m = c["n_in"], c["n_out"]
    if kind == "linear_weight":
        grads = torch.empty((n, m, k), dtype=torch.float32, device="cuda")
        for i, (a, b) in enumerate(spans):
            grads[i] = s["d"][a:b].float().t() @ s["x"][a:b].float()
        return grads.view(n, -1)
    src = s["x"] if kind == "linear" else s["d"]
    out = torch.empty((c["rows"], m if kind == "linear" else k), dtype=act, device="cuda")
    for i, (a, b) in enumerate(spans):
        weight = params[i, at:at + m * k].view(m, k).to(act).float()
        out[a:b] = (src[a:b].float() @ (weight.t() if kind == "linear" else weight)).to(act)
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(c, seed):
    """The operators' definitions in fp64."""
    s = _inputs(c, seed)
    kind, at, ptr, n = c["pass"], c["shift"], s["ptr"], c["n"]
    worker = torch.repeat_interleave(torch.arange(n, device="cuda"),
                                     torch.tensor([b - a for a, b in zip(ptr, ptr[1:])], device="cuda"))
    if kind == "embedding":
        v, w = c["vocab"], c["width"]
        flat = s["params"][:, at:at + v * w].reshape(n * v, w)
        return flat.index_select(0, worker * v + s["tokens"].long()).double().mul_(SCALE)
    if kind == "embedding_grad":
        # sorted rows, running sums, differences at the ends of each token's stretch
        v, w = c["vocab"], c["width"]
        out = torch.zeros((n * v, w), dtype=torch.float64, device="cuda")
        key, order = torch.sort(worker * v + s["tokens"].long(), stable=True)
        if len(key):
            last = torch.ones_like(key, dtype=torch.bool)
            last[:-1] = key[1:] != key[:-1]
            ends = torch.nonzero(last).flatten()
            for j in range(0, w, 256):
                run_sum = s["d"][:, j:j + 256].double()[order].cumsum(0)[ends]
                run_sum[1:] -= run_sum[:-1].clone()
                out[key[ends], j:j + 256] = run_sum * SCALE
        return out.view(n, v * w)
    if kind in ("norm", "norm_grad"):
        w = c["width"]
        x = s["x"].double()
        gain = s["params"][:, at:at + w].double()[worker]
        if kind == "norm":
            mean = x.sum(1) / w
            centred = x - mean[:, None]
            rstd = 1.0 / torch.sqrt((centred * centred).sum(1) / w + EPS)
            out = centred * rstd[:, None] * gain + s["params"][:, at + w:at + 2 * w].double()[worker]
            return out, torch.stack((mean, rstd), 1)
        mean, rstd = s["stats"].double().unbind(1)
        hat = (x - mean[:, None]) * rstd[:, None]
        d = s["d"].double()
        h = d * gain
        dx = (h - (h.sum(1) / w)[:, None] - hat * ((h * hat).sum(1) / w)[:, None]) * rstd[:, None]
        both = torch.cat((d * hat, d), 1)
        grads = torch.stack([both[a:b].sum(0) for a, b in zip(ptr, ptr[1:])])
        return dx, grads
    k, m = c["n_in"], c["n_out"]
    if kind == "linear_weight":
        return torch.stack([torch.mm(s["x"][a:b].double().t().contiguous(), s["d"][a:b].double()).t().contiguous()
                            for a, b in zip(ptr, ptr[1:])]).view(n, m * k)
    out = []
    for i, (a, b) in enumerate(zip(ptr, ptr[1:])):
        weight = s["params"][i, at:at + m * k].to(_TYPE[c["act"]]).double().view(m, k)
        if kind == "linear":
            out.append(torch.mm(weight, s["x"][a:b].double().t().contiguous()).t())
        else:
            out.append(torch.mm(weight.t().contiguous(), s["d"][a:b].double().t().contiguous()).t())
    return torch.cat(out).contiguous()
