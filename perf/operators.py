"""Performance cases of the operators over ragged cluster rows, dropout and label scores, through the public binding.

Five kinds of pass:

  forward     gcpsl.group_forward: every cluster's rows through its own weights, y_r = W_g x_r + b_g, where asked with
              the ReLU and the dropout that follow it (rows sorted by cluster, of unequal counts, some of none);
  backward    gcpsl.group_input_grad and gcpsl.group_weight_grad: the gradients of that layer's input (through the ReLU
              and dropout that made it), weights and bias;
  dropout     gcpsl.dropout: y = x / (1 - p) where the counter-based draw of the element keeps it, else 0;
  score       gcpsl.score: each row's log probability of its label, entropy, log sum of exponentials and most likely
              classes;
  score_grad  gcpsl.score_grad: the logits' gradient, given those of the log probabilities and of the entropies.

`own` false runs the same in elementary torch operations in 32 bits.  The draw of element (r, j) of a [rows][cols]
tensor: the 64-bit word mix64(mix64(seed + tag) + (c + 1) golden), c = r ceil(cols / 4) + j / 4, holds four draws of 16
bits, element j takes bits 16 (j mod 4) on, and is kept if they are at least t = rint(65536 p); mix64 is SplitMix64's
finaliser.  Row counts of the clusters are a function of the case, everything else of the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_TAG, _GOLDEN = 0x44524F50, 0x9E3779B97F4A7C15
_MUL1, _MUL2 = 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


# ------------------------------------------------------------------- cases

def listed():
    return [
        # the classifier heads (128 features, 10 classes) of 8 clusters on about 64 examples each: a latency
        {"name": "head_f32", "do": "forward", "type": "f32", "groups": 8, "rows": 512, "k": 128, "n": 10,
         "split": "ragged", "p": 0.0, "relu": False},
        # serving: one row or so for each of 16 clusters' wide layers, all weights read for 16 rows
        {"name": "single_rows_bf16", "do": "forward", "type": "bf16", "groups": 16, "rows": 16, "k": 4096, "n": 4096,
         "split": "ragged", "p": 0.0, "relu": False},
        # a wide hidden layer over the whole pools of 16 clusters, with its ReLU and dropout: the largest
        {"name": "hidden_bf16", "do": "forward", "type": "bf16", "groups": 16, "rows": 32768, "k": 4096, "n": 4096,
         "split": "ragged", "p": 0.1, "relu": True},
        # the training step's other direction at half the rows
        {"name": "hidden_grad_bf16", "do": "backward", "type": "bf16", "groups": 16, "rows": 16384, "k": 4096,
         "n": 4096, "split": "ragged", "p": 0.1, "relu": True},
        # fp32, sizes that fill no tile, and a cluster without rows
        {"name": "odd_f32", "do": "forward", "type": "f32", "groups": 7, "rows": 5003, "k": 1001, "n": 777,
         "split": "empty", "p": 0.0, "relu": True},
        # fp32 training step of 8 clusters' middle-sized layers
        {"name": "mid_grad_f32", "do": "backward", "type": "f32", "groups": 8, "rows": 8192, "k": 1024, "n": 1024,
         "split": "ragged", "p": 0.25, "relu": True},
        # dropout of a hidden layer's activations, far past the caches
        {"name": "dropout_bf16", "do": "dropout", "type": "bf16", "rows": 32768, "cols": 4096, "p": 0.1},
        # a small one, rows of odd length
        {"name": "dropout_odd_f32", "do": "dropout", "type": "f32", "rows": 777, "cols": 1001, "p": 0.5},
        # evaluation of 16 clusters' batches of 128 over 10 classes, top 5
        {"name": "classes_f32", "do": "score", "type": "f32", "rows": 2048, "classes": 10, "top": 5, "masked": False},
        # serving: one row of many classes, an eighth of them ruled out, 20 alternatives
        {"name": "single_row_bf16", "do": "score", "type": "bf16", "rows": 1, "classes": 131072, "top": 20,
         "masked": True},
        # evaluation over many rows of many classes
        {"name": "vocabulary_bf16", "do": "score", "type": "bf16", "rows": 4096, "classes": 131072, "top": 8,
         "masked": False},
        # the gradient of an fp32 loss with an entropy term, an odd number of classes
        {"name": "vocabulary_grad_f32", "do": "score_grad", "type": "f32", "rows": 4096, "classes": 50021,
         "masked": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["forward", "forward", "backward", "dropout", "score", "score", "score_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if do in ("forward", "backward"):
        k, n = _log(rng, 64, 3000), _log(rng, 10, 3000)
        if rng.random() < 0.6:  # widths are more often multiples of 64 than not
            k, n = max(64, k // 64 * 64), max(64, n // 64 * 64)
        if rng.random() < 0.2:
            k, n = rng.choice([(4096, 1024), (1024, 4096), (4096, 4096)])
        rows = _log(rng, 16, 32768 if dtype == "bf16" and do == "forward" else 8192)
        return {"do": do, "type": dtype, "groups": min(_log(rng, 1, 64), rows), "rows": rows, "k": k, "n": n,
                "split": rng.choice(["ragged", "empty", "even"]),
                **rng.choice([{"p": 0.0, "relu": False}, {"p": 0.0, "relu": True}, {"p": 0.1, "relu": True},
                              {"p": 0.5, "relu": True}])}
    if do == "dropout":
        return {"do": do, "type": dtype, "rows": _log(rng, 16, 16384), "cols": _log(rng, 64, 8192),
                "p": rng.choice([0.05, 0.1, 0.25, 0.5])}
    classes = _log(rng, 10, 131072)
    case = {"do": do, "type": dtype, "rows": min(_log(rng, 1, 4096), max(1, 200_000_000 // classes)),
            "classes": classes, "masked": rng.random() < 0.5}
    return {**case, "top": rng.randint(0, 10)} if do == "score" else case


def _sizes(case):
    """Rows of each cluster: equal ones, unequal ones (a factor of about ten between the ends), or unequal ones of
    which about a quarter are zero."""
    g, rows = case["groups"], case["rows"]
    r = random.Random(g * 1_000_003 + rows)
    w = [1.0 if case["split"] == "even" else math.exp(r.uniform(-1.15, 1.15)) for _ in range(g)]
    if case["split"] == "empty":
        w = [0.0 if i % 4 == 1 else v for i, v in enumerate(w)]
    at = [0]
    for i in range(g):
        at.append(round(rows * sum(w[:i + 1]) / sum(w)))
    return [b - a for a, b in zip(at, at[1:])]


# ------------------------------------------------------------------ inputs

def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = _TYPES[case["type"]]
    s = dict(case, seed=(int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 64))
    if case["do"] in ("forward", "backward"):
        g, rows, k, n = case["groups"], case["rows"], case["k"], case["n"]
        s["sizes"] = _sizes(case)
        s["offsets"] = torch.tensor([sum(s["sizes"][:i]) for i in range(g + 1)], dtype=torch.int32, device="cuda")
        x = torch.randn((rows, k), generator=gen, device="cuda")
        if case["do"] == "backward" and case["relu"]:  # the layer's input is itself what a ReLU and a dropout left
            kept = torch.rand((rows, k), generator=gen, device="cuda") >= case["p"]
            x = torch.relu(x) * kept * _factor(case["p"])
        s["x"] = x.to(dtype)
        s["w"] = torch.stack([_normal(gen, (n, k), dtype, 1 / math.sqrt(k)) for _ in range(g)])
        s["b"] = _normal(gen, (g, n), torch.float32, 0.1)
        if case["do"] == "backward":
            s["dy"] = _normal(gen, (rows, n), dtype, 1 / max(1, rows // g))
    elif case["do"] == "dropout":
        s["x"] = _normal(gen, (case["rows"], case["cols"]), dtype)
    else:
        rows, classes = case["rows"], case["classes"]
        z = torch.randn((rows, classes), generator=gen, device="cuda") * 2.5
        s["labels"] = torch.randint(0, classes, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        if case["masked"]:  # classes that a constraint rules out, the label never among them
            out = torch.rand((rows, classes), generator=gen, device="cuda") < 0.125
            out[torch.arange(rows, device="cuda"), s["labels"].long()] = False
            z = z.masked_fill(out, -math.inf)
        s["z"] = z.to(dtype)
        if case["do"] == "score_grad":
            lse = torch.logsumexp(s["z"].double(), 1)
            logp = s["z"].double() - lse[:, None]
            p = logp.exp()
            s["lse"] = lse.float()
            s["entropy"] = -(p * torch.where(p > 0, logp, 0)).sum(1).float()
            s["g_logp"] = -torch.rand((rows,), generator=gen, device="cuda") / rows
            s["g_entropy"] = 0.01 * torch.randn((rows,), generator=gen, device="cuda") / rows
            del logp, p
    return s


# ------------------------------------------------- the plain form's parts

def _signed(v):
    return v - (1 << 64) if v >= 1 << 63 else v


def _mix64(z):
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(_MUL1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(_MUL2)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _factor(p):
    return 65536.0 / (65536 - round(65536 * p))


def _plain_dropout(x, p, seed):
    """x (fp32) with the elements that the draws drop at zero, the others scaled."""
    rows, cols = x.shape
    t = round(65536 * p)
    words = (cols + 3) // 4
    key = _mix64(torch.tensor(_signed((seed + _TAG) % (1 << 64)), device=x.device))
    z = _mix64(key + (torch.arange(rows * words, device=x.device) + 1) * _signed(_GOLDEN))
    drawn = (z.view(rows, words, 1) >> torch.tensor([0, 16, 32, 48], device=x.device)) & 0xFFFF
    kept = drawn.view(rows, 4 * words)[:, :cols] >= t
    return torch.where(kept, x * _factor(p), 0.0)


def _parts(sizes):
    ends = np.cumsum(sizes).tolist()
    return [(g, b - c, b) for g, (b, c) in enumerate(zip(ends, sizes))]


def _plain_forward(s):
    x, w, b = s["x"], s["w"], s["b"]
    y = torch.cat([x[i:j].float() @ w[g].float().T + b[g] for g, i, j in _parts(s["sizes"]) if j > i])
    y = torch.relu(y) if s["relu"] else y
    y = _plain_dropout(y, s["p"], s["seed"]) if s["p"] else y
    return y.to(x.dtype)


def _plain_backward(s):
    x, w, dy = s["x"], s["w"], s["dy"]
    parts = _parts(s["sizes"])
    dx = torch.cat([dy[i:j].float() @ w[g].float() for g, i, j in parts if j > i])
    dx = torch.where(x > 0, dx * _factor(s["p"]), 0.0) if s["relu"] else dx
    dw = torch.stack([dy[i:j].float().T @ x[i:j].float() for g, i, j in parts])
    db = torch.stack([dy[i:j].float().sum(0) for g, i, j in parts])
    return dx.to(x.dtype), dw, db


def _plain_score(s):
    z = s["z"].float()
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    logp = z - m - log_total
    p = e / total
    entropy = -(p * torch.where(p > 0, logp, 0.0)).sum(1)
    lse = (m + log_total).squeeze(1)
    given = logp.gather(1, s["labels"].long()[:, None]).squeeze(1)
    # one whole number per class that orders by value, then by the lower index
    bits = (z + 0.0).view(torch.int32).long()
    order = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) + torch.arange(z.shape[1] - 1, -1, -1, device=z.device)
    top = z.shape[1] - 1 - (order.topk(s["top"], 1).values & 0xFFFFFFFF)
    return given, entropy, lse, logp.gather(1, top), top.int()


def _plain_score_grad(s):
    z, at = s["z"].float(), s["labels"].long()[:, None]
    logp = z - s["lse"][:, None]
    p = torch.exp(logp)
    d = -s["g_logp"][:, None] * p
    d -= s["g_entropy"][:, None] * p * (torch.where(p > 0, logp, 0.0) + s["entropy"][:, None])
    d.scatter_add_(1, at, s["g_logp"][:, None])
    return d.to(s["z"].dtype)


_PLAIN = {"forward": _plain_forward, "backward": _plain_backward, "score": _plain_score,
          "score_grad": _plain_score_grad,
          "dropout": lambda s: _plain_dropout(s["x"].float(), s["p"], s["seed"]).to(s["x"].dtype)}


# --------------------------------------------------------------------- run

def _own(s):
    from paper_2609_29395_amd import gcpsl
    if s["do"] == "forward":
        return gcpsl.group_forward(s["x"], s["offsets"], s["w"], s["b"], relu=s["relu"], p=s["p"], seed=s["seed"])
    if s["do"] == "backward":
        dx = gcpsl.group_input_grad(s["dy"], s["offsets"], s["w"], gate=s["x"] if s["relu"] else None, p=s["p"])
        return (dx,) + tuple(gcpsl.group_weight_grad(s["dy"], s["x"], s["offsets"]))
    if s["do"] == "dropout":
        return gcpsl.dropout(s["x"], s["p"], s["seed"])
    if s["do"] == "score":
        r = gcpsl.score(s["z"], s["labels"], top=s["top"])
        return r.logp, r.entropy, r.lse, r.top_logp, r.top_class
    return gcpsl.score_grad(s["z"], s["labels"], s["lse"], s["entropy"], s["g_logp"], s["g_entropy"])


def run(state):
    return _own(state) if own else _PLAIN[state["do"]](state)


def work(case):
    e = 4 if case["type"] == "f32" else 2
    if case["do"] in ("forward", "backward"):
        rows, k, n, g = case["rows"], case["k"], case["n"], case["groups"]
        used = sum(c > 0 for c in _sizes(case))
        if case["do"] == "forward":
            return {"bytes": e * (rows * (k + n) + used * n * k) + 4 * used * n, "flops": 2 * rows * n * k}
        # dy and x read, dx written; weights read, their gradients and the bias's written in fp32
        return {"bytes": e * (rows * (2 * k + n) + used * n * k) + 4 * g * n * (k + 1), "flops": 4 * rows * n * k}
    if case["do"] == "dropout":
        return {"bytes": 2 * e * case["rows"] * case["cols"], "flops": 2 * case["rows"] * case["cols"]}
    rows, classes = case["rows"], case["classes"]
    if case["do"] == "score":
        return {"bytes": rows * (e * classes + 16 + 8 * case["top"]), "flops": 6 * rows * classes}
    return {"bytes": rows * (2 * e * classes + 20), "flops": 8 * rows * classes}


# ----------------------------------------------------- 64-bit definitions

def _kept64(rows, cols, p, seed):
    """Which elements the draws keep, with NumPy's unsigned 64-bit arithmetic."""
    def finish(v):
        v = (v ^ (v >> np.uint64(30))) * np.uint64(_MUL1)
        v = (v ^ (v >> np.uint64(27))) * np.uint64(_MUL2)
        return v ^ (v >> np.uint64(31))

    with np.errstate(over="ignore"):
        key = finish(np.array([(seed + _TAG) % (1 << 64)], dtype=np.uint64))
        words = -(-cols // 4)
        z = finish(key + np.arange(1, rows * words + 1, dtype=np.uint64) * np.uint64(_GOLDEN))
    draws = z.astype("<u8").view("<u2").reshape(rows, 4 * words)[:, :cols]
    return torch.from_numpy(draws >= round(65536 * p)).to("cuda")


def exact(case, seed):
    s = prepare(case, seed)
    if case["do"] == "dropout" or (case["do"] == "forward" and case["p"]):
        rows, cols = case["rows"], case["cols"] if case["do"] == "dropout" else case["n"]
        keep = _kept64(rows, cols, case["p"], s["seed"])
        factor = 1 / (1 - round(65536 * case["p"]) / 65536)
    if case["do"] == "dropout":
        return torch.where(keep, s["x"].double() * factor, 0.0)
    if case["do"] == "forward":
        out = torch.empty((case["rows"], case["n"]), dtype=torch.float64, device="cuda")
        i = 0
        for g, c in enumerate(s["sizes"]):
            if c:
                out[i:i + c] = torch.addmm(s["b"][g].double(), s["x"][i:i + c].double(), s["w"][g].double().t())
            i += c
        if case["relu"]:
            out.clamp_(min=0)
        return torch.where(keep, out * factor, 0.0) if case["p"] else out
    if case["do"] == "backward":
        dx = torch.empty((case["rows"], case["k"]), dtype=torch.float64, device="cuda")
        dw = torch.zeros((case["groups"], case["n"], case["k"]), dtype=torch.float64, device="cuda")
        db = torch.zeros((case["groups"], case["n"]), dtype=torch.float64, device="cuda")
        i = 0
        for g, c in enumerate(s["sizes"]):
            if c:
                d = s["dy"][i:i + c].double()
                torch.mm(d, s["w"][g].double(), out=dx[i:i + c])
                dw[g] = torch.mm(d.t(), s["x"][i:i + c].double())
                db[g] = d.sum(0)
            i += c
        if case["relu"]:
            dx = dx / (1 - round(65536 * case["p"]) / 65536) * (s["x"] > 0)
        return dx, dw, db
    rows, step = case["rows"], max(1, 50_000_000 // case["classes"])
    got = []
    for i in range(0, rows, step):
        z, y = s["z"][i:i + step].double(), s["labels"][i:i + step].long()
        r = torch.arange(z.shape[0], device="cuda")
        if case["do"] == "score":
            lse = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            ordered = torch.sort(z, dim=1, descending=True, stable=True)
            top = slice(0, case["top"])
            got.append((z[r, y] - lse, torch.special.entr(p).sum(1), lse, ordered.values[:, top] - lse[:, None],
                        ordered.indices[:, top].int()))
        else:
            lse, h = s["lse"][i:i + step].double()[:, None], s["entropy"][i:i + step].double()[:, None]
            gl, gh = s["g_logp"][i:i + step].double()[:, None], s["g_entropy"][i:i + step].double()[:, None]
            p = torch.exp(z - lse)
            d = gh * (torch.special.entr(p) - p * h) - gl * p
            d[r, y] += gl[:, 0]
            got.append((d,))
    out = tuple(torch.cat(v) for v in zip(*got))
    return out if case["do"] == "score" else out[0]
