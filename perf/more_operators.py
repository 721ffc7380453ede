"""Performance cases of gated layers, residual norms and distillation, through the public binding.

Six kinds of pass, two for each of three operators:

  gated          gcpsl.group_gated_forward: every cluster's rows through its own gated layer, (g, u) = W_g x_r + b_g,
                 y = f(g) u, f one of silu, gelu (with the normal distribution's own Phi) and relu; in training with
                 the pair (g | u) kept;
  gated_grad     gcpsl.group_gated_grad: dh = V_g^T dy_r through the layer after it, and from that the gradients
                 (f'(g) u dh | f(g) dh) of the pair;
  norm           gcpsl.group_residual_norm: x' = alpha x + beta sigmoid(gate) (w1_g y / rms(y)), h = w2_g x' / rms(x'),
                 rms(v) = sqrt(mean v^2 + eps), and both reciprocal rms of every row;
  norm_grad      gcpsl.group_residual_norm_grad: from the gradients of x' and h those of x, y, gate and both weights;
  distill        gcpsl.distill: the divergence sum_k q_k (log q_k - log p_k) of a student's classes p = softmax(z / T)
                 from a teacher's K best ones, q = softmax(v / T), beside the labels' log probabilities at T = 1;
  distill_grad   gcpsl.distill_grad: the logits' gradient, given those of the divergences and log probabilities.

`own` false runs the same in elementary torch operations in 32 bits.  Row counts of the clusters are a function of the
case, everything else of the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS, _ALPHA, _BETA = 1e-5, 1.0, 0.5


# ------------------------------------------------------------------- cases

def listed():
    return [
        # a wide gated layer over the pools of 16 clusters in training, its pair kept: the largest
        {"name": "gated_train_bf16", "do": "gated", "type": "bf16", "groups": 16, "rows": 16384, "k": 4096, "n": 4096,
         "split": "ragged", "act": "silu", "keep": True},
        # serving: one row or so for each of 16 clusters, all weights read for 16 rows
        {"name": "gated_single_rows_bf16", "do": "gated", "type": "bf16", "groups": 16, "rows": 16, "k": 4096,
         "n": 4096, "split": "ragged", "act": "silu", "keep": False},
        # fp32, sizes that fill no tile, clusters without rows
        {"name": "gated_odd_f32", "do": "gated", "type": "f32", "groups": 7, "rows": 3001, "k": 501, "n": 333,
         "split": "empty", "act": "gelu", "keep": True},
        # the backward pass of the largest, through the layer after it
        {"name": "gated_grad_bf16", "do": "gated_grad", "type": "bf16", "groups": 16, "rows": 16384, "m": 4096,
         "n": 4096, "split": "ragged", "act": "silu"},
        # fp32 training of 8 clusters' middle-sized layers
        {"name": "gated_grad_f32", "do": "gated_grad", "type": "f32", "groups": 8, "rows": 8192, "m": 1024, "n": 1024,
         "split": "ragged", "act": "silu"},
        # the residual stream of the wide blocks, far past the caches
        {"name": "norm_bf16", "do": "norm", "type": "bf16", "groups": 16, "rows": 32768, "n": 4096, "split": "ragged"},
        # serving: a row for each cluster
        {"name": "norm_single_rows_f32", "do": "norm", "type": "f32", "groups": 16, "rows": 16, "n": 4096,
         "split": "even"},
        # the wide blocks' backward pass
        {"name": "norm_grad_bf16", "do": "norm_grad", "type": "bf16", "groups": 16, "rows": 16384, "n": 4096,
         "split": "ragged"},
        # small odd rows, clusters without rows
        {"name": "norm_grad_odd_f32", "do": "norm_grad", "type": "f32", "groups": 7, "rows": 777, "n": 1001,
         "split": "empty"},
        # batches of 16 clusters over 10 classes, the teacher's 5 best
        {"name": "distill_classes_f32", "do": "distill", "type": "f32", "rows": 2048, "classes": 10, "top": 5,
         "temperature": 2.0, "labels": True, "masked": False},
        # many rows of many classes, softened
        {"name": "distill_vocabulary_bf16", "do": "distill", "type": "bf16", "rows": 4096, "classes": 131072, "top": 20,
         "temperature": 2.0, "labels": True, "masked": False},
        # their gradient, an odd number of classes
        {"name": "distill_grad_vocabulary_bf16", "do": "distill_grad", "type": "bf16", "rows": 4096, "classes": 50021,
         "top": 20, "temperature": 2.0, "labels": True, "masked": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["gated", "gated", "gated_grad", "norm", "norm_grad", "distill", "distill_grad"])
    dtype = rng.choice(["f32", "bf16"])
    split = rng.choice(["ragged", "empty", "even"])
    act = rng.choice(["silu", "silu", "gelu", "relu"])
    if do in ("gated", "gated_grad"):
        k, n = _log(rng, 64, 2500), _log(rng, 16, 2500)
        if rng.random() < 0.6:  # widths are more often multiples of 64 than not
            k, n = max(64, k // 64 * 64), max(64, n // 64 * 64)
        if rng.random() < 0.2:
            k, n = rng.choice([(4096, 1024), (1024, 4096), (4096, 4096)])
        rows = _log(rng, 1, 16384 if dtype == "bf16" else 4096)
        case = {"do": do, "type": dtype, "groups": min(_log(rng, 1, 32), rows), "rows": rows}
        if do == "gated":
            return {**case, "k": k, "n": n, "split": split, "act": act, "keep": rng.random() < 0.5}
        return {**case, "m": k, "n": n, "split": split, "act": act}
    if do in ("norm", "norm_grad"):
        rows = _log(rng, 1, 16384)
        return {"do": do, "type": dtype, "groups": min(_log(rng, 1, 32), rows), "rows": rows, "n": _log(rng, 64, 8192),
                "split": split}
    classes = _log(rng, 10, 131072)
    return {"do": do, "type": dtype, "rows": min(_log(rng, 1, 4096), max(1, 200_000_000 // classes)),
            "classes": classes, "top": min(classes, _log(rng, 1, 64)), "temperature": rng.choice([1.0, 1.5, 2.0, 4.0]),
            "labels": rng.random() < 0.6, "masked": rng.random() < 0.5}


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


def _rms_of(v):
    """Reciprocal rms of the rows, as the forward pass leaves it."""
    return torch.rsqrt(v.double().pow(2).mean(1) + _EPS).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = _TYPES[case["type"]]
    s = dict(case)
    if "groups" in case:
        s["sizes"] = _sizes(case)
        s["offsets"] = torch.tensor([sum(s["sizes"][:i]) for i in range(case["groups"] + 1)], dtype=torch.int32,
                                    device="cuda")
        g, rows, n = case["groups"], case["rows"], case["n"]
    if case["do"] == "gated":
        k = case["k"]
        s["x"] = _normal(gen, (rows, k), dtype)
        s["w"] = torch.stack([_normal(gen, (2 * n, k), dtype, 1 / math.sqrt(k)) for _ in range(g)])
        s["b"] = _normal(gen, (g, 2 * n), torch.float32, 0.1)
    elif case["do"] == "gated_grad":
        m = case["m"]
        s["dy"] = _normal(gen, (rows, m), dtype, 1 / max(1, rows // g))
        s["w"] = torch.stack([_normal(gen, (m, n), dtype, 1 / math.sqrt(n)) for _ in range(g)])
        s["pre"] = _normal(gen, (rows, 2 * n), dtype)
    elif case["do"] in ("norm", "norm_grad"):
        s["y"], s["gate"] = _normal(gen, (rows, n), dtype, 2.0), _normal(gen, (rows, n), dtype)
        s["w_block"] = 1 + _normal(gen, (g, n), torch.float32, 0.1)
        s["w_next"] = 1 + _normal(gen, (g, n), torch.float32, 0.1)
        s["x"] = _normal(gen, (rows, n), dtype, 3.0)  # in the backward pass the updated one
        if case["do"] == "norm_grad":
            s["dx"] = _normal(gen, (rows, n), dtype, 1 / max(1, rows // g))
            s["dh"] = _normal(gen, (rows, n), dtype, 1 / max(1, rows // g))
            s["r_block"], s["r_next"] = _rms_of(s["y"]), _rms_of(s["x"])
    else:
        rows, classes, top = case["rows"], case["classes"], case["top"]
        z = torch.randn((rows, classes), generator=gen, device="cuda") * 2.5
        best = (z + torch.randn((rows, classes), generator=gen, device="cuda")).topk(top, 1)  # a teacher that half agrees
        s["t_value"], s["t_class"] = best.values.contiguous(), best.indices.int().contiguous()
        del best
        s["y"] = None
        if case["labels"]:
            s["y"] = torch.randint(0, classes, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        if case["masked"]:  # classes that a constraint rules out, the label and the teacher's never among them
            out = torch.rand((rows, classes), generator=gen, device="cuda") < 0.125
            out.scatter_(1, s["t_class"].long(), False)
            if case["labels"]:
                out.scatter_(1, s["y"].long()[:, None], False)
            z = z.masked_fill_(out, -math.inf)
        s["z"] = z.to(dtype)
        del z
        if case["do"] == "distill_grad":
            step = max(1, 50_000_000 // classes)
            parts = [s["z"][i:i + step].double() for i in range(0, rows, step)]
            s["lse_t"] = torch.cat([torch.logsumexp(p / case["temperature"], 1) for p in parts]).float()
            s["lse"] = torch.cat([torch.logsumexp(p, 1) for p in parts]).float()
            s["g_kl"] = torch.rand((rows,), generator=gen, device="cuda") * case["temperature"] ** 2 / rows
            s["g_logp"] = -torch.rand((rows,), generator=gen, device="cuda") / rows if case["labels"] else None
    return s


# ------------------------------------------------- the plain form's parts

def _parts(sizes):
    at = 0
    for g, c in enumerate(sizes):
        if c:
            yield g, at, at + c
        at += c


def _act(g, name):
    if name == "silu":
        return g / (1 + torch.exp(-g))
    if name == "gelu":
        return 0.5 * g * torch.special.erfc(-g * math.sqrt(0.5))
    return torch.where(g > 0, g, 0.0)


def _act_grad(g, name):
    if name == "silu":
        e = 1 / (1 + torch.exp(-g))
        return e * (1 + g * (1 - e))
    if name == "gelu":
        return 0.5 * torch.special.erfc(-g * math.sqrt(0.5)) + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    return torch.where(g > 0, 1.0, 0.0)


def _plain_gated(s):
    x, n = s["x"], s["n"]
    pre = torch.cat([x[i:j].float() @ s["w"][g].float().T + s["b"][g] for g, i, j in _parts(s["sizes"])])
    y = _act(pre[:, :n], s["act"]) * pre[:, n:]
    return (y.to(x.dtype), pre.to(x.dtype)) if s["keep"] else y.to(x.dtype)


def _plain_gated_grad(s):
    n, dy = s["n"], s["dy"]
    dh = torch.cat([dy[i:j].float() @ s["w"][g].float() for g, i, j in _parts(s["sizes"])])
    g, u = s["pre"][:, :n].float(), s["pre"][:, n:].float()
    return torch.cat((_act_grad(g, s["act"]) * u * dh, _act(g, s["act"]) * dh), 1).to(dy.dtype)


def _by_row(s, w):
    return torch.repeat_interleave(w, torch.diff(s["offsets"]).long(), 0)


def _plain_norm(s):
    dtype = s["x"].dtype
    x, y = s["x"].float(), s["y"].float()
    r1 = 1 / torch.sqrt((y * y).mean(1) + _EPS)
    t = _by_row(s, s["w_block"]) * (y * r1[:, None])
    new = _ALPHA * x + _BETA * t / (1 + torch.exp(-s["gate"].float()))
    r2 = 1 / torch.sqrt((new * new).mean(1) + _EPS)
    h = _by_row(s, s["w_next"]) * (new * r2[:, None])
    return new.to(dtype), h.to(dtype), r1, r2


def _plain_norm_grad(s):
    dtype = s["x"].dtype
    r1, r2 = s["r_block"][:, None], s["r_next"][:, None]
    n1, n2, dh = s["y"].float() * r1, s["x"].float() * r2, s["dh"].float()
    a = _by_row(s, s["w_next"]) * dh
    d = s["dx"].float() + r2 * (a - n2 * (a * n2).mean(1, keepdim=True))
    sig, w1 = 1 / (1 + torch.exp(-s["gate"].float())), _by_row(s, s["w_block"])
    e = _BETA * d * sig
    c = e * w1
    dy = r1 * (c - n1 * (c * n1).mean(1, keepdim=True))
    dw1, dw2 = torch.zeros_like(s["w_block"]), torch.zeros_like(s["w_next"])
    for g, i, j in _parts(s["sizes"]):
        dw1[g], dw2[g] = (e[i:j] * n1[i:j]).sum(0), (dh[i:j] * n2[i:j]).sum(0)
    return (_ALPHA * d).to(dtype), dy.to(dtype), (c * n1 * (1 - sig)).to(dtype), dw1, dw2


def _log_softmax(v):
    v = v - v.amax(1, keepdim=True)
    return v - torch.log(torch.exp(v).sum(1, keepdim=True))


def _plain_distill(s):
    z, temp = s["z"].float(), s["temperature"]
    m = z.amax(1, keepdim=True)
    d = z - m
    log_t = torch.log(torch.exp(d / temp).sum(1, keepdim=True))
    lq = _log_softmax(s["t_value"] / temp)
    kl = (torch.exp(lq) * (lq - (d.gather(1, s["t_class"].long()) / temp - log_t))).sum(1)
    out = (kl, (m / temp + log_t)[:, 0])
    if s["labels"]:
        log_1 = torch.log(torch.exp(d).sum(1, keepdim=True))
        out += ((d.gather(1, s["y"].long()[:, None]) - log_1)[:, 0], (m + log_1)[:, 0])
    return out


def _plain_distill_grad(s):
    z, temp = s["z"].float(), s["temperature"]
    gk = (s["g_kl"] / temp)[:, None]
    d = gk * torch.exp(z / temp - s["lse_t"][:, None])
    d.scatter_add_(1, s["t_class"].long(), -gk * torch.exp(_log_softmax(s["t_value"] / temp)))
    if s["labels"]:
        gl = s["g_logp"][:, None]
        d -= gl * torch.exp(z - s["lse"][:, None])
        d.scatter_add_(1, s["y"].long()[:, None], gl)
    return d.to(s["z"].dtype)


_PLAIN = {"gated": _plain_gated, "gated_grad": _plain_gated_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
          "distill": _plain_distill, "distill_grad": _plain_distill_grad}


# --------------------------------------------------------------------- run

def _own(s):
    from paper_2609_29395_amd import gcpsl
    if s["do"] == "gated":
        r = gcpsl.group_gated_forward(s["x"], s["offsets"], s["w"], s["b"], act=s["act"], keep=s["keep"])
        return (r.y, r.pre) if s["keep"] else r.y
    if s["do"] == "gated_grad":
        return gcpsl.group_gated_grad(s["dy"], s["offsets"], s["w"], s["pre"], act=s["act"])
    if s["do"] == "norm":
        return tuple(gcpsl.group_residual_norm(s["x"], s["offsets"], y=s["y"], gate=s["gate"], w_block=s["w_block"],
                                               w_next=s["w_next"], alpha=_ALPHA, beta=_BETA, eps=_EPS))
    if s["do"] == "norm_grad":
        return tuple(gcpsl.group_residual_norm_grad(
            s["x"], s["offsets"], g_out=s["dx"], g_h=s["dh"], y=s["y"], gate=s["gate"], w_block=s["w_block"],
            w_next=s["w_next"], r_block=s["r_block"], r_next=s["r_next"], alpha=_ALPHA, beta=_BETA))
    if s["do"] == "distill":
        r = gcpsl.distill(s["z"], s["t_class"], s["t_value"], temperature=s["temperature"], labels=s["y"])
        return (r.kl, r.lse_t, r.logp, r.lse) if s["labels"] else (r.kl, r.lse_t)
    return gcpsl.distill_grad(s["z"], s["t_class"], s["t_value"], s["lse_t"], temperature=s["temperature"],
                              labels=s["y"], lse=s["lse"] if s["labels"] else None, g_kl=s["g_kl"], g_logp=s["g_logp"])


def run(state):
    return _own(state) if own else _PLAIN[state["do"]](state)


def work(case):
    e, rows = 4 if case["type"] == "f32" else 2, case["rows"]
    if "groups" in case:
        used, n = sum(c > 0 for c in _sizes(case)), case["n"]
    if case["do"] == "gated":
        out = 3 * n if case["keep"] else n
        return {"bytes": e * (rows * (case["k"] + out) + used * 2 * n * case["k"]) + 8 * used * n,
                "flops": 4 * rows * n * case["k"]}
    if case["do"] == "gated_grad":
        return {"bytes": e * (rows * (case["m"] + 4 * n) + used * n * case["m"]), "flops": 2 * rows * n * case["m"]}
    if case["do"] == "norm":
        return {"bytes": 5 * e * rows * n + 8 * rows + 8 * used * n, "flops": 14 * rows * n}
    if case["do"] == "norm_grad":
        return {"bytes": 8 * e * rows * n + 8 * rows + 8 * (used + case["groups"]) * n, "flops": 30 * rows * n}
    classes, labels = case["classes"], 3 if case["labels"] else 0
    if case["do"] == "distill":
        return {"bytes": rows * (e * classes + 8 * case["top"] + 8 + 4 * labels), "flops": (6 + labels) * rows * classes}
    return {"bytes": rows * (2 * e * classes + 8 * case["top"] + 8 + 4 * labels), "flops": (5 + labels) * rows * classes}


# ----------------------------------------------------- 64-bit definitions

def _phi(g):
    return torch.erfc(g / -math.sqrt(2)) / 2  # (special.ndtr takes 1 + erf, which loses the lower tail)


def _exact_act(g, name):
    """f and its derivative."""
    if name == "silu":
        e = torch.sigmoid(g)
        return g * e, e + g * e * torch.sigmoid(-g)
    if name == "gelu":
        return g * _phi(g), _phi(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g.clamp(min=0), (g > 0).double()


def exact(case, seed):
    s = prepare(case, seed)
    rows, n = case["rows"], case.get("n")
    f64 = {"dtype": torch.float64, "device": "cuda"}
    if case["do"] == "gated":
        y, pre = torch.empty((rows, n), **f64), torch.empty((rows, 2 * n), **f64)
        for g, i, j in _parts(s["sizes"]):
            pre[i:j] = torch.addmm(s["b"][g].double(), s["x"][i:j].double(), s["w"][g].double().t())
            y[i:j] = _exact_act(pre[i:j, :n], case["act"])[0] * pre[i:j, n:]
        return (y, pre) if case["keep"] else y
    if case["do"] == "gated_grad":
        out = torch.empty((rows, 2 * n), **f64)
        for g, i, j in _parts(s["sizes"]):
            dh = torch.mm(s["dy"][i:j].double(), s["w"][g].double())
            f, d = _exact_act(s["pre"][i:j, :n].double(), case["act"])
            out[i:j, :n], out[i:j, n:] = d * s["pre"][i:j, n:].double() * dh, f * dh
        return out
    if case["do"] == "norm":
        new, h, r1, r2 = torch.empty((rows, n), **f64), torch.empty((rows, n), **f64), [], []
        for g, i, j in _parts(s["sizes"]):
            y = s["y"][i:j].double()
            r1.append((y.pow(2).sum(1) / n + _EPS) ** -0.5)
            y = torch.einsum("rn,n,r->rn", y, s["w_block"][g].double(), r1[-1])
            new[i:j] = s["x"][i:j].double() * _ALPHA + y * torch.sigmoid(s["gate"][i:j].double()) * _BETA
            r2.append((new[i:j].pow(2).sum(1) / n + _EPS) ** -0.5)
            h[i:j] = torch.einsum("rn,n,r->rn", new[i:j], s["w_next"][g].double(), r2[-1])
        return new, h, torch.cat(r1), torch.cat(r2)
    if case["do"] == "norm_grad":
        out = [torch.empty((rows, n), **f64) for _ in range(3)]
        dw1, dw2 = torch.zeros((case["groups"], n), **f64), torch.zeros((case["groups"], n), **f64)
        for g, i, j in _parts(s["sizes"]):
            x, y, dh = s["x"][i:j].double(), s["y"][i:j].double(), s["dh"][i:j].double()
            sig = torch.sigmoid(s["gate"][i:j].double())
            w1, w2 = s["w_block"][g].double(), s["w_next"][g].double()
            r1, r2 = s["r_block"][i:j].double()[:, None], s["r_next"][i:j].double()[:, None]
            d = s["dx"][i:j].double() + r2 * w2 * dh - x * r2 ** 3 * ((w2 * dh * x).sum(1, keepdim=True) / n)
            d_out = _BETA * d  # of sigmoid(gate) * t
            out[0][i:j] = _ALPHA * d
            out[2][i:j] = d_out * w1 * y * r1 * sig * (1 - sig)
            d_norm = d_out * sig  # of t
            dw1[g], dw2[g] = (d_norm * y * r1).sum(0), (dh * x * r2).sum(0)
            v = d_norm * w1
            out[1][i:j] = r1 * v - y * r1 ** 3 * ((v * y).sum(1, keepdim=True) / n)
        return (*out, dw1, dw2)
    temp, step, got = case["temperature"], max(1, 50_000_000 // case["classes"]), []
    for i in range(0, rows, step):
        z, c = s["z"][i:i + step].double(), s["t_class"][i:i + step].long()
        lq = torch.log_softmax(s["t_value"][i:i + step].double() / temp, 1)
        y = s["y"][i:i + step].long()[:, None] if case["labels"] else None
        if case["do"] == "distill":
            lse_t, lse = torch.logsumexp(z / temp, 1), torch.logsumexp(z, 1)
            kl = (lq.exp() * (lq - z.gather(1, c) / temp + lse_t[:, None])).sum(1)
            got.append((kl, lse_t) + ((z.gather(1, y)[:, 0] - lse, lse) if case["labels"] else ()))
        else:
            gk = s["g_kl"][i:i + step].double()[:, None] / temp
            d = torch.exp(z / temp - s["lse_t"][i:i + step].double()[:, None]) * gk
            d = d.scatter_add(1, c, -lq.exp() * gk)
            if case["labels"]:
                gl = s["g_logp"][i:i + step].double()[:, None]
                d = d - gl * torch.exp(z - s["lse"][i:i + step].double()[:, None])
                d = d.scatter_add(1, y, gl)
            got.append((d,))
    out = tuple(torch.cat(v) for v in zip(*got))
    return out if case["do"] == "distill" else out[0]
