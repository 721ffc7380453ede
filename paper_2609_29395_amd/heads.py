"""A head of its own for every cluster, trained and scored on all the cluster's examples at once.

A round of Alg. 2 draws the same number of examples from every cluster.  What follows a run has no such batch: the fused
model is scored, or fitted to each cluster's own distribution, on the n_n examples that cluster n holds, and the n_n
differ.  Here the split model is kept as it is; a layer with ReLU and dropout and a classifier are trained per cluster
on the pooled features of all its examples, the rows of all clusters one after another and every operator one launch
for all of them (gcpsl.group_forward, dropout, score and their gradients).

    python -m paper_2609_29395_amd.heads [--workload tiny_epoch] [--steps 60] [--dtype f32] [--blocks 2]

runs a workload, fuses it, and prints each cluster's loss, accuracy, top classes and entropy before and after.  With
--blocks, deeper heads follow (residual gated blocks), which learn from the labels and from the top classes that the
fused heads give each row: what the other clusters know reaches a cluster's own head without their examples.
PyTorch holds memory, casts the fp32 masters for bf16 products, and adds the SGD update.
"""
from __future__ import annotations

import argparse

import torch

from . import driver, gcpsl

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class ClusterHeads:
    """Heads of G clusters on k features: hidden units with ReLU and dropout, then L classes.

    Their parameters are one fp32 vector per cluster, [G][P]: weights and biases of the first layer, then of the
    second, as in the split model's own parameter vector, so that gcpsl.fuse_replicas (Eq. 5) applies to them too."""

    def __init__(self, G, k, hidden, L, dtype="f32", lr=0.1, momentum=0.9, p=0.1, p_input=0.05, seed=0):
        self.G, self.dtype, self.lr, self.momentum, self.p, self.p_input = G, DTYPES[dtype], lr, momentum, p, p_input
        self.seed, self.steps = int(seed), 0
        self.shapes = [(hidden, k), (hidden,), (L, hidden), (L,)]
        gen = torch.Generator().manual_seed(self.seed)
        one = torch.cat([(torch.rand(s, generator=gen) * 2 - 1).flatten() * (k if i < 2 else hidden) ** -0.5
                         for i, s in enumerate(self.shapes)])
        self.theta = one.cuda().repeat(G, 1).contiguous()  # every cluster starts alike
        self.mom = torch.zeros_like(self.theta)
        self.grad = torch.zeros_like(self.theta)

    def _views(self, flat):
        """[weights [G][hidden][k], biases, weights, biases] inside a [G][P] tensor."""
        out, at = [], 0
        for s in self.shapes:
            n = s[0] * (s[1] if len(s) == 2 else 1)
            out.append(flat[:, at:at + n].view(self.G, *s))
            at += n
        return out

    def _weights(self):
        w1, b1, w2, b2 = self._views(self.theta)
        return w1.to(self.dtype), b1, w2.to(self.dtype), b2

    def logits(self, x, offsets):
        """[rows][L] of the features x [rows][k], rows offsets[g] to offsets[g + 1] by cluster g's head."""
        w1, b1, w2, b2 = self._weights()
        return gcpsl.group_forward(gcpsl.group_forward(x, offsets, w1, b1, relu=True), offsets, w2, b2)

    def score(self, x, offsets, labels, top=1):
        """gcpsl.Scores of every row under its cluster's head."""
        return gcpsl.score(self.logits(x, offsets), labels, top=top)

    def step(self, x, offsets, labels, row_weight):
        """One SGD step of every cluster on the mean loss of its rows (row_weight [rows]: 1 / n_n); returns the rows'
        losses before it."""
        w1, b1, w2, b2 = self._weights()
        g1, gb1, g2, gb2 = self._views(self.grad)
        seed = (self.seed << 32) + 2 * self.steps  # a seed for each dropout of each step
        x = gcpsl.dropout(x, self.p_input, seed)
        h = gcpsl.group_forward(x, offsets, w1, b1, relu=True, p=self.p, seed=seed + 1)
        z = gcpsl.group_forward(h, offsets, w2, b2)
        s = gcpsl.score(z, labels)
        dz = gcpsl.score_grad(z, labels, s.lse, g_logp=-row_weight, out=z)
        gcpsl.group_weight_grad(dz, h, offsets, dw=g2, db=gb2)
        dh = gcpsl.group_input_grad(dz, offsets, w2, gate=h, p=self.p)
        gcpsl.group_weight_grad(dh, x, offsets, dw=g1, db=gb1)
        self.mom.mul_(self.momentum).add_(self.grad)
        self.theta.sub_(self.mom, alpha=self.lr)
        self.steps += 1
        return -s.logp

    def fuse(self, sizes):
        """Eq. 5 over the heads, by the clusters' example counts."""
        gcpsl.fuse_replicas(self.theta, sizes)


class BlockHeads:
    """Heads of G clusters on k features with residual gated blocks: a layer to d features, `depth` blocks

        h = norm(x);  v = W_2 (silu(g) u) + b_2, (g, u) = W_1 h + b_1;  q = W_q h + b_q
        x <- x + beta sigmoid(q) norm(v)

    each norm with weights of its own per cluster, and a classifier on the last norm.  One fp32 vector per cluster,
    [G][P], as for ClusterHeads."""

    def __init__(self, G, k, d, hidden, L, depth=2, dtype="f32", lr=0.1, momentum=0.9, beta=1.0, eps=1e-6, seed=0):
        self.G, self.depth, self.dtype, self.lr, self.momentum = G, depth, DTYPES[dtype], lr, momentum
        self.beta, self.eps = float(beta), eps
        self.shapes = {"w_in": (d, k), "b_in": (d,), "norm_in": (d,)}
        for i in range(depth):
            self.shapes.update({f"w1_{i}": (2 * hidden, d), f"b1_{i}": (2 * hidden,), f"w2_{i}": (d, hidden),
                                f"b2_{i}": (d,), f"wq_{i}": (d, d), f"bq_{i}": (d,), f"norm_block_{i}": (d,),
                                f"norm_next_{i}": (d,)})
        self.shapes.update(w_out=(L, d), b_out=(L,))
        gen = torch.Generator().manual_seed(int(seed))
        one = torch.cat([(torch.ones(s) if name.startswith("norm") else torch.zeros(s) if name.startswith("b") else
                          (torch.rand(s, generator=gen) * 2 - 1) * s[1] ** -0.5).flatten()
                         for name, s in self.shapes.items()])
        self.theta = one.cuda().repeat(G, 1).contiguous()  # every cluster starts alike
        self.mom = torch.zeros_like(self.theta)
        self.grad = torch.zeros_like(self.theta)

    def _views(self, flat):
        """{name: [G][..]} inside a [G][P] tensor."""
        out, at = {}, 0
        for name, s in self.shapes.items():
            n = s[0] * (s[1] if len(s) == 2 else 1)
            out[name] = flat[:, at:at + n].view(self.G, *s)
            at += n
        return out

    def _forward(self, x, offsets, keep):
        """(logits, what the backward pass needs)."""
        p = {name: v.to(self.dtype) if v.dim() == 3 else v for name, v in self._views(self.theta).items()}
        first = gcpsl.group_residual_norm(gcpsl.group_forward(x, offsets, p["w_in"], p["b_in"]), offsets,
                                          w_next=p["norm_in"], eps=self.eps)
        state, blocks = first, []
        for i in range(self.depth):
            h = state.h
            gated = gcpsl.group_gated_forward(h, offsets, p[f"w1_{i}"], p[f"b1_{i}"], keep=keep)
            v = gcpsl.group_forward(gated.y, offsets, p[f"w2_{i}"], p[f"b2_{i}"])
            q = gcpsl.group_forward(h, offsets, p[f"wq_{i}"], p[f"bq_{i}"])
            state = gcpsl.group_residual_norm(state.out, offsets, y=v, gate=q, w_block=p[f"norm_block_{i}"],
                                              w_next=p[f"norm_next_{i}"], beta=self.beta, eps=self.eps)
            blocks.append((h, gated, v, q, state) if keep else None)
        return gcpsl.group_forward(state.h, offsets, p["w_out"], p["b_out"]), (p, first, blocks, state)

    def logits(self, x, offsets):
        return self._forward(x, offsets, False)[0]

    def score(self, x, offsets, labels, top=1):
        return gcpsl.score(self.logits(x, offsets), labels, top=top)

    def _layer_grads(self, g, w, b, dy, x, offsets):
        gcpsl.group_weight_grad(dy, x, offsets, dw=g[w], db=g[b])

    def gradients(self, x, offsets, labels, row_weight, teacher=None, temperature=2.0, share=0.5):
        """Fills self.grad with the gradient of every cluster's mean loss (row_weight [rows]: 1 / n_n); returns the
        rows' losses.  teacher: (top classes, their values) [rows][K], as score gives them; the loss is then (1 - share)
        of the labels' and share of T^2 times the divergence from the teacher at temperature T."""
        z, (p, first, blocks, state) = self._forward(x, offsets, True)
        g = self._views(self.grad)
        if teacher is None:
            s = gcpsl.score(z, labels)
            loss = -s.logp
            dz = gcpsl.score_grad(z, labels, s.lse, g_logp=-row_weight, out=z)
        else:
            weight = share * temperature ** 2
            s = gcpsl.distill(z, *teacher, temperature=temperature, labels=labels)
            loss = weight * s.kl - (1 - share) * s.logp
            dz = gcpsl.distill_grad(z, *teacher, s.lse_t, temperature=temperature, labels=labels, lse=s.lse,
                                    g_kl=weight * row_weight, g_logp=(share - 1) * row_weight, out=z)
        self._layer_grads(g, "w_out", "b_out", dz, state.h, offsets)
        g_out, g_h = None, gcpsl.group_input_grad(dz, offsets, p["w_out"])
        for i in reversed(range(self.depth)):
            h, gated, v, q, r = blocks[i]
            d = gcpsl.group_residual_norm_grad(r.out, offsets, g_out=g_out, g_h=g_h, y=v, gate=q,
                                               w_block=p[f"norm_block_{i}"], w_next=p[f"norm_next_{i}"],
                                               r_block=r.r_block, r_next=r.r_next, beta=self.beta)
            g[f"norm_block_{i}"].copy_(d.dw_block)
            g[f"norm_next_{i}"].copy_(d.dw_next)
            self._layer_grads(g, f"w2_{i}", f"b2_{i}", d.dy, gated.y, offsets)
            dpre = gcpsl.group_gated_grad(d.dy, offsets, p[f"w2_{i}"], gated.pre)
            self._layer_grads(g, f"w1_{i}", f"b1_{i}", dpre, h, offsets)
            self._layer_grads(g, f"wq_{i}", f"bq_{i}", d.dgate, h, offsets)
            g_out = d.dx
            g_h = gcpsl.group_input_grad(dpre, offsets, p[f"w1_{i}"])
            g_h += gcpsl.group_input_grad(d.dgate, offsets, p[f"wq_{i}"])
        d = gcpsl.group_residual_norm_grad(first.out, offsets, g_out=g_out, g_h=g_h, w_next=p["norm_in"],
                                           r_next=first.r_next)
        g["norm_in"].copy_(d.dw_next)
        self._layer_grads(g, "w_in", "b_in", d.dx, x, offsets)
        return loss

    def step(self, x, offsets, labels, row_weight, **distillation):
        """One SGD step of every cluster; returns the rows' losses before it."""
        loss = self.gradients(x, offsets, labels, row_weight, **distillation)
        self.mom.mul_(self.momentum).add_(self.grad)
        self.theta.sub_(self.mom, alpha=self.lr)
        return loss

    def fuse(self, sizes):
        """Eq. 5 over the heads, by the clusters' example counts."""
        gcpsl.fuse_replicas(self.theta, sizes)


def cluster_features(ctx):
    """(x [rows][channels], labels [rows], offsets [C + 1], sizes [C]) of one epoch of every cluster: the pooled features
    that the split model gives each example, rows sorted by cluster.  The context runs its rounds, so one with lr 0 is
    meant; an epoch has floor(n_n / B) B of a cluster's n_n examples."""
    C, B, layers = ctx.cfg["C"], ctx.cfg["B"], ctx.cfg["layers"]
    rounds, R = ctx.epoch_rounds()
    rows, labels = [[] for _ in range(C)], [[] for _ in range(C)]
    for s in range(R):
        ctx.sample(s)
        ctx.step(s)
        f = ctx.tensor(f"act{len(layers) - 2}").view(C, B, layers[-1][1])
        y = ctx.tensor("y")[:C * B].view(C, B)
        for n in range(C):
            if s < rounds[n]:
                rows[n].append(f[n].clone())
                labels[n].append(y[n].clone())
    sizes = [B * int(r) for r in rounds]
    offsets = torch.tensor([sum(sizes[:n]) for n in range(C + 1)], dtype=torch.int32, device="cuda")
    return torch.cat(sum(rows, [])).contiguous(), torch.cat(sum(labels, [])), offsets, sizes


def by_cluster(values, sizes):
    return [float(v.double().mean()) for v in values.split(sizes)]


def main(argv=None):
    from gcpsl_inputs import get_config
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", default="tiny_epoch")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--hidden", type=int, default=64)
    ap.add_argument("--dtype", choices=sorted(DTYPES), default="f32")
    ap.add_argument("--blocks", type=int, default=0, help="residual gated blocks of heads taught by the fused ones")
    a = ap.parse_args(argv)
    cfg = get_config(a.workload, schedule="epoch")
    ctx, _ = driver.setup(cfg)
    driver.train(ctx, cfg["T"])
    ctx.fuse()
    frozen, _ = driver.setup(dict(cfg, lr=0.0, momentum=0.0, weight_decay=0.0))
    frozen.theta.copy_(ctx.theta)
    if ctx.S:
        frozen.norm_state.copy_(ctx.norm_state)
    x, labels, offsets, sizes = cluster_features(frozen)
    x = x.to(DTYPES[a.dtype])
    weight = torch.cat([torch.full((n,), 1.0 / n) for n in sizes]).cuda()
    heads = ClusterHeads(cfg["C"], x.shape[1], a.hidden, cfg["L"], dtype=a.dtype, seed=cfg["seed"])
    top = min(3, cfg["L"])

    def report(what, of=heads):
        s = of.score(x, offsets, labels, top=top)
        loss, entropy = by_cluster(-s.logp, sizes), by_cluster(s.entropy, sizes)
        right = s.top_class == labels[:, None]
        first, among = by_cluster(right[:, 0], sizes), by_cluster(right.any(1), sizes)
        for n, rows in enumerate(sizes):
            print(f"{what}: cluster {n}, {rows} examples: loss {loss[n]:.4f}, accuracy {first[n]:.3f}, "
                  f"among the top {top} {among[n]:.3f}, entropy {entropy[n]:.3f}", flush=True)
        return loss, first

    before = report("before")
    for _ in range(a.steps):
        heads.step(x, offsets, labels, weight)
    after = report("after")
    heads.fuse(sizes)
    report("heads fused")
    if a.blocks:
        best = heads.score(x, offsets, labels, top=top)
        deep = BlockHeads(cfg["C"], x.shape[1], a.hidden, a.hidden, cfg["L"], depth=a.blocks, dtype=a.dtype,
                          seed=cfg["seed"])
        for _ in range(a.steps):
            deep.step(x, offsets, labels, weight, teacher=(best.top_class, best.top_logp))
        report("blocks taught", deep)
    return before, after


if __name__ == "__main__":
    main()
