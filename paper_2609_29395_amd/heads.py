"""A head of its own for every cluster, trained and scored on all the cluster's examples at once.

A round of Alg. 2 draws the same number of examples from every cluster.  What follows a run has no such batch: the fused
model is scored, or fitted to each cluster's own distribution, on the n_n examples that cluster n holds, and the n_n
differ.  Here the split model is kept as it is; a layer with ReLU and dropout and a classifier are trained per cluster
on the pooled features of all its examples, the rows of all clusters one after another and every operator one launch
for all of them (gcpsl.group_forward, dropout, score and their gradients).

    python -m paper_2609_29395_amd.heads [--workload tiny_epoch] [--steps 60] [--dtype f32]

runs a workload, fuses it, and prints each cluster's loss, accuracy, top classes and entropy before and after.
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

    def report(what):
        s = heads.score(x, offsets, labels, top=top)
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
    return before, after


if __name__ == "__main__":
    main()
