"""The clusters' heads (heads.py): a chain of every operator on tensors, against the same training in 64 bits under the
same draws, and the command on a workload."""
import numpy as np
import pytest
import torch

import ops_plain as plain

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import heads  # noqa: E402


def plain_step(theta, mom, shapes, x, offsets, labels, weight, lr, momentum, p, p_input, seed, steps):
    """One step in 64 bits; returns the rows' losses."""
    G = theta.shape[0]
    v, at = [], 0
    for s in shapes:
        n = int(np.prod(s))
        v.append(theta[:, at:at + n].view(G, *s))
        at += n
    w1, b1, w2, b2 = v
    seed = (seed << 32) + 2 * steps
    x = torch.where(plain.kept(*x.shape, p_input, seed), x * plain.factor(p_input), 0.0)
    h = plain.forward(x, offsets, w1, b1, True, p, seed + 1)[0]
    z = plain.forward(h, offsets, w2, b2)[0]
    logp, _, lse, _, _ = plain.score(z, labels, 1)
    dz = plain.score_grad(z, labels, lse, None, -weight, None)
    dw2, db2, _, _ = plain.weight_grad(dz, h, offsets)
    dh = plain.input_grad(dz, offsets, w2, h, p)[0]
    dw1, db1, _, _ = plain.weight_grad(dh, x, offsets)
    grad = torch.cat([t.reshape(G, -1) for t in (dw1, db1, dw2, db2)], 1)
    mom.mul_(momentum).add_(grad)
    theta.sub_(mom, alpha=lr)
    return -logp


# relative bars of a training run, as everywhere in this suite: 1e-4 in fp32, 2e-2 in bf16 (2-norm per cluster)
@pytest.mark.parametrize("dtype,bar", [("f32", 1e-4), ("bf16", 2e-2)])
@pytest.mark.parametrize("counts,k,hidden,L", [([40, 0, 75, 13], 36, 24, 7), ([130, 64], 64, 128, 10)])
def test_training_matches_64_bits(counts, k, hidden, L, dtype, bar):
    offsets = [int(v) for v in np.cumsum([0] + counts)]
    rows, G, steps = offsets[-1], len(counts), 6
    gen = torch.Generator().manual_seed(7)
    labels = torch.randint(0, L, (rows,), generator=gen).int()
    x = (torch.randn(L, k, generator=gen)[labels.long()] + 0.5 * torch.randn(rows, k, generator=gen)).to(heads.DTYPES[dtype])
    weight = torch.cat([torch.full((n,), 1.0 / max(n, 1)) for n in counts])
    own = heads.ClusterHeads(G, k, hidden, L, dtype=dtype, lr=0.05, p=0.2, seed=3)
    theta, mom = own.theta.cpu().double(), own.mom.cpu().double()
    start = theta.clone()
    off = torch.tensor(offsets, dtype=torch.int32).cuda()
    for i in range(steps):
        got = own.step(x.cuda(), off, labels.cuda(), weight.cuda()).cpu().double()
        want = plain_step(theta, mom, own.shapes, x.double(), offsets, labels, weight.double(), 0.05, 0.9, 0.2, 0.05, 3, i)
        for g, a, b in plain.parts(offsets):
            if b > a:
                assert (got[a:b] - want[a:b]).norm() <= 4 * bar * want[a:b].norm(), (i, g)
    for g, n in enumerate(counts):
        moved, want = own.theta[g].cpu().double() - start[g], theta[g] - start[g]
        assert (moved - want).norm() <= bar * want.norm() * (4 if dtype == "bf16" else 1) + 1e-30, g
        if n == 0:
            assert (moved == 0).all()
    s = own.score(x.cuda(), off, labels.cuda(), top=2)
    assert s.top_class.shape == (rows, 2) and torch.isfinite(s.logp).all()
    own.fuse(counts)
    assert (own.theta == own.theta[0]).all()


@pytest.mark.parametrize("workload,dtype", [("tiny_epoch", "f32"), ("ragged_epoch", "bf16")])
def test_command(workload, dtype, capsys):
    before, after = heads.main(["--workload", workload, "--steps", "40", "--dtype", dtype])
    assert all(a < b for a, b in zip(after[0], before[0]))  # every cluster's loss fell
    assert np.mean(after[1]) > np.mean(before[1])
    assert "heads fused" in capsys.readouterr().out
