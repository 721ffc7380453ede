"""Deeper heads (heads.BlockHeads): gated layers, residual norms and distillation in a chain, forward and backward,
against autograd in 64 bits; alone and replayed from a captured graph; and the command."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl, heads  # noqa: E402


def plain_loss(own, theta, x, offsets, labels, weight, teacher, T, share):
    """The same loss in 64 bits from a [G][P] leaf; products' weights rounded as the head's are (straight through)."""
    v = own._views(theta)
    if own.dtype == torch.bfloat16:
        v = {k: t + (t.detach().float().bfloat16().double() - t.detach()) if t.dim() == 3 else t for k, t in v.items()}
    norm = lambda t, w: torch.nn.functional.rms_norm(t, (t.shape[1],), eps=own.eps) * w  # noqa: E731
    total = 0.0
    for g, (a, b) in enumerate(zip(offsets, offsets[1:])):
        if a == b:
            continue
        p = {k: t[g] for k, t in v.items()}
        s = x[a:b] @ p["w_in"].T + p["b_in"]
        h = norm(s, p["norm_in"])
        for i in range(own.depth):
            pre = h @ p[f"w1_{i}"].T + p[f"b1_{i}"]
            gate, value = pre.chunk(2, 1)
            y = torch.nn.functional.silu(gate) * value
            out = y @ p[f"w2_{i}"].T + p[f"b2_{i}"]
            q = h @ p[f"wq_{i}"].T + p[f"bq_{i}"]
            s = s + own.beta * torch.sigmoid(q) * norm(out, p[f"norm_block_{i}"])
            h = norm(s, p[f"norm_next_{i}"])
        z = h @ p["w_out"].T + p["b_out"]
        ce = torch.nn.functional.cross_entropy(z, labels[a:b].long(), reduction="none")
        if teacher is None:
            total = total + (ce * weight[a:b]).sum()
            continue
        lp = torch.log_softmax(z / T, 1).gather(1, teacher[0][a:b].long())
        q = torch.softmax(teacher[1][a:b].double() / T, 1)
        kl = (q * (torch.log(q) - lp)).sum(1)
        total = total + ((share * T * T * kl + (1 - share) * ce) * weight[a:b]).sum()
    return total


def data(counts, k, L, dtype, seed=7):
    offsets = [int(v) for v in np.cumsum([0] + counts)]
    rows = offsets[-1]
    gen = torch.Generator().manual_seed(seed)
    labels = torch.randint(0, L, (rows,), generator=gen).int()
    x = (torch.randn(L, k, generator=gen)[labels.long()] + 0.5 * torch.randn(rows, k, generator=gen)).to(heads.DTYPES[dtype])
    best = torch.randn(rows, L, generator=gen).topk(3, 1)
    weight = torch.cat([torch.full((n,), 1.0 / max(n, 1)) for n in counts])
    return offsets, x, labels, weight, (best.indices.int().contiguous(), best.values.contiguous())


# relative bars as everywhere in this suite: 1e-4 in fp32, 2e-2 in bf16 (2-norm per cluster), times the two blocks
@pytest.mark.parametrize("dtype,bar", [("f32", 1e-4), ("bf16", 4e-2)])
@pytest.mark.parametrize("taught", [False, True])
@pytest.mark.parametrize("counts,k,d,hidden,L", [([40, 0, 75, 13], 36, 24, 20, 7), ([130, 64], 64, 128, 200, 70)])
def test_gradients_match_64_bits(counts, k, d, hidden, L, taught, dtype, bar):
    offsets, x, labels, weight, teacher = data(counts, k, L, dtype)
    own = heads.BlockHeads(len(counts), k, d, hidden, L, depth=2, dtype=dtype, beta=0.7, seed=3)
    own.theta += 0.02 * torch.randn(own.theta.shape, generator=torch.Generator().manual_seed(1)).cuda()
    o = torch.tensor(offsets, dtype=torch.int32).cuda()
    kind = dict(teacher=tuple(t.cuda() for t in teacher), temperature=2.0, share=0.25) if taught else {}
    loss = own.gradients(x.cuda(), o, labels.cuda(), weight.cuda(), **kind)
    theta = own.theta.cpu().double().requires_grad_()
    want = plain_loss(own, theta, x.double(), offsets, labels, weight.double(), teacher if taught else None, 2.0, 0.25)
    want.backward()
    got = float((loss.cpu().double() * weight.double()).sum())
    want = float(want.detach())
    assert abs(got - want) <= bar * abs(want)
    for g, n in enumerate(counts):
        d_own, d_want = own.grad[g].cpu().double(), theta.grad[g]
        assert (d_own - d_want).norm() <= bar * d_want.norm(), g
        if n == 0:
            assert (d_own == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(dtype):
    """A step's gradients captured into a graph: every replay on new inputs gives the eager bits, with eager work of the
    same heads between the replays."""
    counts, k, d, hidden, L = [60, 5, 0, 99], 40, 64, 96, 33
    offsets, x, labels, weight, teacher = data(counts, k, L, dtype)
    own = heads.BlockHeads(len(counts), k, d, hidden, L, dtype=dtype, seed=5)
    o = torch.tensor(offsets, dtype=torch.int32).cuda()
    x, labels, weight, teacher = x.cuda(), labels.cuda(), weight.cuda(), tuple(t.cuda() for t in teacher)
    run = lambda v: own.gradients(v, o, labels, weight, teacher=teacher)  # noqa: E731
    static = x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = run(static)
    for i in range(4):
        new = x + 0.1 * i
        want_loss = run(new).clone()
        want = own.grad.clone()
        own.grad.fill_(float("nan"))
        static.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(own.grad, want) and torch.equal(loss, want_loss), i


def test_serving_rows_match_training_rows():
    """The logits of few rows, by the kernels that few rows take, agree with those of the same rows among many."""
    counts, k, d, hidden, L = [200, 300, 150], 64, 256, 320, 50
    offsets, x, labels, _, _ = data(counts, k, L, "f32")
    own = heads.BlockHeads(3, k, d, hidden, L, seed=9)
    many = own.logits(x.cuda(), torch.tensor(offsets, dtype=torch.int32).cuda())
    at = torch.tensor([5, 250, 600])
    few = own.logits(x[at].cuda(), torch.tensor([0, 1, 2, 3], dtype=torch.int32).cuda())
    # products of up to 640 terms, five in a row, each off by about sqrt(640) 2^-24 of its magnitude
    assert (few - many[at.cuda()]).abs().max() <= 640 * 2.0 ** -23 * many.abs().max()


@pytest.mark.parametrize("workload,dtype", [("tiny_epoch", "f32"), ("ragged_epoch", "bf16")])
def test_command(workload, dtype, capsys):
    heads.main(["--workload", workload, "--steps", "3", "--dtype", dtype, "--blocks", "2"])
    assert "blocks taught" in capsys.readouterr().out
