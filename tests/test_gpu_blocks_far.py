"""Gated layers, residual norms and distillation on tensors of more than 2^31 elements: rows on either side of every
32-bit limit against the 64-bit definitions, and other rows than those of the groups left as they were."""
import pytest
import torch

import blocks_plain as blocks
from test_gpu_group import check

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


def around(rows, cols):
    """Rows at the ends, and those in which element 2^31 and 2^32 lie (bytes 2^32 and 2^33 of bf16 too)."""
    at = {0, 1, rows - 2, rows - 1}
    for limit in (2 ** 30, 2 ** 31, 2 ** 32):
        at |= {r for r in (limit // cols - 1, limit // cols, limit // cols + 1) if 0 <= r < rows}
    return sorted(at)


def part_of(t, at):
    return None if t is None else t[at].cpu()


def test_gated():
    rows, n, k = 270_000, 4096, 64  # pre: 2.2e9 elements
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, k, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(2, 2 * n, k, generator=gen, device="cuda") / 8).bfloat16()
    v = (torch.randn(2, k, n, generator=gen, device="cuda") / 8).bfloat16()
    at = around(rows, 2 * n)
    cut, end = at[-4], rows - 1  # two groups, and a last row outside
    o = torch.tensor([0, cut, end], dtype=torch.int32, device="cuda")
    y = torch.full((rows, n), 7.0, dtype=torch.bfloat16, device="cuda")
    pre = torch.full((rows, 2 * n), 7.0, dtype=torch.bfloat16, device="cuda")
    gcpsl.group_gated_forward(x, o, w, out=y, pre=pre)
    offsets = [0, sum(r < cut for r in at), sum(r < end for r in at)]
    wy, ey, wp, ep, written = blocks.gated_forward(x[at].cpu(), offsets, w.cpu())
    keep = written.nonzero()[:, 0]
    check(part_of(y, at)[keep], wy[keep], ey[keep], "forward")
    check(part_of(pre, at)[keep], wp[keep], ep[keep], "pairs")
    assert (y[end] == 7).all() and (pre[end] == 7).all()
    del y
    d = torch.full((rows, 2 * n), 7.0, dtype=torch.bfloat16, device="cuda")
    gcpsl.group_gated_grad(x, o, v, pre, out=d)
    want, bound, _ = blocks.gated_grad(x[at].cpu(), offsets, v.cpu(), part_of(pre, at))
    check(part_of(d, at)[keep], want[keep], bound[keep], "gradient")
    assert (d[end] == 7).all()


def test_residual():
    rows, n = 540_000, 4096
    gen = torch.Generator(device="cuda").manual_seed(2)
    one = torch.randn(1024, n, generator=gen, device="cuda").bfloat16()
    # rows that repeat, each tensor from another row on
    t = [one.roll(i, 0).repeat(rows // 1024 + 1, 1)[:rows] for i in range(5)]
    w = 1 + 0.1 * torch.randn(2, n, generator=gen, device="cuda")
    at = around(rows, n)
    cut = at[-3]
    o = torch.tensor([0, cut, rows], dtype=torch.int32, device="cuda")
    got = gcpsl.group_residual_norm(t[0], o, y=t[1], gate=t[2], w_block=w, w_next=w, beta=0.5)
    offsets = [0, sum(r < cut for r in at), len(at)]
    want, _ = blocks.residual(*[part_of(v, at) for v in t[:1]], offsets, *[part_of(v, at) for v in t[1:3]], w.cpu(), w.cpu(),
                              1.0, 0.5)
    for name, value in got._asdict().items():
        check(part_of(value, at), *want[name], name)
    res = gcpsl.group_residual_norm_grad(got.out, o, g_out=t[3], g_h=t[4], y=t[1], gate=t[2], w_block=w, w_next=w,
                                         r_block=got.r_block, r_next=got.r_next, beta=0.5)
    want, _ = blocks.residual_grad(part_of(got.out, at), offsets, *[part_of(t[i], at) for i in (3, 4, 1, 2)], w.cpu(), w.cpu(),
                                   part_of(got.r_block, at), part_of(got.r_next, at), 1.0, 0.5)
    for name in ("dx", "dy", "dgate"):
        check(part_of(getattr(res, name), at), *want[name], name)
    # the weights' gradients against fp64 sums of the same terms on the GPU, a block of rows at a time
    sums = torch.zeros(2, n, dtype=torch.float64, device="cuda")
    mags = torch.zeros_like(sums)
    for i in range(0, rows, 30_000):
        r = slice(i, min(i + 30_000, rows))
        terms = t[4][r].double() * got.out[r].double() * got.r_next[r].double()[:, None]
        which = (torch.arange(r.start, r.stop, device="cuda") >= cut).long()
        for g in range(2):
            sums[g] += terms[which == g].sum(0)
            mags[g] += terms[which == g].abs().sum(0)
    # a column's rows are added by pieces, in chains of at most rows / 480 + 600 (pieces, then their sums)
    assert ((res.dw_next.double() - sums).abs() <= (rows / 480 + 600) * 2.0 ** -24 * mags).all()


def test_distillation():
    rows, L = 17_000, 131_072  # 2.2e9 logits
    gen = torch.Generator(device="cuda").manual_seed(3)
    one = (2 * torch.randn(17, L, generator=gen, device="cuda")).bfloat16()
    z = one.repeat(1000, 1)
    best = torch.randn(17, L, generator=gen, device="cuda").topk(7, 1)
    cls, val = best.indices.int().repeat(1000, 1), best.values.repeat(1000, 1)
    labels = torch.randint(0, L, (rows,), generator=gen, device="cuda").int()
    at = around(rows, L)
    got = gcpsl.distill(z, cls, val, temperature=2.0, labels=labels)
    want = blocks.distill(part_of(z, at), part_of(cls, at), part_of(val, at), 2.0, part_of(labels, at))
    for name, value in got._asdict().items():
        check(part_of(value, at), *want[name], name)
    g = torch.randn(rows, generator=gen, device="cuda")
    dz = gcpsl.distill_grad(z, cls, val, got.lse_t, temperature=2.0, labels=labels, lse=got.lse, g_kl=g, g_logp=g, out=z)
    check(part_of(dz, at), *blocks.distill_grad(one[[r % 17 for r in at]].cpu(), part_of(cls, at), part_of(val, at),
                                                part_of(got.lse_t, at), 2.0, part_of(labels, at), part_of(got.lse, at),
                                                part_of(g, at), part_of(g, at)), "dz")
