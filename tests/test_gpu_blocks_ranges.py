"""The ends of what residual norms and distillation take, as their documentation states them: squares that add up to
just below and above fp32's range, teacher's entries with and without a weight in fp32."""
import math

import pytest
import torch

import blocks_plain as blocks
from test_gpu_group import TYPES, check, gpu, make

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [7, 64, 200, 4096, 9000, 16400])
def test_largest_squares(n, dtype):
    """Rows of +-2^e whose squares add up to more than 2^125 and no more than 2^127 are normed as any others, those of four
    times as large values, 2^129 or more, have r = 0."""
    T, rows = TYPES[dtype], 5
    v = 2.0 ** math.floor((127 - math.log2(n)) / 2)
    assert 2.0 ** 125 < n * v * v <= 2.0 ** 127
    sign = torch.where(make(1, rows, n) < 0, -1.0, 1.0)
    x, w = (v * sign).to(T), 1 + make(2, 1, n, scale=0.3)
    o = torch.tensor([0, rows], dtype=torch.int32).cuda()
    got = gcpsl.group_residual_norm(gpu(x), o, w_next=gpu(w))
    want, _ = blocks.residual(x, [0, rows], w_next=w)
    check(got.h, *want["h"], "h")
    check(got.r_next, *want["r_next"], "r_next")
    again = gcpsl.group_residual_norm(torch.zeros_like(x, device="cuda"), o, y=gpu(x), w_block=gpu(w))
    assert torch.equal(again.out, got.h) and torch.equal(again.r_block, got.r_next)
    gh = make(3, rows, n, dtype=T)
    res = gcpsl.group_residual_norm_grad(gpu(x), o, g_h=gpu(gh), w_next=gpu(w), r_next=got.r_next)
    want, _ = blocks.residual_grad(x, [0, rows], g_h=gh, w_next=w, r_next=got.r_next.cpu())
    check(res.dx, *want["dx"], "dx")
    check(res.dw_next, *want["dw_next"], "dw_next")
    far = gcpsl.group_residual_norm(gpu(4 * x), o, w_next=gpu(w))
    assert (far.r_next == 0).all() and (far.h == 0).all()


@pytest.mark.parametrize("T", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("L", [40, 300, 70_000])
def test_entries_far_below_the_best(L, T):
    """An entry 88 T below the row's best one has no weight, so that a class that the row rules out may be among such; 86 T
    below it has, and makes the divergence infinite."""
    z = make(1, 2, L)
    z[:, 3] = -math.inf
    cls = torch.tensor([[0, 3, 7]] * 2, dtype=torch.int32)
    val = torch.tensor([[1.0, 1.0 - 88 * T, 0.5], [1.0, 1.0 - 86 * T, 0.5]])
    got = gcpsl.distill(gpu(z), gpu(cls), gpu(val), temperature=T)
    without = gcpsl.distill(gpu(z), gpu(cls[:, ::2].contiguous()), gpu(val[:, ::2].contiguous()), temperature=T)
    assert got.kl[1] == math.inf
    # the same terms w (log w - log p) and weights, added in another order: a few roundings of their magnitude, which is
    # at most the entries' distance (0.5 / T), a logit's from the row's best one (8 / T at most here) and log L
    assert abs(got.kl[0] - without.kl[0]) <= 16 * 2.0 ** -24 * (abs(without.kl[0]) + 8 / T + math.log(L))
