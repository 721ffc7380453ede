"""The logits' gradient in rows whose mask, a finite fill, leaves no class."""
import math

import pytest
import torch

import ops_plain as plain
from test_gpu_score import TYPES, make

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


def gradient(z, labels):
    """(dz, in place) for gradients of one by both scores."""
    z, labels = z.cuda(), labels.cuda()
    r = gcpsl.score(z, labels)
    one = torch.ones(z.shape[0], device="cuda")
    d = gcpsl.score_grad(z, labels, r.lse, r.entropy, one, one)
    assert torch.equal(gcpsl.score_grad(z, labels, r.lse, r.entropy, one, one, out=z).isnan(), d.isnan())
    assert torch.equal(z.nan_to_num(), d.nan_to_num())
    return d.cpu(), r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [1, 10, 100, 5000])
def test_rows_ruled_out_by_a_finite_fill_take_no_gradient(L, dtype):
    """From -2^23 on, where fp32 steps are 1 and more, lse no longer holds log L: 0, not L times the gradient."""
    fills = [-float(2 ** 23 + 64 * 1024), -1e7, -1e9, -1e10, -1e20, -1e30, -3e38]
    z, labels = make(len(fills), L, dtype, seed=21)
    z = (torch.tensor(fills)[:, None] + 0 * z.float()).to(TYPES[dtype])
    d, _ = gradient(z, labels)
    assert (d == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [10, 100, 5000])
def test_rows_with_a_class_left_keep_theirs(L, dtype):
    fills = [-1e7, -1e9, -1e20, -1e30]
    z, labels = make(len(fills), L, dtype, seed=22)
    one = torch.ones(len(fills))
    for i, f in enumerate(fills):
        z[i, L // 2:] = f
        labels[i] = i % (L // 2)
    d, r = gradient(z, labels)
    want = plain.score_grad(z, labels, r.lse.cpu(), r.entropy.cpu(), one, one)
    lp = torch.where(z.float() < -1e6, 0.0, (z.float() - r.lse.cpu()[:, None]).abs()).double()
    bound = (2 + lp + r.entropy.cpu()[:, None]) * (lp + 24) * 4 * plain.U32
    assert ((d.double() - want).abs() <= plain.rounded(bound, want, z.dtype)).all()
    assert (d[:, L // 2:] == 0).all() and (d[:, :L // 2] != 0).any(1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [10, 100, 5000])
def test_uniform_rows_above_that(L, dtype):
    """p = exp(z - lse) is off by what lse's rounding, at most 2^-24 |lse|, makes of it."""
    values = [-1e6, -1e5, -1e4, -100.0, 0.0, 1e4, 1e6]
    z = torch.tensor(values)[:, None].expand(-1, L).to(TYPES[dtype]).contiguous()
    labels = torch.full((len(values),), L - 1, dtype=torch.int32)
    one = torch.ones(len(values), device="cuda")
    r = gcpsl.score(z.cuda(), labels.cuda())
    d = gcpsl.score_grad(z.cuda(), labels.cuda(), r.lse, g_logp=one).cpu().double()
    want = torch.full((len(values), L), -1 / L, dtype=torch.float64)
    want[:, L - 1] += 1
    off = torch.expm1((z[:, :1].double().abs() + math.log(L)) * 2 * plain.U32 + (L / 64 + 60) * plain.U32) / L
    assert ((d - want).abs() <= plain.rounded(off + 2 * plain.U32, want, z.dtype)).all()
