"""Dropout from a counter, on the GPU: the same elements as the draws' definition in unsigned 64-bit arithmetic, and
their values rounded once."""
import numpy as np
import pytest
import torch

import ops_plain as plain

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def want_of(x, p, seed):
    # one product and, for bf16, one rounding: exactly what torch gives on the CPU
    v = x.float() * torch.tensor(plain.factor(p), dtype=torch.float32)
    return torch.where(plain.kept(*x.shape, p, seed), v, torch.zeros(())).to(x.dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 4), (5, 8), (2, 64), (17, 33), (64, 1000), (129, 257),
                                       (1, 40000), (4097, 3), (300, 1024)])
@pytest.mark.parametrize("p,seed", [(0.1, 0), (0.5, 2 ** 64 - 1)])
def test_elements_and_values(rows, cols, p, seed, dtype):
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(rows + cols)).to(TYPES[dtype])
    assert torch.equal(gcpsl.dropout(x.cuda(), p, seed).cpu(), want_of(x, p, seed))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first,cols,ld", [(0, 64, 72), (1, 64, 72), (3, 61, 65), (8, 128, 136)])
def test_strides_do_not_change_the_draws(first, cols, ld, dtype):
    x = torch.randn(50, ld + 8).to(TYPES[dtype])
    wide = x.cuda()
    xv = wide[:, first:first + cols]
    out = torch.full((50, cols + 5), 7.0, dtype=x.dtype, device="cuda")
    want = want_of(x[:, first:first + cols], 0.3, 5)
    gcpsl.dropout(xv, 0.3, 5, out=out[:, 2:2 + cols])
    assert torch.equal(out[:, 2:2 + cols].cpu(), want) and (out[:, :2] == 7).all() and (out[:, 2 + cols:] == 7).all()
    gcpsl.dropout(xv, 0.3, 5, out=xv)  # in place
    assert torch.equal(xv.cpu(), want)
    keep = torch.ones(ld + 8, dtype=torch.bool)
    keep[first:first + cols] = False
    assert torch.equal(wide.cpu()[:, keep], x[:, keep])


def test_rows_past_32_bits_of_elements():
    rows, ld = 2300, 1 << 20
    store = torch.empty(rows * ld + 64, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(rows, 40).bfloat16()
    v = store.as_strided((rows, 40), (ld, 1))
    v.copy_(x)
    assert torch.equal(gcpsl.dropout(v, 0.2, 8, out=v).cpu(), want_of(x, 0.2, 8))


def test_probabilities_at_the_ends():
    x = torch.randn(100, 100, device="cuda")
    assert torch.equal(gcpsl.dropout(x, 0.0, 1), x)
    assert torch.equal(gcpsl.dropout(x, 2.0 ** -18, 1), x)  # rounds to no element at all
    y = gcpsl.dropout(x, 65535 / 65536, 1)
    assert torch.equal(y.cpu(), want_of(x.cpu(), 65535 / 65536, 1)) and int((y != 0).sum()) < 10
    for p in (-1e-3, 1.0, 65535.6 / 65536, float("nan"), float("inf")):
        with pytest.raises(gcpsl.GCPSLError) as e:
            gcpsl.dropout(x, p, 1)
        assert e.value.code == gcpsl.EINVAL


def test_dropped_values_are_zero_and_kept_ones_go_through():
    x = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.0e38] * 64, device="cuda").view(1, 256)
    y, keep = gcpsl.dropout(x, 0.5, 77).cpu(), plain.kept(1, 256, 0.5, 77)
    assert (y[~keep] == 0).all() and torch.equal(torch.isnan(y), torch.isnan(x.cpu()) & keep)
    assert torch.equal(y[keep & ~torch.isnan(y)], (x.cpu() * 2)[keep & ~torch.isnan(y)])


def test_share_seeds_and_gradient():
    x = torch.ones(2048, 512, device="cuda")
    for p in (0.1, 0.25):
        n, t = x.numel(), round(65536 * p) / 65536
        share = float((gcpsl.dropout(x, p, 123) == 0).double().mean())
        assert abs(share - t) < 5 * np.sqrt(t * (1 - t) / n)  # five standard deviations of n draws
    a, b = gcpsl.dropout(x, 0.5, 1) != 0, gcpsl.dropout(x, 0.5, 2) != 0
    assert abs(float((a == b).double().mean()) - 0.5) < 5 * 0.5 / np.sqrt(x.numel())
    # y is linear in x, so its difference along any direction d is what the same call gives for d
    d, v = torch.randn(64, 96).cuda(), torch.randn(64, 96).cuda()
    diff = (gcpsl.dropout(v + d, 0.5, 3).double() - gcpsl.dropout(v - d, 0.5, 3).double()) / 2
    assert ((diff - gcpsl.dropout(d, 0.5, 3).double()).abs() <= 4 * plain.U32 * 2 * (v.abs() + d.abs())).all()


def test_refusals():
    x = torch.zeros(4, 8, device="cuda")
    for call in (lambda: gcpsl.dropout(x.cpu(), 0.5, 0), lambda: gcpsl.dropout(x.t(), 0.5, 0),
                 lambda: gcpsl.dropout(x.double(), 0.5, 0), lambda: gcpsl.dropout(x, 0.5, 0, out=x[:3]),
                 lambda: gcpsl.dropout(x[0], 0.5, 0)):
        with pytest.raises(ValueError):
            call()
    assert gcpsl.dropout(x[:0], 0.5, 0).shape == (0, 8) and gcpsl.dropout(x[:, :0], 0.5, 0).shape == (4, 0)
