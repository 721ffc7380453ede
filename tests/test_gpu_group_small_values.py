"""fp32 products of values that run out of bf16's exponents, whose sum of three parts is then exact to 2^-134 only (half of
bf16's smallest step), in the kernels that take values apart so; and whole in the others, by the sizes of the call."""
import pytest
import torch

import ops_plain as plain

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

STEP = 2.0 ** -134


def check(got, a, b, size):
    """a [m][q] by b [q][c]: the sums' bound, and each operand's missing part by the other's size."""
    a, b = a.double(), b.double()
    want = a @ b
    bound = (size + 8) * plain.UACC * (a.abs() @ b.abs())
    bound = bound + STEP * (a.abs().sum(1)[:, None] + b.abs().sum(0)[None, :]) * (1 + size * plain.UACC)
    assert ((got.double().cpu() - want).abs() <= bound + want.abs() * 2 * plain.U32).all()


# many tiles of 128 x 128, fewer of 64 x 64 than CUs, few rows, few columns
@pytest.mark.parametrize("rows,n,k", [(4096, 256, 320), (1000, 128, 256), (8, 256, 256), (3000, 24, 64)])
@pytest.mark.parametrize("small", [-112, -120, -127, -131])
def test_small_operands(rows, n, k, small):
    g = torch.Generator().manual_seed(rows - small)
    o = torch.tensor([0, rows], dtype=torch.int32).cuda()
    for ex, ew in ((small, 40), (40, small)):
        x = torch.randn(rows, k, generator=g) * 2.0 ** ex
        w = torch.randn(1, n, k, generator=g) * 2.0 ** ew
        check(gcpsl.group_forward(x.cuda(), o, w.cuda()), x, w[0].T, k)
        dy = torch.randn(rows, n, generator=g) * 2.0 ** ex
        check(gcpsl.group_input_grad(dy.cuda(), o, w.cuda()), dy, w[0], n)
        xw = torch.randn(rows, k, generator=g) * 2.0 ** ew
        check(gcpsl.group_weight_grad(dy.cuda(), xw.cuda(), o)[0][0], dy.T, xw, rows)
