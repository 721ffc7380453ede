"""Products over rows grouped by cluster at sizes of many 128 x 128 tiles: the kernels that larger layers take, at every
remainder of their vectors, with gates, strides, infinities and the largest values (tests/ops_plain.py's bounds)."""
import numpy as np
import pytest
import torch

import ops_plain as plain
from test_gpu_group import TYPES, check, gpu, make, offsets_of

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

COUNTS = [1500, 0, 700, 333, 1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rest", range(8))
def test_every_remainder_through_relu_dropout_and_gate(rest, dtype):
    """Operands inside wider tensors of NaN, in rows that start at any element."""
    T, off, G = TYPES[dtype], offsets_of(COUNTS), len(COUNTS)
    rows, n, k, p = off[-1], 328 + rest, 520 + rest, 0.25
    x, dy = make(1, rows, k, dtype=T), make(2, rows, n, dtype=T)
    w, b = make(3, G, n, k, dtype=T, scale=k ** -0.5), make(4, G, n, scale=0.3)
    wide = [torch.full((rows + 1, c + 5), float("nan"), dtype=T, device="cuda") for c in (k, n, n, k)]
    xv, dv, yv, gv = (t[:rows, 1:c + 1] for t, c in zip(wide, (k, n, n, k)))
    xv.copy_(x)
    dv.copy_(dy)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    gcpsl.group_forward(xv, o, gpu(w), gpu(b), relu=True, p=p, seed=77, out=yv)
    check(yv, *plain.forward(x, off, w, b, True, p, 77)[:2], "forward")
    gcpsl.group_input_grad(dv, o, gpu(w), gate=xv, p=p, out=gv)
    check(gv, *plain.input_grad(dy, off, w, x, p)[:2], "input gradient")
    for t, c in ((wide[2], n), (wide[3], k)):  # nothing is written beside the results
        assert torch.isnan(t[rows]).all() and torch.isnan(t[:, 0]).all() and torch.isnan(t[:, c + 1:]).all()
    dw, db = gcpsl.group_weight_grad(dv, xv, o)
    want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
    check(dw, want_w, bound_w, "weight gradient")
    check(db, want_b, bound_b, "bias gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,n,k", [([9000, 0, 5000], 40, 72), ([7000, 7001], 33, 3), ([40000], 7, 5), ([5, 30000], 2, 300)])
def test_many_rows_of_narrow_layers(counts, n, k, dtype):
    T, off, G = TYPES[dtype], offsets_of(counts), len(counts)
    rows = off[-1]
    x, dy, w = make(11, rows, k, dtype=T), make(12, rows, n, dtype=T), make(13, G, n, k, dtype=T, scale=k ** -0.5)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    check(gcpsl.group_forward(gpu(x), o, gpu(w)), *plain.forward(x, off, w)[:2], "forward")
    check(gcpsl.group_input_grad(gpu(dy), o, gpu(w)), *plain.input_grad(dy, off, w)[:2], "input gradient")
    dw, db = gcpsl.group_weight_grad(gpu(dy), gpu(x), o)
    want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
    check(dw, want_w, bound_w, "weight gradient")
    check(db, want_b, bound_b, "bias gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(328, 264), (331, 269)])
def test_infinities_as_the_sums_give_them(n, k, dtype):
    T, rows = TYPES[dtype], 2600
    x, w = make(21, rows, k, dtype=T), make(22, 1, n, k, dtype=T)
    x[3, 5], x[1700, 0], x[1700, 9] = float("inf"), float("inf"), float("-inf")
    w[0, 4, 5] = 0
    x[40, 7] = float("nan")
    o = torch.tensor([0, rows], dtype=torch.int32).cuda()
    want = x.double() @ w[0].double().T
    y = gcpsl.group_forward(gpu(x), o, gpu(w)).cpu().float()
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.isnan(y[3, 4]) and torch.isnan(y[40]).all()
    assert torch.equal(y[torch.isinf(want)], want[torch.isinf(want)].float())
    # the same as an input gradient: w transposed, x the outputs' gradient
    y = gcpsl.group_input_grad(gpu(x), o, gpu(w.transpose(1, 2).contiguous())).cpu().float()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y[torch.isinf(want)], want[torch.isinf(want)].float())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(328, 264), (331, 269)])
def test_large_finite_values(n, k, dtype):
    """Products near the largest finite value, which the sum must not lose to an overflow on its way."""
    T, rows = TYPES[dtype], 2600
    x, w = torch.zeros(rows, k, dtype=T), torch.zeros(1, n, k, dtype=T)
    top = torch.finfo(T).max
    x[:, 0], w[0, :, 0] = top, 0.5
    x[0, 1], w[0, 3, 1] = top, -0.25
    o = torch.tensor([0, rows], dtype=torch.int32).cuda()
    check(gcpsl.group_forward(gpu(x), o, gpu(w)), *plain.forward(x, [0, rows], w)[:2])
    check(gcpsl.group_input_grad(gpu(x), o, gpu(w.transpose(1, 2).contiguous())), *plain.forward(x, [0, rows], w)[:2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(200, 1), (96, 3), (1, 96), (5, 200), (4, 8), (8, 4), (24, 2000), (2000, 24)])
def test_few_results_at_the_edges_of_the_vectors(n, k, dtype):
    T, counts = TYPES[dtype], [1, 0, 15, 16, 17, 40]
    off, G = offsets_of(counts), len(counts)
    x, dy, w = make(31, off[-1], k, dtype=T), make(32, off[-1], n, dtype=T), make(33, G, n, k, dtype=T, scale=k ** -0.5)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    check(gcpsl.group_forward(gpu(x), o, gpu(w)), *plain.forward(x, off, w)[:2], "forward")
    check(gcpsl.group_input_grad(gpu(dy), o, gpu(w)), *plain.input_grad(dy, off, w)[:2], "input gradient")


def test_the_same_bits_again():
    off = offsets_of(COUNTS)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    for T in TYPES.values():
        for n, k in ((328, 520), (64, 520), (328, 72)):
            x, dy, w = make(41, off[-1], k, dtype=T), make(42, off[-1], n, dtype=T), make(43, len(COUNTS), n, k, dtype=T)
            a = [gcpsl.group_forward(gpu(x), o, gpu(w)), gcpsl.group_input_grad(gpu(dy), o, gpu(w))]
            b = [gcpsl.group_forward(gpu(x), o, gpu(w)), gcpsl.group_input_grad(gpu(dy), o, gpu(w))]
            assert all(np.array_equal(u.float().cpu().numpy(), v.float().cpu().numpy()) for u, v in zip(a, b))
