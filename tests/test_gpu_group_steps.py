"""Products over rows grouped by cluster at every number of steps that their sums take, and dropout of more elements
than one launch's short form, against their 64-bit definitions (tests/ops_plain.py's bounds)."""
import pytest
import torch

import ops_plain as plain
from test_gpu_group import TYPES, check, gpu, make, offsets_of

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

# about 1,100 tiles of 32 x 32 results, 160 of 64 x 128: more than products from registers take, fewer than two a CU
COUNTS, OTHER = [700, 0, 1290, 1], 520
# sums that end with, one before and one past a step of 64, and of 16, from the shortest to eight steps
LENGTHS = [8, 9, 16, 17, 63, 64, 65, 127, 128, 129, 191, 192, 193, 200, 256, 257, 319, 320, 321, 384, 385, 447, 448, 449, 505]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", LENGTHS)
def test_every_number_of_steps(length, dtype):
    T, off, G = TYPES[dtype], offsets_of(COUNTS), len(COUNTS)
    rows, p = off[-1], 0.1
    x, dy = make(1, rows, length, dtype=T), make(2, rows, length, dtype=T)
    w, b = make(3, G, OTHER, length, dtype=T, scale=length ** -0.5), make(4, G, OTHER, scale=0.3)
    v, gate = make(5, G, length, 1000, dtype=T, scale=length ** -0.5), make(6, rows, 1000, dtype=T)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    y = gcpsl.group_forward(gpu(x), o, gpu(w), gpu(b), relu=True, p=p, seed=5)
    check(y, *plain.forward(x, off, w, b, True, p, 5)[:2], "forward")
    dx = gcpsl.group_input_grad(gpu(dy), o, gpu(v), gate=gpu(gate), p=p)
    check(dx, *plain.input_grad(dy, off, v, gate, p)[:2], "input gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count", [1, 63, 64, 65, 191, 192, 193, 383, 384, 385, 577, 769])
def test_weight_gradients_with_and_without_pieces(count, dtype):
    """Groups that hold almost all rows, next to groups of none or few."""
    T = TYPES[dtype]
    for counts in ([count], [0, count, 2, 0]):
        off, G, n, k = offsets_of(counts), len(counts), 65, 40
        dy, x = make(7, off[-1], n, dtype=T), make(8, off[-1], k, dtype=T)
        dw, db = gcpsl.group_weight_grad(gpu(dy), gpu(x), torch.tensor(off, dtype=torch.int32).cuda())
        want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
        check(dw, want_w, bound_w, "weight gradient")
        check(db, want_b, bound_b, "bias gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1001, 1002, 1004, 1007])
def test_dropout_of_many_rows_with_ends(cols, dtype):
    """More than 2^19 pieces of eight elements; written in place inside a wider tensor."""
    T, rows, p, seed = TYPES[dtype], 4300, 0.25, 99
    x = make(9, rows, cols, dtype=T)
    want = torch.where(plain.kept(rows, cols, p, seed), x.double() * plain.factor(p), 0.0)
    wide = torch.full((rows, cols + 3), 7.0, dtype=T, device="cuda")
    view = wide[:, 1:cols + 1]
    view.copy_(x)
    assert gcpsl.dropout(view, p, seed, out=view) is view
    got = gcpsl.dropout(gpu(x), p, seed)
    assert torch.equal(got, view) and (wide[:, 0] == 7).all() and (wide[:, cols + 1:] == 7).all()
    check(got, want, plain.rounded(want.abs() * 2 * plain.U32, want, T))


# fewer tiles of 64 x 64 than CUs, and too many of 32 x 32 for products from registers: 225 and 816 (forward), 250 and
# 480 of 32 x 64 (input gradient, sums of 256 on)
FEWER, WIDE, NARROW = [500, 0, 999, 1], 520, 600
LONGER = [l for l in LENGTHS if l >= 256] + [511, 512, 513, 575, 577, 640, 641, 703, 705, 1001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", LENGTHS + [513, 577, 640, 641, 1001])
def test_every_number_of_steps_of_fewer_tiles(length, dtype):
    T, off, G = TYPES[dtype], offsets_of(FEWER), len(FEWER)
    rows = off[-1]
    x, w = make(11, rows, length, dtype=T), make(12, G, WIDE, length, dtype=T, scale=length ** -0.5)
    b, o = make(13, G, WIDE, scale=0.3), torch.tensor(off, dtype=torch.int32).cuda()
    wide = torch.full((rows + 1, length + 3), float("nan"), dtype=T, device="cuda")  # rows between values not theirs
    view = wide[:rows, 1:length + 1]
    view.copy_(x)
    check(gcpsl.group_forward(view, o, gpu(w), gpu(b), relu=True), *plain.forward(x, off, w, b, True)[:2], "forward")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [NARROW, NARROW + 1, NARROW - 7])
@pytest.mark.parametrize("length", LONGER)
def test_input_gradients_of_fewer_tiles(length, width, dtype):
    T, off, G = TYPES[dtype], offsets_of(FEWER), len(FEWER)
    rows, p = off[-1], 0.2
    dy, w = make(14, rows, length, dtype=T), make(15, G, length, width, dtype=T, scale=length ** -0.5)
    gate, o = make(16, rows, width, dtype=T), torch.tensor(off, dtype=torch.int32).cuda()
    dx = gcpsl.group_input_grad(gpu(dy), o, gpu(w), gate=gpu(gate), p=p)
    check(dx, *plain.input_grad(dy, off, w, gate, p)[:2], "input gradient")


@pytest.mark.parametrize("big", [float("inf"), -float("inf"), float("nan"), 3e38, 2.0 ** 60])
def test_large_values_of_fewer_tiles(big):
    """A value without a split into three parts, in one row and in one weight: every other result stays finite and
    right, those that meet it are what fp32 products give."""
    off, G, k = offsets_of(FEWER), len(FEWER), 321
    x, w = make(17, off[-1], k), make(18, G, WIDE, k, scale=k ** -0.5)
    x[77, 300] = big
    w[2, 5, 13] = big
    o = torch.tensor(off, dtype=torch.int32).cuda()
    y = gcpsl.group_forward(gpu(x), o, gpu(w)).cpu().double()
    want, bound, _ = plain.forward(x, off, w)
    touched = torch.zeros_like(want, dtype=torch.bool)
    touched[77] = True
    touched[off[2]:off[3], 5] = True
    assert ((y - want).abs() <= bound)[~touched].all()
    if not torch.isfinite(torch.tensor(big)):
        got, ref = y[touched], want[touched]
        assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[~torch.isnan(got)], ref[~torch.isnan(ref)])
    elif big < 1e30:  # (the largest ones overflow or not by the order of a sum)
        assert ((y - want).abs() <= bound)[touched].all()
