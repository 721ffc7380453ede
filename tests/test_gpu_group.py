"""Products over rows grouped by cluster, on the GPU, against their 64-bit definition: every element within the bound
that its sum's length and magnitude give (tests/ops_plain.py)."""
import numpy as np
import pytest
import torch

import ops_plain as plain

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def offsets_of(counts, first=0):
    return [first + int(v) for v in np.cumsum([0] + list(counts))]


def gpu(t):
    return None if t is None else t.cuda()


def make(seed, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def check(got, want, bound, what=""):
    got = got.detach().cpu().double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], bound[bad][:4])


# (rows of each group, n, k): single rows, groups of none, tiles not filled and just passed, widths from one on, odd
# ones and multiples of 8, 64 and 128, more groups than a wave has lanes, long sums
SHAPES = [
    ([1], 1, 1), ([1], 10, 128), ([0, 1, 0], 3, 5), ([3, 0, 2, 1], 16, 32), ([63, 64, 65], 64, 64),
    ([200, 0, 55, 1], 72, 136), ([129, 31], 130, 257), ([5] * 70, 24, 40), ([0] * 66 + [17, 9], 8, 16),
    ([300], 77, 1001), ([1, 2, 1, 0, 3], 256, 512), ([257, 700, 3], 256, 192), ([40, 0, 513], 520, 264),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,n,k", SHAPES)
def test_three_products(counts, n, k, dtype):
    T, off, G = TYPES[dtype], offsets_of(counts), len(counts)
    rows = off[-1]
    x, w, b = make(1, rows, k, dtype=T), make(2, G, n, k, dtype=T, scale=k ** -0.5), make(3, G, n, scale=0.3)
    dy, o = make(4, rows, n, dtype=T), torch.tensor(off, dtype=torch.int32).cuda()
    y = gcpsl.group_forward(gpu(x), o, gpu(w), gpu(b))
    assert y.dtype == T
    check(y, *plain.forward(x, off, w, b)[:2], "forward")
    dx = gcpsl.group_input_grad(gpu(dy), o, gpu(w))
    check(dx, *plain.input_grad(dy, off, w)[:2], "input gradient")
    dw, db = gcpsl.group_weight_grad(gpu(dy), gpu(x), o)
    want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
    check(dw, want_w, bound_w, "weight gradient")
    check(db, want_b, bound_b, "bias gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rest", range(8))
@pytest.mark.parametrize("counts,n,k", [([5, 0, 70], 128, 64), ([200, 131], 264, 136), ([129], 8, 200)])
def test_every_remainder_of_the_vectors(counts, n, k, rest, dtype):
    """Widths that leave every number of elements past a 16-byte piece, at the end of the sum and of the columns, next
    to values that must not be read as theirs."""
    T, off, G = TYPES[dtype], offsets_of(counts), len(counts)
    rows, n, k = off[-1], n + rest, k + rest
    w = make(102, G, n, k, dtype=T, scale=k ** -0.5)
    wide_x, wide_d = (torch.full((rows + 1, c + 5), float("nan"), dtype=T, device="cuda") for c in (k, n))
    x, dy = make(101, rows, k, dtype=T), make(103, rows, n, dtype=T)
    xv, dv = wide_x[:rows, :k], wide_d[:rows, :n]
    xv.copy_(x)
    dv.copy_(dy)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    check(gcpsl.group_forward(xv, o, gpu(w)), *plain.forward(x, off, w)[:2], "forward")
    check(gcpsl.group_input_grad(dv, o, gpu(w)), *plain.input_grad(dy, off, w)[:2], "input gradient")
    dw, db = gcpsl.group_weight_grad(dv, xv, o)
    want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
    check(dw, want_w, bound_w, "weight gradient")
    check(db, want_b, bound_b, "bias gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,n,k", [([4000, 0, 1300, 700], 48, 40), ([9000], 136, 128), ([3, 5000, 2000], 40, 33)])
def test_weight_gradients_in_pieces(counts, n, k, dtype):
    """Long sums of few outputs, taken in pieces that are joined; groups of one piece and of none beside them."""
    T, off, G = TYPES[dtype], offsets_of(counts), len(counts)
    x, dy = make(111, off[-1], k, dtype=T), make(112, off[-1], n, dtype=T)
    assert gcpsl.group_workspace_bytes(dtype, G, off[-1], n, k) > 0
    o = torch.tensor(off, dtype=torch.int32).cuda()
    dw, db = gcpsl.group_weight_grad(gpu(dy), gpu(x), o)
    want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
    check(dw, want_w, bound_w)
    check(db, want_b, bound_b)
    again = gcpsl.group_weight_grad(gpu(dy), gpu(x), o)
    assert torch.equal(again[0], dw) and torch.equal(again[1], db)
    need = gcpsl.group_workspace_bytes(dtype, G, off[-1], n, k)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")  # NaN throughout
    again = gcpsl.group_weight_grad(gpu(dy), gpu(x), o, workspace=ws, bias=False)
    assert torch.equal(again[0], dw) and again[1] is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,n,k", [([70, 0, 33], 65, 48), ([260, 5], 264, 128), ([2, 1, 0, 1], 512, 256)])
def test_relu_dropout_and_the_gradient_through_them(counts, n, k, dtype):
    T, off, G, p, seed = TYPES[dtype], offsets_of(counts), len(counts), 0.3, 2 ** 63 + 11
    rows = off[-1]
    x, w, b = make(5, rows, k, dtype=T), make(6, G, n, k, dtype=T, scale=k ** -0.5), make(7, G, n, scale=0.3)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    y = gcpsl.group_forward(gpu(x), o, gpu(w), gpu(b), relu=True, p=p, seed=seed)
    want, bound, _ = plain.forward(x, off, w, b, True, p, seed)
    check(y, want, bound)
    dropped = ~plain.kept(rows, n, p, seed)
    assert (y.cpu()[dropped] == 0).all()
    # the same elements as the dropout of the layer without it
    alone = gcpsl.dropout(gcpsl.group_forward(gpu(x), o, gpu(w), gpu(b), relu=True), p, seed)
    assert torch.equal(alone == 0, y == 0)
    # next layer's input gradient, gated by this one's output
    w2, dz = make(8, G, 24, n, dtype=T, scale=n ** -0.5), make(9, rows, 24, dtype=T)
    dx = gcpsl.group_input_grad(gpu(dz), o, gpu(w2), gate=y, p=p)
    check(dx, *plain.input_grad(dz, off, w2, y.cpu(), p)[:2])
    assert (dx[y <= 0] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_against_differences(dtype):
    """The loss sum(y dy) is linear in x, w and b each, so its central difference along any direction is its gradient
    there, whatever the step: along a random direction the kernels' gradients agree with differences of the 64-bit
    forward pass to their own rounding."""
    T, counts, n, k = TYPES[dtype], [9, 0, 20], 40, 24
    off, G = offsets_of(counts), 3
    rows = off[-1]
    x, w, b = make(11, rows, k, dtype=T), make(12, G, n, k, dtype=T), make(13, G, n)
    dy, o = make(14, rows, n, dtype=T), torch.tensor(off, dtype=torch.int32).cuda()

    def loss(x, w, b):
        return float((plain.forward(x.double(), off, w.double(), b.double())[0] * dy.double()).sum())

    dx = gcpsl.group_input_grad(gpu(dy), o, gpu(w)).cpu().double()
    dw, db = (t.cpu().double() for t in gcpsl.group_weight_grad(gpu(dy), gpu(x), o))
    bounds = (plain.input_grad(dy, off, w)[1], *plain.weight_grad(dy, x, off)[2:])
    for i, (grad, bound) in enumerate(zip((dx, dw, db), bounds)):
        direction = make(20 + i, *grad.shape).double()
        at = [t.double() for t in (x, w, b)]
        hi, lo = list(at), list(at)
        hi[i], lo[i] = at[i] + direction, at[i] - direction
        difference = (loss(*hi) - loss(*lo)) / 2
        assert abs(difference - float((grad * direction).sum())) <= float((bound * direction.abs()).sum()) + 1e-9


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(40, 72), (256, 128), (33, 65)])
def test_strides_and_offsets_of_every_operand(n, k, dtype):
    """Rows inside wider tensors, from odd first elements; weights, biases and their gradients inside one flat vector
    per group; shared weights; rows outside every group left as they are."""
    T, counts = TYPES[dtype], [50, 0, 81, 3]
    off, G = offsets_of(counts, first=2), 4
    rows = off[-1] + 5
    wide_x = torch.full((rows, k + 13), float("nan"), dtype=T, device="cuda")
    x = make(31, rows, k, dtype=T)
    xv = wide_x[:, 5:5 + k]
    xv.copy_(x)
    P = n * k + n + 7
    flat = torch.full((G, P), float("nan"), dtype=T, device="cuda")
    w = make(32, G, n, k, dtype=T, scale=k ** -0.5)
    wv = flat[:, 3:3 + n * k].view(G, n, k)
    wv.copy_(w)
    flat_b = torch.full((G, P), float("nan"), device="cuda")
    b = make(33, G, n)
    bv = flat_b[:, n * k:n * k + n]
    bv.copy_(b)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    wide_y = torch.full((rows, n + 9), 7.0, dtype=T, device="cuda")
    yv = wide_y[:, 1:1 + n]
    assert gcpsl.group_forward(xv, o, wv, bv, out=yv) is yv
    want, bound, written = plain.forward(x, off, w, b)
    check(yv[written.cuda()], want[written], bound[written])
    assert (yv[~written.cuda()] == 7).all() and (wide_y[:, 0] == 7).all() and (wide_y[:, 1 + n:] == 7).all()

    dy = make(34, rows, n, dtype=T)
    wide_y[:, 1:1 + n] = dy.cuda()
    wide_dx = torch.full((rows, k + 3), 7.0, dtype=T, device="cuda")
    dxv = wide_dx[:, 2:2 + k]
    gcpsl.group_input_grad(yv, o, wv, out=dxv)
    want, bound, written = plain.input_grad(dy, off, w)
    check(dxv[written.cuda()], want[written], bound[written])
    assert (dxv[~written.cuda()] == 7).all() and (wide_dx[:, :2] == 7).all() and (wide_dx[:, 2 + k:] == 7).all()

    grad = torch.full((G, P), 7.0, device="cuda")
    dwv, dbv = grad[:, 1:1 + n * k].view(G, n, k), grad[:, 2 + n * k:2 + n * k + n]
    gcpsl.group_weight_grad(yv, xv, o, dw=dwv, db=dbv)
    want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
    check(dwv, want_w, bound_w)
    check(dbv, want_b, bound_b)
    assert (grad[:, 0] == 7).all() and (grad[:, 1 + n * k] == 7).all() and (grad[:, 2 + n * k + n:] == 7).all()

    shared = gcpsl.group_forward(xv, o, wv[:1].expand(G, n, k), bv[:1].expand(G, n))
    want, bound, written = plain.forward(x, off, w[:1].expand(G, n, k), b[:1].expand(G, n))
    check(shared[written.cuda()], want[written], bound[written])
    same = gcpsl.group_forward(xv[:1].expand(rows, k), o, wv)
    want, bound, written = plain.forward(x[:1].expand(rows, k), off, w)
    check(same[written.cuda()], want[written], bound[written])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(64, 128), (37, 51)])
def test_groups_do_not_see_each_other(n, k, dtype):
    """A NaN or infinity in one group's rows or weights shows in that group alone."""
    T, counts = TYPES[dtype], [30, 41, 50]
    off = offsets_of(counts)
    x, w, dy = make(41, off[-1], k, dtype=T), make(42, 3, n, k, dtype=T), make(43, off[-1], n, dtype=T)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    clean = [gcpsl.group_forward(gpu(x), o, gpu(w)), gcpsl.group_input_grad(gpu(dy), o, gpu(w)),
             *gcpsl.group_weight_grad(gpu(dy), gpu(x), o)]
    x[off[1]:off[2]] = float("inf")
    dy[off[1]:off[2]] = float("nan")
    w[1] = float("nan")
    got = [gcpsl.group_forward(gpu(x), o, gpu(w)), gcpsl.group_input_grad(gpu(dy), o, gpu(w)),
           *gcpsl.group_weight_grad(gpu(dy), gpu(x), o)]
    for a, c in zip(got[:2], clean[:2]):
        assert torch.equal(a[:off[1]], c[:off[1]]) and torch.equal(a[off[2]:], c[off[2]:])
        assert torch.isnan(a[off[1]:off[2]]).all()
    for a, c in zip(got[2:], clean[2:]):
        assert torch.equal(a[0], c[0]) and torch.equal(a[2], c[2]) and torch.isnan(a[1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_as_the_sums_give_them(dtype):
    """One infinite input: its row's sums are infinite with the weight's sign, or NaN for a zero weight; sums of
    opposite infinities are NaN; the ReLU keeps a NaN, the dropout's zero covers it."""
    T, n, k = TYPES[dtype], 48, 64
    x, w = make(51, 40, k, dtype=T), make(52, 1, n, k, dtype=T)
    x[3, 5], x[7, 0], x[7, 9] = float("inf"), float("inf"), float("-inf")
    w[0, 4, 5] = 0
    o = torch.tensor([0, 40], dtype=torch.int32).cuda()
    y = gcpsl.group_forward(gpu(x), o, gpu(w)).cpu().float()
    want = x.double() @ w[0].double().T
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.isnan(y[3, 4])
    assert torch.equal(y[torch.isinf(want)], want[torch.isinf(want)].float())
    y = gcpsl.group_forward(gpu(x), o, gpu(w), relu=True, p=0.5, seed=9).cpu()
    keep = plain.kept(40, n, 0.5, 9)
    assert torch.equal(torch.isnan(y), torch.isnan(want) & keep) and (y[~keep] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_finite_values(dtype):
    """Products near the largest finite value, which the sum must not lose to an overflow on its way."""
    T, n, k = TYPES[dtype], 32, 32
    x, w = torch.zeros(33, k, dtype=T), torch.zeros(1, n, k, dtype=T)
    top = torch.finfo(T).max
    x[:, 0], w[0, :, 0] = top, 0.5
    x[0, 1], w[0, 3, 1] = top, -0.25
    o = torch.tensor([0, 33], dtype=torch.int32).cuda()
    y = gcpsl.group_forward(gpu(x), o, gpu(w)).cpu()
    check(y, *plain.forward(x, [0, 33], w)[:2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(dtype):
    T = TYPES[dtype]
    o = torch.zeros(4, dtype=torch.int32, device="cuda")
    x, dy = torch.empty(0, 16, dtype=T, device="cuda"), torch.empty(0, 8, dtype=T, device="cuda")
    w = torch.randn(3, 8, 16, device="cuda").to(T)
    assert gcpsl.group_forward(x, o, w).shape == (0, 8) and gcpsl.group_input_grad(dy, o, w).shape == (0, 16)
    dw, db = gcpsl.group_weight_grad(dy, x, o, dw=torch.ones(3, 8, 16, device="cuda"), db=torch.ones(3, 8, device="cuda"))
    assert (dw == 0).all() and (db == 0).all()
    dw, db = gcpsl.group_weight_grad(dy, x, o, bias=False)
    assert (dw == 0).all() and db is None


@pytest.mark.parametrize("bad", [[-5, 10, 20, 30], [0, 10, 20, 99], [0, 25, 10, 30], [2 ** 31 - 1, -2 ** 31, 7, 30]])
def test_offsets_out_of_range_stay_inside_the_tensors(bad):
    """Rows next to the tensors, and inside them those of the groups whose offsets are in order, are as they should
    be."""
    rows, n, k = 30, 16, 24
    room = torch.full((rows + 40, n), 7.0, device="cuda")
    x, w = make(61, rows, k), make(62, 3, n, k)
    gcpsl.group_forward(gpu(x), torch.tensor(bad, dtype=torch.int32).cuda(), gpu(w), out=room[20:20 + rows])
    assert (room[:20] == 7).all() and (room[20 + rows:] == 7).all()
    gcpsl.group_weight_grad(make(63, rows, n).cuda(), gpu(x), torch.tensor(bad, dtype=torch.int32).cuda())


@pytest.mark.parametrize("dtype,n,k", [("bf16", 24, 64), ("f32", 24, 64), ("bf16", 24, 33)])
def test_offsets_past_32_bits(dtype, n, k):
    """Rows 4 MiB apart: byte offsets reach 9 GiB, element offsets 2^31 and more."""
    T, rows, ld = TYPES[dtype], 2300, (4 << 20) // (2 if dtype == "bf16" else 4)
    store = torch.empty(rows * ld + 64, dtype=T, device="cuda")
    xv, yv = store.as_strided((rows, k), (ld, 1), 0), store.as_strided((rows, n), (ld, 1), ld // 2)
    x, w, dy = make(71, rows, k, dtype=T), make(72, 2, n, k, dtype=T), make(73, rows, n, dtype=T)
    xv.copy_(x)
    off = [0, 1500, 2300]
    o = torch.tensor(off, dtype=torch.int32).cuda()
    gcpsl.group_forward(xv, o, gpu(w), out=yv)
    check(yv, *plain.forward(x, off, w)[:2])
    yv.copy_(dy)
    dw, db = gcpsl.group_weight_grad(yv, xv, o)
    want_w, want_b, bound_w, bound_b = plain.weight_grad(dy, x, off)
    check(dw, want_w, bound_w)
    check(db, want_b, bound_b)
    gcpsl.group_input_grad(yv, o, gpu(w), out=xv)
    check(xv, *plain.input_grad(dy, off, w)[:2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(1024, 1024), (512, 1032), (1000, 777)])
def test_wide_layers_of_many_rows(n, k, dtype):
    """Sizes of many tiles, in 64 bits on the GPU; the same bits on a second call."""
    T, counts = TYPES[dtype], [700, 0, 1400, 333, 1, 64]
    off, G = offsets_of(counts), len(counts)
    x, w = make(81, off[-1], k, dtype=T).cuda(), make(82, G, n, k, dtype=T, scale=k ** -0.5).cuda()
    dy, o = make(83, off[-1], n, dtype=T).cuda(), torch.tensor(off, dtype=torch.int32).cuda()
    y, dx = gcpsl.group_forward(x, o, w), gcpsl.group_input_grad(dy, o, w)
    dw, db = gcpsl.group_weight_grad(dy, x, o)
    for g, a, b in plain.parts(off):
        xg, wg, dg = x[a:b].double(), w[g].double(), dy[a:b].double()
        for got, left, right, size in ((y[a:b], xg, wg.T, k), (dx[a:b], dg, wg, n), (dw[g], dg.T, xg, b - a)):
            want = left @ right
            bound = (size + 8) * plain.UACC * (left.abs() @ right.abs())
            bound = plain.rounded(bound, want, got.dtype)
            assert ((got.double() - want).abs() <= bound).all()
        assert ((db[g].double() - dg.sum(0)).abs() <= (b - a + 8) * plain.UACC * dg.abs().sum(0) + 1e-37).all()
    assert torch.equal(gcpsl.group_forward(x, o, w), y) and torch.equal(gcpsl.group_input_grad(dy, o, w), dx)
    again = gcpsl.group_weight_grad(dy, x, o)
    assert torch.equal(again[0], dw) and torch.equal(again[1], db)


def test_another_stream_and_a_captured_graph():
    """Calls on a stream of their own, and replays of a captured chain with eager work between them."""
    off = [0, 100, 160]
    x, w, b = make(91, 160, 96).cuda(), make(92, 2, 80, 96).cuda(), make(93, 2, 80).cuda()
    labels = torch.randint(0, 80, (160,), dtype=torch.int32).cuda()
    o = torch.tensor(off, dtype=torch.int32).cuda()

    def chain(stream=None):
        y = gcpsl.group_forward(x, o, w, b, relu=True, p=0.25, seed=3, stream=stream)
        s = gcpsl.score(y, labels, top=3, stream=stream)
        d = gcpsl.score_grad(y, labels, s.lse, g_logp=torch.ones_like(s.logp), stream=stream)
        dw, db = gcpsl.group_weight_grad(d, x, o, stream=stream)
        return [y, *s, d, gcpsl.group_input_grad(d, o, w, gate=x, stream=stream), dw, db, gcpsl.dropout(y, 0.5, 4, stream=stream)]

    want = chain()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = chain(side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain()
    for i in range(3):
        for t in out:
            t.zero_()
        x.copy_(make(94 + i, 160, 96))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, chain())), i


def test_refusals():
    x, w = torch.zeros(6, 8, device="cuda"), torch.zeros(2, 4, 8, device="cuda")
    o = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    bad = [lambda: gcpsl.group_forward(x.cpu(), o, w), lambda: gcpsl.group_forward(x, o.long(), w),
           lambda: gcpsl.group_forward(x, o.cpu(), w), lambda: gcpsl.group_forward(x, o[:2], w),
           lambda: gcpsl.group_forward(x, o, w.bfloat16()), lambda: gcpsl.group_forward(x.half(), o, w.half()),
           lambda: gcpsl.group_forward(x.t(), o, w), lambda: gcpsl.group_forward(x[:, :7], o, w),
           lambda: gcpsl.group_forward(x, o, w.transpose(1, 2)), lambda: gcpsl.group_forward(x, o, w[:, :, ::2]),
           lambda: gcpsl.group_forward(x, o, w, bias=torch.zeros(2, 5, device="cuda")),
           lambda: gcpsl.group_forward(x, o, w, out=torch.zeros(6, 5, device="cuda")),
           lambda: gcpsl.group_input_grad(torch.zeros(6, 5, device="cuda"), o, w),
           lambda: gcpsl.group_input_grad(torch.zeros(6, 4, device="cuda"), o, w, gate=x[:5]),
           lambda: gcpsl.group_weight_grad(torch.zeros(5, 4, device="cuda"), x, o),
           lambda: gcpsl.group_weight_grad(torch.zeros(6, 4, device="cuda"), x, o, dw=torch.zeros(2, 4, 7, device="cuda"))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for p in (-0.1, 1.0, float("nan")):
        with pytest.raises(gcpsl.GCPSLError) as e:
            gcpsl.group_forward(x, o, w, p=p)
        assert e.value.code == gcpsl.EINVAL
    with pytest.raises(gcpsl.GCPSLError):  # dropout's factor needs the gate
        gcpsl.group_input_grad(torch.zeros(6, 4, device="cuda"), o, w, p=0.5)
    with pytest.raises(gcpsl.GCPSLError):  # rows of an output on top of each other
        gcpsl.group_forward(x, o, w, out=torch.zeros(4, device="cuda").expand(6, 4))
    with pytest.raises(gcpsl.GCPSLError):
        gcpsl.group_weight_grad(torch.zeros(6, 4, device="cuda"), x, o, dw=torch.zeros(4, 8, device="cuda").expand(2, 4, 8))
