"""Gated layers over rows grouped by cluster, on the GPU, against their 64-bit definition (tests/blocks_plain.py)."""
import pytest
import torch

import blocks_plain as blocks
import ops_plain as plain
from test_gpu_group import SHAPES, TYPES, check, gpu, make, offsets_of

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

ACTS = ["silu", "gelu", "relu"]


def inputs(seed, counts, n, k, T, m=None):
    off, G = offsets_of(counts), len(counts)
    rows = off[-1]
    x, w = make(seed, rows, k, dtype=T), make(seed + 1, G, 2 * n, k, dtype=T, scale=k ** -0.5)
    b = make(seed + 2, G, 2 * n, scale=0.3)
    m = k if m is None else m
    dz, v = make(seed + 3, rows, m, dtype=T), make(seed + 4, G, m, n, dtype=T, scale=m ** -0.5)
    return off, torch.tensor(off, dtype=torch.int32).cuda(), x, w, b, dz, v, make(seed + 5, rows, 2 * n, dtype=T, scale=2.0)


def check_both(off, o, x, w, b, dz, v, pre, act):
    got = gcpsl.group_gated_forward(gpu(x), o, gpu(w), gpu(b), act=act, keep=True)
    y, ey, p, ep, _ = blocks.gated_forward(x, off, w, b, act)
    assert got.y.dtype == x.dtype and got.pre.dtype == x.dtype
    check(got.y, y, ey, "forward")
    check(got.pre, p, ep, "pairs")
    alone = gcpsl.group_gated_forward(gpu(x), o, gpu(w), gpu(b), act=act)
    assert alone.pre is None and torch.equal(alone.y, got.y)
    d = gcpsl.group_gated_grad(gpu(dz), o, gpu(v), gpu(pre), act=act)
    check(d, *blocks.gated_grad(dz, off, v, pre, act)[:2], "gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_both_directions(i, dtype):
    counts, n, k = SHAPES[i]
    check_both(*inputs(200, counts, n, k, TYPES[dtype]), ACTS[i % 3])


# more rows: tiles of every size, whole and cut ones, groups of none and of one row beside long ones
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("counts,n,k,m", [([700, 0, 1, 1300], 264, 136, 200), ([2048], 256, 128, 64), ([37, 900], 129, 67, 131),
                                          ([16] * 16, 512, 256, 256)])
def test_larger(counts, n, k, m, act, dtype):
    check_both(*inputs(300, counts, n, k, TYPES[dtype], m), act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,n,k,m", [([3000, 1096, 4], 1024, 64, 64), ([8192], 512, 72, 40)])
def test_many_tiles(counts, n, k, m, dtype):
    """As many tiles as make the largest ones worth while."""
    check_both(*inputs(350, counts, n, k, TYPES[dtype], m), "silu")


@pytest.mark.parametrize("k", [1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 64, 65, 95, 96, 97])
def test_sums_shared_by_two_teams(k):
    """Fewer tiles than compute units, whose k tiles two teams of waves take in turn: sums that end in either's."""
    check_both(*inputs(370, [700, 0, 1, 1300], 600, k, torch.float32), ACTS[k % 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rest", range(8))
@pytest.mark.parametrize("counts,n,k", [([5, 0, 70], 128, 64), ([200, 131], 72, 136), ([129], 8, 200)])
def test_every_remainder_of_the_vectors(counts, n, k, rest, dtype):
    """Widths that leave every number of elements past a 16-byte piece, next to values that must not be read."""
    T, G = TYPES[dtype], len(counts)
    off, o, x, w, b, dz, v, pre = inputs(400, counts, n + rest, k + rest, T)
    n, k, rows = n + rest, k + rest, off[-1]
    wide = {name: torch.full((rows + 1, c + 5), float("nan"), dtype=T, device="cuda")
            for name, c in (("x", k), ("dz", k), ("pre", 2 * n), ("y", n), ("kept", 2 * n), ("d", 2 * n))}
    view = {name: t[:rows, :t.shape[1] - 5] for name, t in wide.items()}
    for name, t in (("x", x), ("dz", dz), ("pre", pre)):
        view[name].copy_(t)
    got = gcpsl.group_gated_forward(view["x"], o, gpu(w), out=view["y"], pre=view["kept"])
    assert got.y is view["y"] and got.pre is view["kept"]
    y, ey, p, ep, _ = blocks.gated_forward(x, off, w)
    check(got.y, y, ey, "forward")
    check(got.pre, p, ep, "pairs")
    gcpsl.group_gated_grad(view["dz"], o, gpu(v), view["pre"], out=view["d"])
    check(view["d"], *blocks.gated_grad(dz, off, v, pre)[:2], "gradient")
    for name, t in wide.items():  # nothing beside the tensors is written
        assert torch.isnan(t[rows]).all() and torch.isnan(t[:, -5:]).all(), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(40, 24), (264, 136)])
def test_rows_outside_the_groups_stay(n, k, dtype):
    T, off = TYPES[dtype], [7, 40, 40, 300]
    rows = 350
    x, w = make(1, rows, k, dtype=T), make(2, 3, 2 * n, k, dtype=T, scale=k ** -0.5)
    dz, v, pre = make(3, rows, k, dtype=T), make(4, 3, k, n, dtype=T), make(5, rows, 2 * n, dtype=T)
    o = torch.tensor(off, dtype=torch.int32).cuda()
    y, p, d = (torch.full((rows, c), 7.0, dtype=T, device="cuda") for c in (n, 2 * n, 2 * n))
    gcpsl.group_gated_forward(gpu(x), o, gpu(w), out=y, pre=p)
    gcpsl.group_gated_grad(gpu(dz), o, gpu(v), gpu(pre), out=d)
    wy, ey, wp, ep, written = blocks.gated_forward(x, off, w)
    for got, want, bound in ((y, wy, ey), (p, wp, ep), (d, *blocks.gated_grad(dz, off, v, pre)[:2])):
        check(got[off[0]:off[-1]], want[off[0]:off[-1]], bound[off[0]:off[-1]])
        assert (got[~written.cuda()] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_far_gates(act, dtype):
    """Gates from deep in the saturated range, through 0, in a layer whose product is exact: x one-hot, w the values."""
    T = TYPES[dtype]
    far = torch.tensor([-2e4, -300.0, -100.0, -88.0, -40.0, -12.0, -3.0, -0.5, -1e-3, 0.0, 1e-3, 0.5, 3.0, 12.0, 40.0,
                        100.0, 300.0, 2e4]).to(T)
    n = far.numel()
    w = torch.cat((far, make(1, n, dtype=T)))[None, :, None].contiguous()
    x = torch.ones(5, 1, dtype=T)
    o = torch.tensor([0, 5], dtype=torch.int32).cuda()
    got = gcpsl.group_gated_forward(gpu(x), o, gpu(w), act=act, keep=True)
    y, ey, p, _, _ = blocks.gated_forward(x, [0, 5], w, None, act)
    check(got.y, y, ey)
    assert torch.equal(got.pre.cpu().double(), p)
    dz, v = make(2, 5, 1, dtype=T), torch.ones(1, 1, n, dtype=T)
    check(gcpsl.group_gated_grad(gpu(dz), o, gpu(v), got.pre, act=act),
          *blocks.gated_grad(dz, [0, 5], v, got.pre.cpu(), act)[:2])


@pytest.mark.parametrize("act", ACTS)
def test_nans_stay_in_their_rows(act):
    off, o, x, w, b, dz, v, pre = inputs(500, [40, 30], 136, 72, torch.bfloat16)
    x[3, 5] = float("nan")
    y = gcpsl.group_gated_forward(gpu(x), o, gpu(w), gpu(b), act=act).y
    assert torch.isnan(y[3]).all() and not torch.isnan(y[[i for i in range(70) if i != 3]]).any()
    pre[9, 17] = float("nan")  # a gate: of its own pair only
    d = torch.isnan(gcpsl.group_gated_grad(gpu(dz), o, gpu(v), gpu(pre), act=act)).nonzero().tolist()
    assert d == [[9, 17], [9, 136 + 17]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,n,k", [([5, 0, 70], 130, 67), ([700, 0, 1, 1300], 264, 131), ([16] * 16, 72, 501),
                                        ([700, 0, 1, 1300], 600, 67), ([3], 10, 3), ([1, 1], 300, 258)])
def test_infinities_at_the_products_end(counts, n, k, dtype):
    """An infinite value in the last column makes its row's sums infinite, an infinite weight its column's: none is NaN."""
    off, o, x, w, b, dz, v, pre = inputs(550, counts, n, k, TYPES[dtype])
    x[0, k - 1] = float("inf")
    w[-1, 1, k - 1] = -float("inf")
    p = gcpsl.group_gated_forward(gpu(x), o, gpu(w), keep=True).pre.cpu()
    want = torch.zeros(p.shape, dtype=torch.bool)
    want[0] = want[off[-2]:off[-1], 1] = True
    assert not torch.isnan(p).any() and torch.equal(torch.isinf(p), want)
    dz[0, k - 1] = float("inf")
    d = gcpsl.group_gated_grad(gpu(dz), o, gpu(v), gpu(pre), act="silu").cpu()
    assert torch.equal(torch.isinf(d).nonzero()[:, 0].unique(), torch.tensor([0])) and not torch.isnan(d).any()
    assert torch.isinf(d[0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shared_weights(dtype):
    """A group stride of 0: every group the same weights; their gradient is the groups' sum."""
    T, counts, n, k = TYPES[dtype], [30, 0, 41], 24, 40
    off, o, x, w, b, dz, v, pre = inputs(600, counts, n, k, T)
    one, many = w[:1].expand(3, -1, -1), w[:1].repeat(3, 1, 1)
    got = gcpsl.group_gated_forward(gpu(x), o, gpu(w[:1]).expand(3, -1, -1), gpu(b[:1]).expand(3, -1))
    y, ey, *_ = blocks.gated_forward(x, off, many, b[:1].repeat(3, 1))
    check(got.y, y, ey)
    assert one.stride(0) == 0
    d = gcpsl.group_gated_grad(gpu(dz), o, gpu(v[:1]).expand(3, -1, -1), gpu(pre))
    check(d, *blocks.gated_grad(dz, off, v[:1].repeat(3, 1, 1), pre)[:2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_against_differences(dtype):
    """A whole backward pass, pairs to weights, against central differences of the 64-bit forward pass."""
    T, counts, n, k, m = TYPES[dtype], [9, 0, 20], 40, 24, 16
    off, o, x, w, b, dz, v, _ = inputs(700, counts, n, k, T, m)

    def loss(x, w, b):
        pre = plain.forward(x, off, w, b)[0]
        y = blocks.act(pre[:, :n], "silu")[0] * pre[:, n:]
        return float((plain.forward(y, off, v.double())[0] * dz.double()).sum())

    kept = gcpsl.group_gated_forward(gpu(x), o, gpu(w), gpu(b), keep=True)
    dpre = gcpsl.group_gated_grad(gpu(dz), o, gpu(v), kept.pre)
    dx = gcpsl.group_input_grad(dpre, o, gpu(w)).cpu().double()
    dw, db = (t.cpu().double() for t in gcpsl.group_weight_grad(dpre, gpu(x), o))
    at = [t.double() for t in (x, w, b)]
    for i, grad in enumerate((dx, dw, db)):
        u = torch.randn(at[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
        h = 1e-5  # the differences themselves are off by about h^2
        ends = [loss(*(t + s * h * u if j == i else t for j, t in enumerate(at))) for s in (1, -1)]
        want = (ends[0] - ends[1]) / (2 * h)
        # roundings of pre, dpre and the gradients, of either sign, next to the sum's magnitude
        eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
        assert abs(float((grad * u).sum()) - want) <= 4 * eps * float((grad * u).abs().sum()) + 1e-6


def test_refusals():
    x, o = gpu(make(1, 8, 16)), torch.tensor([0, 8], dtype=torch.int32).cuda()
    w, v = gpu(make(2, 1, 12, 16)), gpu(make(3, 1, 16, 6))
    pre = gpu(make(4, 8, 12))
    for a in ({}, {"stream": torch.cuda.current_stream()}):
        for bad in (lambda: gcpsl.group_gated_forward(x, o, w[:, :11].contiguous(), **a),
                    lambda: gcpsl.group_gated_forward(x, o, w, act="tanh", **a),
                    lambda: gcpsl.group_gated_forward(x, o, w, act=0, **a),
                    lambda: gcpsl.group_gated_forward(x, o, w, torch.zeros(1, 6, device="cuda"), **a),
                    lambda: gcpsl.group_gated_forward(x.half(), o, w, **a),
                    lambda: gcpsl.group_gated_forward(x, o, w, pre=torch.zeros(8, 6, device="cuda"), **a),
                    lambda: gcpsl.group_gated_forward(x, o.long(), w, **a),
                    lambda: gcpsl.group_gated_grad(x, o, v, pre[:, :6], **a),
                    lambda: gcpsl.group_gated_grad(x, o, v, pre, act="swish", **a),
                    lambda: gcpsl.group_gated_grad(x, o, v.bfloat16(), pre, **a)):
            with pytest.raises(ValueError):
                bad()
