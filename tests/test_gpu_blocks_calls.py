"""Ways to call gated layers, residual norms and distillation: the native call and the binding's own checks (the same
bits), streams of their own, captured graphs that are replayed, two at a time on workspaces of their own."""
import pytest
import torch

from test_gpu_group import TYPES, gpu, make, offsets_of

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


def calls(dtype, counts=(5, 0, 40, 3), n=24, k=56, L=300):
    """(name, call of the keyword arguments that choose the way) for every operator."""
    T, off = TYPES[dtype], offsets_of(counts)
    G, rows = len(counts), off[-1]
    o = torch.tensor(off, dtype=torch.int32).cuda()
    x, w, b = gpu(make(1, rows, k, dtype=T)), gpu(make(2, G, 2 * n, k, dtype=T)), gpu(make(3, G, 2 * n))
    dz, v, pre = gpu(make(4, rows, k, dtype=T)), gpu(make(5, G, k, n, dtype=T)), gpu(make(6, rows, 2 * n, dtype=T))
    y, gate, go, gh = (gpu(make(7 + i, rows, k, dtype=T)) for i in range(4))
    w1, w2 = gpu(make(11, G, k)), gpu(make(12, G, k))
    f = gcpsl.group_residual_norm(x, o, y=y, gate=gate, w_block=w1, w_next=w2, beta=0.5)
    z = gpu(make(13, rows, L, dtype=T))
    best = make(14, rows, L).topk(6, 1)
    cls, val = best.indices.int().cuda(), best.values.cuda()
    lab = torch.randint(0, L, (rows,), generator=torch.Generator().manual_seed(7), dtype=torch.int32).cuda()
    r = gcpsl.distill(z, cls, val, temperature=3.0, labels=lab)
    g = gpu(make(15, rows))
    norm_grad = dict(g_out=go, g_h=gh, y=y, gate=gate, w_block=w1, w_next=w2, r_block=f.r_block, r_next=f.r_next, beta=0.5)
    return [("gated", lambda **a: gcpsl.group_gated_forward(x, o, w, b, **a)),
            ("gated, kept", lambda **a: gcpsl.group_gated_forward(x, o, w, act="gelu", keep=True, **a)),
            ("gated gradient", lambda **a: gcpsl.group_gated_grad(dz, o, v, pre, act="relu", **a)),
            ("norm", lambda **a: gcpsl.group_residual_norm(x, o, y=y, gate=gate, w_block=w1, w_next=w2, alpha=2, **a)),
            ("norm alone", lambda **a: gcpsl.group_residual_norm(x, o, w_next=w2, **a)),
            ("residual alone", lambda **a: gcpsl.group_residual_norm(x, o, y=y, **a)),
            ("norm gradient", lambda **a: gcpsl.group_residual_norm_grad(f.out, o, **norm_grad, **a)),
            ("norm alone, gradient", lambda **a: gcpsl.group_residual_norm_grad(x, o, g_h=gh, w_next=w2, r_next=f.r_next, **a)),
            ("residual alone, gradient", lambda **a: gcpsl.group_residual_norm_grad(x, o, g_out=go, y=y, **a)),
            ("distill", lambda **a: gcpsl.distill(z, cls, val, temperature=3.0, labels=lab, **a)),
            ("distill without labels", lambda **a: gcpsl.distill(z, cls, val, **a)),
            ("distill gradient", lambda **a: gcpsl.distill_grad(z, cls, val, r.lse_t, temperature=3, labels=lab, lse=r.lse,
                                                                g_kl=g, g_logp=g, **a))]


def flat(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


def same(a, b):
    return type(a) is type(b) and len(flat(a)) == len(flat(b)) and all(
        u.dtype == v.dtype and u.shape == v.shape and torch.equal(u, v) for u, v in zip(flat(a), flat(b)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_results_both_ways(dtype):
    for name, call in calls(dtype):
        assert same(call(), call(stream=torch.cuda.current_stream())), name


# the second of enough rows that gradients are summed in pieces, rows cut into parts and products in large tiles
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [{}, {"counts": (900, 0, 400, 1), "n": 128, "k": 264, "L": 20000}])
def test_other_streams_and_replays(sizes, dtype):
    for name, call in calls(dtype, **sizes):
        want = call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        side.synchronize()
        assert same(got, want), name
        with torch.cuda.stream(side):  # the current stream another one, and the native call
            got = call()
        side.synchronize()
        assert same(got, want), name
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        held = []
        for graph in graphs:
            with torch.cuda.graph(graph):
                held.append(call())
        for _ in range(3):
            for t in (u for h in held for u in flat(h)):
                if t.data_ptr() not in {u.data_ptr() for u in flat(want)}:
                    t.fill_(3)
            eager = call()
            graphs[0].replay()
            graphs[1].replay()
            torch.cuda.synchronize()
            assert same(eager, want) and all(same(h, want) for h in held), name


def test_current_device_is_checked():
    for name, call in calls("f32"):
        assert call() is not None, name
    x, o = torch.zeros(4, 8), torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        gcpsl.group_gated_forward(x, o, torch.zeros(1, 4, 8))
    with pytest.raises(ValueError):
        gcpsl.group_residual_norm(x, o, w_next=torch.ones(1, 8))
    with pytest.raises(ValueError):
        gcpsl.distill(x, torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 1))
