"""The two ways from Python to the operators, the native call and the binding's own checks: the same bits, and the same
refusals."""
import numpy as np
import pytest
import torch

from test_gpu_group import TYPES, gpu, make, offsets_of

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


def calls(dtype):
    """(name, call of the keyword arguments that choose the way) for every operator."""
    T, off = TYPES[dtype], offsets_of([5, 0, 40, 3])
    rows, n, k, L = off[-1], 24, 56, 300
    o = torch.tensor(off, dtype=torch.int32).cuda()
    x, dy, w = gpu(make(1, rows, k, dtype=T)), gpu(make(2, rows, n, dtype=T)), gpu(make(3, 4, n, k, dtype=T))
    b, gate, z = gpu(make(4, 4, n)), gpu(make(5, rows, k, dtype=T)), gpu(make(6, rows, L, dtype=T))
    y = torch.randint(0, L, (rows,), generator=torch.Generator().manual_seed(7), dtype=torch.int32).cuda()
    s = gcpsl.score(z, y)
    g = gpu(make(8, rows))
    return [("forward", lambda **a: gcpsl.group_forward(x, o, w, b, relu=True, p=0.25, seed=3, **a)),
            ("no bias", lambda **a: gcpsl.group_forward(x[:, :-1], o, w[:, :, :-1].contiguous(), **a)),
            ("input gradient", lambda **a: gcpsl.group_input_grad(dy, o, w, gate=gate, p=0.5, **a)),
            ("weight gradient", lambda **a: gcpsl.group_weight_grad(dy, x, o, **a)),
            ("weight gradient alone", lambda **a: gcpsl.group_weight_grad(dy, x, o, bias=False, **a)),
            ("dropout", lambda **a: gcpsl.dropout(x, 0.5, 2 ** 64 - 1, **a)),
            ("score", lambda **a: gcpsl.score(z, y, top=7, **a)),
            ("score without labels", lambda **a: gcpsl.score(z, **a)),
            ("gradient", lambda **a: gcpsl.score_grad(z, y, s.lse, s.entropy, g, g, **a))]


def same(a, b):
    if a is None or b is None:
        return a is b
    if isinstance(a, tuple):
        return type(a) is type(b) and len(a) == len(b) and all(same(u, v) for u, v in zip(a, b))
    return a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_results(dtype):
    for name, call in calls(dtype):
        assert same(call(), call(stream=torch.cuda.current_stream())), name


def test_result_is_the_tensor_given():
    x = gpu(make(1, 9, 20))
    out = torch.empty_like(x)
    assert gcpsl.dropout(x, 0.5, 1, out=out) is out
    assert gcpsl.dropout(x, 0.5, 1, out=out, stream=torch.cuda.current_stream()) is out


def test_arguments_of_other_number_types():
    x = gpu(make(1, 9, 20))
    want = gcpsl.dropout(x, 0.5, 1)
    assert torch.equal(gcpsl.dropout(x, np.float64(0.5), 1), want)
    assert torch.equal(gcpsl.dropout(x, 0.5, 1 + 2 ** 64), want)  # a seed counts modulo 2^64
    assert torch.equal(gcpsl.dropout(x, 0, 1), x)


def test_results_outlive_each_other():
    z = gpu(make(1, 50, 70))
    s = gcpsl.score(z, torch.zeros(50, dtype=torch.int32, device="cuda"), top=3)
    kept, want = s.top_class, s.top_class.clone()
    del s
    for _ in range(20):
        torch.empty(50 * 9, device="cuda").fill_(float("nan"))
    assert torch.equal(kept, want) and kept.is_contiguous() and kept.dtype == torch.int32


@pytest.mark.parametrize("stream", [False, True])
def test_same_refusals(stream):
    a = {"stream": torch.cuda.current_stream()} if stream else {}
    x, o = gpu(make(1, 8, 16)), torch.tensor([0, 8], dtype=torch.int32).cuda()
    w = gpu(make(2, 1, 4, 16))
    with pytest.raises(ValueError):
        gcpsl.dropout(x.cpu(), 0.5, 1, **a)
    with pytest.raises(ValueError):
        gcpsl.dropout(x.half(), 0.5, 1, **a)
    with pytest.raises(ValueError):
        gcpsl.dropout(x.t(), 0.5, 1, **a)
    with pytest.raises(ValueError):
        gcpsl.dropout(x, 0.5, 1, out=x[:4], **a)
    with pytest.raises(ValueError):
        gcpsl.group_forward(x, o.long(), w, **a)
    with pytest.raises(ValueError):
        gcpsl.group_forward(x, o, w[:, :, :8], **a)
    with pytest.raises(ValueError):
        gcpsl.group_forward(x, o, w, torch.zeros(1, 5, device="cuda"), **a)
    with pytest.raises(ValueError):
        gcpsl.score(x, torch.zeros(7, dtype=torch.int32, device="cuda"), **a)
    for bad in (lambda: gcpsl.dropout(x, 1.0, 1, **a), lambda: gcpsl.dropout(x, float("nan"), 1, **a),
                lambda: gcpsl.score(x, top=17, **a), lambda: gcpsl.score(x, top=-1, **a),
                lambda: gcpsl.group_input_grad(gpu(make(3, 8, 4)), o, w, p=0.5, **a)):
        with pytest.raises(gcpsl.GCPSLError):
            bad()
