"""Tensors that require a gradient are taken as plain ones by the operators on tensors: the same bits, and results that
require none, by the native call and by the binding's own checks."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


@pytest.mark.parametrize("stream", [False, True])
def test_results_require_no_gradient(stream):
    a = {"stream": torch.cuda.current_stream()} if stream else {}
    g = torch.Generator().manual_seed(3)
    x, w, b = (torch.randn(s, generator=g).cuda().requires_grad_() for s in ((9, 16), (1, 12, 16), (1, 12)))
    o = torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    labels = torch.zeros(9, dtype=torch.int32, device="cuda")

    def chain(x, w, b):
        y = gcpsl.group_forward(x, o, w, b, relu=True, **a)
        s = gcpsl.score(x, labels, top=2, **a)
        d = gcpsl.score_grad(x, labels, s.lse, g_logp=s.logp, **a)
        return [y, *s, d, gcpsl.group_input_grad(y, o, w, gate=x, **a), *gcpsl.group_weight_grad(y, x, o, **a),
                gcpsl.dropout(x, 0.5, 4, **a)]

    got, want = chain(x, w, b), chain(x.detach(), w.detach(), b.detach())
    assert not any(t.requires_grad for t in got)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
