"""More rows than one launch has room for: 2^24 - 1 workgroups of 256 threads.  Rows are one row's memory where they are
only read (row stride 0), so that each has the same bits."""
import pytest
import torch

import ops_plain as plain

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

FULL = 2 ** 24 - 1


# a workgroup a row in one and in two chunks' kernels (and their join), a wave a row, sixteen rows a workgroup
@pytest.mark.parametrize("rows,L,dtype", [(FULL + 1, 2049, "f32"), (FULL + 9, 4200, "bf16"), (4 * FULL + 12, 65, "bf16"),
                                          (FULL // 2 + 5, 17000, "f32"), (16 * FULL + 35, 3, "f32")])
def test_scores(rows, L, dtype):
    g = torch.Generator().manual_seed(L)
    one = torch.randn(1, L, generator=g).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    z = one.cuda().expand(rows, L)
    labels = torch.full((rows,), L - 1, dtype=torch.int32, device="cuda")
    top = 1 if rows < 4 * FULL else 0
    r = gcpsl.score(z, labels, top=top)
    first = plain.score(one, labels[:1].cpu(), max(top, 1))
    bl, bh = plain.score_bounds(one)
    for got, want, bound in ((r.logp, first[0], 2 * bl), (r.entropy, first[1], bh), (r.lse, first[2], bl)):
        assert abs(got[0].item() - want.item()) <= bound.item()
        assert torch.equal(got, got[:1].expand(rows))
    if top:
        assert (r.top_class == first[4].cuda()).all() and (r.top_logp == r.top_logp[0, 0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,L", [(FULL + 4, 10), (FULL + 1, 130)])
def test_gradient(rows, L, dtype):
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(L)
    one, v = torch.randn(1, L, generator=g).to(T).cuda(), torch.randn(2, 1, generator=g).cuda()
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    r = gcpsl.score(one, labels[:1])
    want = gcpsl.score_grad(one, labels[:1], r.lse, r.entropy, v[0], v[1])
    many = [t.expand(rows).contiguous() for t in (r.lse, r.entropy, v[0], v[1])]
    out = torch.full((rows, L), float("nan"), dtype=T, device="cuda")
    gcpsl.score_grad(one.expand(rows, L), labels, *many, out=out)
    assert torch.equal(out, want.expand(rows, L))
