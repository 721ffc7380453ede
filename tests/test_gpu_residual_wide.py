"""Residual norms' gradients of the widest rows, and of as many groups' columns, that their documentation allows."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


# (groups, columns): 2^28 columns and just over 2^28 columns of all groups together
@pytest.mark.parametrize("G,n", [(1, 2 ** 28), (1024, 2 ** 18 + 264)])
def test_many_columns(G, n):
    """The norm alone, x' = x r w: with every |x| = 2 and eps = 0.25, r = 4.25^-1/2, and by the formula, as the products
    g_h x sum to 0 over a row, dx = r g_h and dw = g_h x r."""
    x = torch.full((2, n), 2.0, dtype=torch.bfloat16, device="cuda")
    x[:, 1::2] = -2
    gh = torch.ones_like(x)
    o = torch.full((G + 1,), 2, dtype=torch.int32, device="cuda")
    o[0], o[1:G] = 0, 1  # a row for the first group and one for the last (both for a single one)
    w = torch.ones(1, n, device="cuda").expand(G, -1)
    r = torch.full((2,), 4.25 ** -0.5, device="cuda")
    res = gcpsl.group_residual_norm_grad(x, o, g_h=gh, w_next=w, r_next=r)
    # dx in bf16: half a step; dw: the fp32 products' roundings
    assert ((res.dx.float() - r[0]).abs() <= r[0] * 2.0 ** -8).all()
    for g, rows in ((0, 1 if G > 1 else 2), (G - 1, 1 if G > 1 else 2)):
        assert ((res.dw_next[g] - rows * r[0] * x[0].float()).abs() <= 8 * 2.0 ** -24 * rows).all()
    assert G == 1 or (res.dw_next[1:G - 1] == 0).all()
