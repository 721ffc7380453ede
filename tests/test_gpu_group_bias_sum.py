"""The fp32 bias gradient's summation: a large first row and ones behind it, which a sum of one value after another
loses."""
import pytest
import torch

import ops_plain as plain

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


# tiles of 128 x 128, of 64 x 64, results of fewer columns than those take
@pytest.mark.parametrize("G,rows,n,k", [(8, 1024, 1024, 1024), (1, 1024, 1024, 1024), (1, 1024, 512, 9), (2, 700, 60, 20)])
def test_eight_rows_at_a_time(G, rows, n, k):
    """2^24 + 1 is 2^24 in fp32, and 2^24 + 8 exact.  A thread adds up eight values in a tree of three levels before they
    join the sum it carries: of `rows` values it has at most rows / 8 such steps, the tree and less than nine more for
    the other threads' and pieces' sums, each off by 2^-24 of the sum of magnitudes."""
    dy = torch.ones(G * rows, n)
    dy[::rows] = 2.0 ** 24
    x = torch.zeros(G * rows, k)
    off = torch.arange(0, G * rows + 1, rows, dtype=torch.int32)
    _, db = gcpsl.group_weight_grad(dy.cuda(), x.cuda(), off.cuda())
    # one chain has half of the rows of a whole group, or all of a piece of at most 128
    steps = (rows // 2 if n * k >= 1024 * 1024 else 128) // 8 + 3 + 9
    want = 2.0 ** 24 + rows - 1
    assert ((db.cpu().double() - want).abs() <= steps * plain.U32 * want).all(), (db.cpu().double() - want).abs().max()
