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
    join the sum it carries, so that what can be lost is less than one unit a level of the tree, a step of the chain
    (taken as that of 512 rows in whole groups and of 128 in pieces) and one of at most nine additions of
    threads' and pieces' sums."""
    dy = torch.ones(G * rows, n)
    dy[::rows] = 2.0 ** 24
    x = torch.zeros(G * rows, k)
    off = torch.arange(0, G * rows + 1, rows, dtype=torch.int32)
    _, db = gcpsl.group_weight_grad(dy.cuda(), x.cuda(), off.cuda())
    steps = (rows // 2 if n * k >= 1024 * 1024 else 128) // 8 + 3 + 9
    want = 2.0 ** 24 + rows - 1
    assert ((db.cpu().double() - want).abs() <= steps * plain.U32 * want).all(), (db.cpu().double() - want).abs().max()
