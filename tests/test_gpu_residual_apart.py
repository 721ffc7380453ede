"""Residual norms of rows that no workgroup holds in registers (here rows of less than a vector), more of them than
workgroups, and with rows outside the groups between those that a workgroup takes."""
import pytest
import torch

import blocks_plain as blocks
from test_gpu_group import TYPES, check, gpu, make

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402


# offsets that decrease leave rows out between others: which rows are then written is not specified, but those that are
# hold the definition's values
@pytest.mark.parametrize("offsets", [[0, 3000, 3000, 6144], [1000, 5000, 5001, 6000], [4096, 6144, 0, 2048]])
@pytest.mark.parametrize("dtype,n", [("f32", 1), ("f32", 3), ("bf16", 7)])
@pytest.mark.parametrize("block", [False, True])
def test_rows_in_turn(block, dtype, n, offsets):
    T, rows, G = TYPES[dtype], 6144, 3
    x, y = make(1, rows, n, dtype=T), make(2, rows, n, dtype=T)
    w = (1 + make(3, 1, n, scale=0.3)).repeat(G, 1)  # (the same in every group)
    o = torch.tensor(offsets, dtype=torch.int32).cuda()
    r = torch.full((rows, n), 768.0, dtype=T, device="cuda")
    if block:
        gcpsl.group_residual_norm(gpu(x), o, y=gpu(y), w_block=gpu(w), beta=0.5, eps=1e-5, out=r)
        want, bound = blocks.residual(x, [0, rows], y, w_block=w[:1], beta=0.5, eps=1e-5)[0]["out"]
    else:
        gcpsl.group_residual_norm(gpu(x), o, w_next=gpu(w), eps=1e-5, h=r)
        want, bound = blocks.residual(x, [0, rows], w_next=w[:1], eps=1e-5)[0]["h"]
    r = r.cpu()
    written = (r != 768.0).any(1)
    if offsets == sorted(offsets):
        assert torch.equal(written.nonzero()[:, 0], torch.arange(offsets[0], offsets[-1]))
    check(r[written], want[written], bound[written])
