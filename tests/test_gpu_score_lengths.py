"""Label scores at the lengths where rows change hands: one lane group, one wave, four waves with more and more vectors a
thread, several chunks; with few rows and with many (tests/ops_plain.py's bounds)."""
import pytest
import torch

from test_gpu_score import check, make

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

EDGES = [64, 256, 512, 1024, 2048, 4096, 8192, 16384]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", sorted(e + d for e in EDGES for d in (-1, 0, 1)))
def test_few_rows_and_many(L, dtype):
    """Many rows are few ones over and over: every copy has the first one's bits, which are right."""
    z, labels = make(6, L, dtype)
    z[4, ::3] = float("-inf")
    z[5] = z[5, 0]  # one value throughout: the lowest classes come first
    for top in (5, 32):
        check(z, labels, top)
        for copies in (100, 200):  # 600 and 1,200 rows
            r = gcpsl.score(z.cuda().repeat(copies, 1), labels.cuda().repeat(copies), top=top)
            first = type(r)(*(v[:6] for v in r))
            check(z, labels, top, r=first)
            for v, f in zip(r, first):
                assert torch.equal(v.view(copies, *f.shape), f.expand(copies, *f.shape))
