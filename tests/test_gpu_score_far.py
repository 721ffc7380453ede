"""Label scores far from zero: finite fills and maxima whose size in units of log 2 fp32 cannot hold to within an
exponent's range, over whole rows and over stretches that a wave or a chunk has to itself (tests/ops_plain.py)."""
import numpy as np
import pytest
import torch

import ops_plain as plain
from test_gpu_score import TYPES, check, make, same

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

FAR = (1e6, 1e9, 3.01e9, 1e10, 1e12, 1e20, 1e30)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [10, 65, 130, 2500, 33000, 131072])
def test_stretches(L, dtype):
    """Classes ruled out by a finite fill, all but one of them among the rows; and a stretch, or one class, far above."""
    parts = [(slice(0, L // 2), -1), (slice(L // 2, L), -1), (slice(L // 4, 3 * L // 4), -1), (slice(0, L - 1), -1),
             (slice(1, L), -1), (slice(L // 4, L // 2), 1), (slice(L // 3, L // 3 + 1), 1)]
    z, labels = make(len(parts) * len(FAR), L, dtype, seed=11)
    for i in range(z.shape[0]):
        part, sign = parts[i % len(parts)]
        z[i, part] = sign * FAR[i // len(parts)]
    labels[::2] = 0
    check(z, labels, min(L, 20))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [10, 65, 130, 2500, 33000, 131072])
def test_uniform_rows(L, dtype):
    """One value throughout: log probabilities of -log L and an entropy of log L, within bounds that do not grow with the
    value, as x - max is exact."""
    values = [s * f for f in FAR for s in (1, -1)]
    z = torch.tensor(values)[:, None].expand(-1, L).to(TYPES[dtype]).contiguous()
    labels = torch.full((len(values),), L - 1, dtype=torch.int32)
    top = min(L, 5)
    r = gcpsl.score(z.cuda(), labels.cuda(), top=top)
    log = np.log(L)
    bound = torch.tensor((8 + L / 64 + 32 + 4 * (log + 1)) * plain.U32)
    same(r.logp, torch.full((len(values),), -log, dtype=torch.float64), bound)
    same(r.entropy, torch.full((len(values),), log, dtype=torch.float64), bound)
    same(r.lse, z[:, 0].double() + log, bound + 2 * plain.U32 * z[:, 0].double().abs())
    same(r.top_logp, torch.full((len(values), top), -log, dtype=torch.float64), bound)
    assert torch.equal(r.top_class.cpu(), torch.arange(top, dtype=torch.int32).expand(len(values), top))
