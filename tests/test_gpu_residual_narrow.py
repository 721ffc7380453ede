"""Residual norms of rows that share a wave with others, in many groups and row counts that leave the last wave partly
filled: every row of a group is written, whichever lanes hold its group's bounds, and no other row."""
import pytest
import torch

import blocks_plain as blocks
from test_gpu_group import TYPES, check, gpu, make, offsets_of

pytestmark = pytest.mark.gpu

from paper_2609_29395_amd import gcpsl  # noqa: E402

UNTOUCHED = 768.0  # exact in either type


def layouts(G):
    """(rows of each group, rows before the first, rows behind the last): one row a group, every remainder of the rows
    modulo 4, every second group without rows, two rows a group, rows outside."""
    yield [1] * G, 0, 0
    for more in (1, 2, 3):
        yield [1] * (G - 1) + [1 + more], 0, 0
    yield [(G - i) % 2 for i in range(G)], 0, 0  # (the last one has a row)
    yield [2] * (G - 1) + [1], 0, 0
    yield [1] * G, 3, 2


def forward(t, offsets, G, alpha, beta, eps):
    """The C entry, so that the reciprocal root mean squares, too, are written into memory that is known before."""
    x, rows, n = t["x"], *t["x"].shape
    made = {"out": torch.empty_like(x), "h": torch.empty_like(x), "r_block": torch.empty(rows, device="cuda"),
            "r_next": torch.empty(rows, device="cuda")}
    for v in made.values():
        v.fill_(UNTOUCHED)
    p = {k: v.data_ptr() for k, v in {**t, **made}.items()}
    block = "y" in t
    rc = gcpsl.lib().gcpsl_group_residual_norm(
        gcpsl.DTYPES["bf16" if x.dtype == torch.bfloat16 else "f32"], G, rows, n, offsets.data_ptr(), p["x"], n, p.get("y"),
        n, p.get("gate"), n, p.get("w_block"), n, p["w_next"], n, alpha, beta, eps, p["out"] if block else None, n, p["h"], n,
        p["r_block"] if block else None, p["r_next"], torch.cuda.current_stream().cuda_stream)
    assert rc == gcpsl.OK
    return made


@pytest.mark.parametrize("G", [16, 17, 32, 33, 48, 49, 64, 65, 130])
@pytest.mark.parametrize("n", [8, 40, 64, 96, 128, 200, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_row_of_many_groups(dtype, n, G):
    T = TYPES[dtype]
    w1, w2 = (1 + make(seed, G, n, scale=0.3) for seed in (1, 2))
    for counts, before, behind in layouts(G):
        off = offsets_of(counts, before)
        rows = off[-1] + behind
        t = {"x": make(3, rows, n, dtype=T, scale=2.0), "y": make(4, rows, n, dtype=T, scale=3.0),
             "gate": make(5, rows, n, dtype=T, scale=2.0), "w_block": w1, "w_next": w2}
        o = torch.tensor(off, dtype=torch.int32).cuda()
        for names in (list(t), ["x", "w_next"]):
            given = {k: t[k] for k in names}
            alpha, beta, eps = (0.75, -1.25, 1e-5) if "y" in given else (1.0, 1.0, 1e-5)
            got = forward({k: gpu(v) for k, v in given.items()}, o, G, alpha, beta, eps)
            want, written = blocks.residual(given["x"], off, *(given.get(k) for k in ("y", "gate", "w_block", "w_next")), alpha,
                                            beta, eps)
            what = (counts[-1], before, len(names))
            for k, v in got.items():
                v = v.cpu()
                if k in want:
                    check(v[written], want[k][0][written], want[k][1][written], (k, *what))
                    assert (v[~written] == UNTOUCHED).all(), (k, *what)
                else:
                    assert (v == UNTOUCHED).all(), (k, *what)


@pytest.mark.parametrize("n", [8, 96, 136])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_after_others_outside(dtype, n):
    """Rows enough that a workgroup takes its share in turns: a wave whose first rows are in no group finds the groups of
    its later ones."""
    counts, before, behind = [40] * 130 + [64_000], 3, 2
    off, T, G = offsets_of(counts, before), TYPES[dtype], len(counts)
    t = {"x": make(3, off[-1] + behind, n, dtype=T), "w_next": 1 + make(1, G, n, scale=0.3)}
    got = forward({k: gpu(v) for k, v in t.items()}, torch.tensor(off, dtype=torch.int32).cuda(), G, 1.0, 1.0, 1e-5)
    want, written = blocks.residual(t["x"], off, w_next=t["w_next"], eps=1e-5)
    for k in ("h", "r_next"):
        v = got[k].cpu()
        check(v[written], want[k][0][written], want[k][1][written], k)
        assert (v[~written] == UNTOUCHED).all(), k
