"""Host-side checks of the operators on caller-owned tensors (no GPU needed): bad arguments are refused with the
documented codes before anything touches the device, calls without rows do nothing, and the 64-bit definitions that
the GPU tests use agree with torch's own where it has them."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import ops_plain as plain

g = pytest.importorskip("paper_2609_29395_amd.gcpsl")

built = pytest.mark.skipif(not os.path.exists(g.LIB_PATH), reason="libgcpsl.so not built")

FAR = 1 << 20  # an aligned address that no refused call may read
MIN32, MAX = 1 << 31, 1 << 40


def call(name, good, **change):
    args = dict(good)
    for key in change:
        assert key in args
    args.update(change)
    return getattr(g.lib(), name)(*args.values())


FORWARD = dict(dtype=0, G=2, rows=5, n=3, k=4, offsets=FAR, x=FAR, ldx=4, w=FAR, w_gs=12, bias=FAR, bias_gs=3, relu=1,
               p=0.5, seed=1, y=FAR, ldy=3, stream=None)
INPUT = dict(dtype=0, G=2, rows=5, n=3, k=4, offsets=FAR, dy=FAR, lddy=3, w=FAR, w_gs=12, gate=FAR, ldgate=4, p=0.5,
             dx=FAR, lddx=4, stream=None)
WEIGHT = dict(dtype=1, G=2, rows=5, n=3, k=4, offsets=FAR, dy=FAR, lddy=3, x=FAR, ldx=4, dw=FAR, dw_gs=12, db=FAR,
              db_gs=3, workspace=None, workspace_bytes=0, stream=None)
DROPOUT = dict(dtype=0, rows=5, cols=4, x=FAR, ldx=4, p=0.5, seed=1, y=FAR, ldy=4, stream=None)
SCORE = dict(dtype=0, rows=5, L=7, z=FAR, ldz=7, labels=FAR, top=2, logp=FAR, entropy=FAR, lse=FAR, top_logp=FAR,
             top_class=FAR, workspace=FAR, workspace_bytes=1 << 30, stream=None)
GRAD = dict(dtype=0, rows=5, L=7, z=FAR, ldz=7, labels=FAR, lse=FAR, entropy=FAR, g_logp=FAR, g_entropy=FAR, dz=FAR,
            lddz=7, stream=None)
GROUPS = [dict(dtype=2), dict(dtype=-1), dict(G=0), dict(G=1025), dict(rows=-1), dict(rows=MIN32), dict(n=0), dict(k=0), dict(n=2 ** 28 + 1),
          dict(offsets=None), dict(offsets=FAR + 2)]


@built
@pytest.mark.parametrize("name,good,bad", [
    ("gcpsl_group_forward", FORWARD, GROUPS + [
        dict(x=None), dict(x=FAR + 2), dict(ldx=-1), dict(ldx=MIN32), dict(w=None), dict(w=FAR + 1), dict(w_gs=-1),
        dict(w_gs=MAX + 1), dict(bias=FAR + 2), dict(bias_gs=-1), dict(y=None), dict(ldy=2), dict(ldy=-3),
        dict(p=1.0), dict(p=-0.25), dict(p=float("nan"))]),
    ("gcpsl_group_input_grad", INPUT, GROUPS + [
        dict(dy=None), dict(lddy=-1), dict(w=None), dict(w_gs=-1), dict(gate=FAR + 2), dict(ldgate=-1), dict(gate=None),
        dict(dx=None), dict(lddx=3), dict(p=2.0)]),
    ("gcpsl_group_weight_grad", WEIGHT, GROUPS + [
        dict(dy=None), dict(x=None), dict(x=FAR + 1), dict(lddy=-1), dict(ldx=MIN32), dict(dw=None), dict(dw=FAR + 2),
        dict(db=FAR + 1), dict(dw_gs=11), dict(db_gs=2), dict(dw_gs=-1)]),
    ("gcpsl_dropout", DROPOUT, [
        dict(dtype=3), dict(rows=-1), dict(cols=-1), dict(rows=MIN32), dict(x=None), dict(x=FAR + 2), dict(y=None),
        dict(ldx=-1), dict(ldy=3), dict(p=1.0), dict(ldx=5)]),  # the last in place with unequal strides
    ("gcpsl_score", SCORE, [
        dict(dtype=2), dict(rows=-1), dict(L=0), dict(L=2 ** 28 + 1), dict(z=None), dict(z=FAR + 2), dict(ldz=-1), dict(top=-1), dict(top=8),
        dict(labels=None), dict(top_logp=None), dict(top_class=None), dict(lse=FAR + 2)]),
    ("gcpsl_score_grad", GRAD, [
        dict(dtype=2), dict(rows=-1), dict(L=0), dict(z=None), dict(dz=None), dict(lddz=6), dict(ldz=8), dict(lse=None),
        dict(labels=None), dict(entropy=None), dict(g_logp=None, g_entropy=None), dict(g_logp=FAR + 1)]),
])
def test_bad_arguments_are_refused(name, good, bad):
    for change in bad:
        assert call(name, good, **change) == g.EINVAL, change
        assert g.lib().gcpsl_last_error(), change


@built
def test_too_many_workgroups_are_refused():
    assert call("gcpsl_group_forward", FORWARD, rows=2 ** 31 - 1, n=2 ** 28, k=1, ldy=2 ** 31 - 1) == g.EUNSUPPORTED


@built
def test_no_rows_need_no_tensors():
    assert call("gcpsl_group_forward", FORWARD, rows=0, x=None, y=None) == g.OK
    assert call("gcpsl_group_input_grad", INPUT, rows=0, dy=None, gate=None, p=0.0, dx=None) == g.OK
    assert call("gcpsl_dropout", DROPOUT, rows=0, x=None, y=None) == g.OK
    assert call("gcpsl_dropout", DROPOUT, cols=0, x=None, y=None) == g.OK
    assert call("gcpsl_score", SCORE, rows=0, z=None, labels=None, logp=None, top_logp=None, top_class=None) == g.OK
    assert call("gcpsl_score_grad", GRAD, rows=0, z=None, dz=None, lse=None, g_logp=None, g_entropy=None) == g.OK


@built
def test_workspaces():
    n = C.c_size_t(1)
    assert g.lib().gcpsl_group_workspace_bytes(0, 2, 0, 3, 4, C.byref(n)) == g.OK and n.value == 0
    assert g.lib().gcpsl_group_workspace_bytes(0, 2, 0, 3, 4, None) == g.EINVAL
    assert g.lib().gcpsl_group_workspace_bytes(0, 0, 0, 3, 4, C.byref(n)) == g.EINVAL
    assert g.lib().gcpsl_score_workspace_bytes(0, 1, 10, 11, C.byref(n)) == g.EINVAL
    assert g.lib().gcpsl_score_workspace_bytes(0, 1, 10, 2, None) == g.EINVAL
    # long sums of few outputs are taken in pieces, and a call without room for them is refused
    need = g.group_workspace_bytes("bf16", 2, 100000, 3, 4)
    assert need > 0
    assert call("gcpsl_group_weight_grad", WEIGHT, rows=100000, workspace=FAR, workspace_bytes=need - 1) == g.EINVAL
    assert call("gcpsl_group_weight_grad", WEIGHT, rows=100000, workspace=None, workspace_bytes=need) == g.EINVAL
    assert call("gcpsl_group_weight_grad", WEIGHT, rows=100000, workspace=FAR + 4, workspace_bytes=need) == g.EINVAL


def test_draws_are_splitmix64s_outputs():
    """The published first outputs for seed 1234567 (tests/golden) through the same finaliser and increment."""
    from conftest import load_golden
    gold = [v for v in load_golden("splitmix64_seed1234567.txt").values()]
    want = [v for row in gold for v in row if v > 2 ** 32]
    state = np.uint64(1234567)
    with np.errstate(over="ignore"):
        got = [int(plain.mix64(state + np.uint64(i + 1) * np.uint64(0x9E3779B97F4A7C15))) for i in range(len(want))]
    assert want and got == want


def test_plain_definitions_against_autograd():
    t = torch.Generator().manual_seed(5)
    z = torch.randn(6, 11, generator=t, dtype=torch.float64, requires_grad=True)
    labels = torch.randint(0, 11, (6,), generator=t).int()
    gl, gh = torch.randn(6, generator=t, dtype=torch.float64), torch.randn(6, generator=t, dtype=torch.float64)
    lp = torch.log_softmax(z, 1)
    h = -(lp.exp() * lp).sum(1)
    given = lp.gather(1, labels.long()[:, None])[:, 0]
    (given * gl + h * gh).sum().backward()
    got = plain.score(z.detach(), labels, 4)
    assert torch.allclose(got[0], given) and torch.allclose(got[1], h) and torch.allclose(got[2], torch.logsumexp(z, 1))
    assert torch.equal(got[4].long(), torch.topk(z, 4, dim=1).indices)
    assert torch.allclose(plain.score_grad(z.detach(), labels, got[2], got[1], gl, gh), z.grad)
    x = torch.randn(7, 5, generator=t, dtype=torch.float64, requires_grad=True)
    w = torch.randn(3, 4, 5, generator=t, dtype=torch.float64, requires_grad=True)
    b = torch.randn(3, 4, generator=t, dtype=torch.float64, requires_grad=True)
    off, dy = [0, 2, 2, 7], torch.randn(7, 4, generator=t, dtype=torch.float64)
    y = torch.cat([x[i:j] @ w[k].T + b[k] for k, i, j in plain.parts(off)])
    (y * dy).sum().backward()
    xd, wd = x.detach(), w.detach()
    assert torch.allclose(plain.forward(xd, off, wd, b.detach())[0], y)
    assert torch.allclose(plain.input_grad(dy, off, wd)[0], x.grad)
    dw, db, _, _ = plain.weight_grad(dy, xd, off)
    assert torch.allclose(dw, w.grad) and torch.allclose(db, b.grad)
