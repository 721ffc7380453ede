"""Host-side checks of gated layers, residual norms and distillation (no GPU needed): bad arguments are refused before
anything touches the device, calls without rows do nothing, and the 64-bit definitions that the GPU tests use agree with
autograd."""
import ctypes as C
import os

import pytest
import torch

import blocks_plain as blocks
import ops_plain as plain
from test_ops_host import FAR, GROUPS, MAX, MIN32

g = pytest.importorskip("paper_2609_29395_amd.gcpsl")

built = pytest.mark.skipif(not os.path.exists(g.LIB_PATH), reason="libgcpsl.so not built")

GATED = dict(dtype=0, G=2, rows=5, n=3, k=4, offsets=FAR, x=FAR, ldx=4, w=FAR, w_gs=24, bias=FAR, bias_gs=6, act=0, y=FAR,
             ldy=3, pre=FAR, ldpre=6, stream=None)
GATED_GRAD = dict(dtype=0, G=2, rows=5, n=3, k=4, offsets=FAR, dz=FAR, lddz=3, v=FAR, v_gs=12, act=1, pre=FAR, ldpre=8,
                  dpre=FAR, lddpre=8, stream=None)  # n: the layer after, k: gates
NORM = dict(dtype=0, G=2, rows=5, n=4, offsets=FAR, x=FAR, ldx=4, y=FAR, ldy=4, gate=FAR, ldgate=4, w_block=FAR,
            w_block_gs=4, w_next=FAR, w_next_gs=4, alpha=1.0, beta=1.0, eps=1e-6, out=FAR, ldo=4, h=FAR, ldh=4,
            r_block=FAR, r_next=FAR, stream=None)
NORM_GRAD = dict(dtype=0, G=2, rows=5, n=4, offsets=FAR, out=FAR, ldo=4, g_out=FAR, ldgo=4, g_h=FAR, ldgh=4, y=FAR, ldy=4,
                 gate=FAR, ldgate=4, w_block=FAR, w_block_gs=4, w_next=FAR, w_next_gs=4, r_block=FAR, r_next=FAR,
                 alpha=1.0, beta=1.0, dx=FAR, lddx=4, dy=FAR, lddy=4, dgate=FAR, lddgate=4, dw_block=FAR, dw_block_gs=4,
                 dw_next=FAR, dw_next_gs=4, workspace=FAR, workspace_bytes=1 << 30, stream=None)
DISTILL = dict(dtype=0, rows=5, L=7, z=FAR, ldz=7, top=2, t_class=FAR, t_value=FAR, temperature=2.0, labels=FAR, kl=FAR,
               lse_t=FAR, logp=FAR, lse=FAR, workspace=FAR, workspace_bytes=1 << 30, stream=None)
DISTILL_GRAD = dict(dtype=0, rows=5, L=7, z=FAR, ldz=7, top=2, t_class=FAR, t_value=FAR, temperature=2.0, labels=FAR,
                    lse_t=FAR, lse=FAR, g_kl=FAR, g_logp=FAR, dz=FAR, lddz=7, stream=None)
NARROW = [c for c in GROUPS if "k" not in c]  # of operators without a k
TEACHER = [dict(top=0), dict(top=257), dict(t_class=None), dict(t_value=None), dict(t_class=FAR + 2), dict(t_value=FAR + 1),
           dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=1e-4),
           dict(temperature=2048.0), dict(temperature=float("inf"))]


def call(name, good, **change):
    args = dict(good)
    for key in change:
        assert key in args, key
    args.update(change)
    return getattr(g.lib(), name)(*args.values())


@built
@pytest.mark.parametrize("name,good,bad", [
    ("gcpsl_group_gated_forward", GATED, GROUPS + [
        dict(x=None), dict(x=FAR + 2), dict(ldx=-1), dict(ldx=MIN32), dict(w=None), dict(w=FAR + 1), dict(w_gs=-1),
        dict(w_gs=MAX + 1), dict(bias=FAR + 2), dict(bias_gs=-1), dict(act=-1), dict(act=3), dict(y=None), dict(ldy=2),
        dict(pre=FAR + 2), dict(ldpre=5), dict(n=2 ** 27 + 1)]),
    ("gcpsl_group_gated_grad", GATED_GRAD, GROUPS + [
        dict(dz=None), dict(lddz=-1), dict(v=None), dict(v_gs=-1), dict(act=7), dict(pre=None), dict(pre=FAR + 1),
        dict(ldpre=-1), dict(dpre=None), dict(lddpre=7), dict(k=2 ** 27 + 1)]),
    ("gcpsl_group_residual_norm", NORM, NARROW + [
        dict(x=None), dict(x=FAR + 2), dict(ldx=-1), dict(y=None), dict(y=FAR + 1), dict(gate=FAR + 2), dict(ldgate=-1),
        dict(w_block=FAR + 2), dict(w_block_gs=-1), dict(w_next=FAR + 1), dict(w_next_gs=MAX + 1), dict(w_next=None),
        dict(h=None), dict(ldh=3), dict(out=None), dict(ldo=3), dict(ldx=5), dict(r_block=FAR + 2), dict(r_next=FAR + 1),
        dict(alpha=float("inf")), dict(alpha=float("nan")), dict(beta=1e39), dict(eps=0.0), dict(eps=-1.0),
        dict(eps=float("nan")), dict(eps=1e31), dict(y=None, gate=None, w_block=None),
        dict(y=None, gate=None, w_block=None, out=None, alpha=2.0),
        dict(y=None, gate=None, w_block=None, out=None, w_next=None, h=None)]),
    ("gcpsl_group_residual_norm_grad", NORM_GRAD, NARROW + [
        dict(out=None), dict(out=FAR + 2), dict(g_out=FAR + 1), dict(g_h=None), dict(w_next=None), dict(r_next=None),
        dict(g_h=FAR + 2), dict(ldgh=-1), dict(y=None), dict(ldy=MIN32), dict(gate=None), dict(w_block=None),
        dict(r_block=None), dict(r_block=FAR + 2), dict(dx=None), dict(lddx=3), dict(dy=None), dict(lddy=3),
        dict(lddgate=3), dict(dw_block=FAR + 2), dict(dw_block_gs=3), dict(dw_next_gs=3), dict(alpha=float("nan")),
        dict(beta=float("inf")), dict(g_out=None, g_h=None, w_next=None, dw_next=None),
        dict(y=None, gate=None, w_block=None, dgate=None, dw_block=None),
        dict(y=None, gate=None, w_block=None, dy=None, dgate=None, dw_block=None, alpha=0.5)]),
    ("gcpsl_distill", DISTILL, TEACHER + [
        dict(dtype=2), dict(rows=-1), dict(L=0), dict(L=2 ** 28 + 1), dict(z=None), dict(z=FAR + 2), dict(ldz=-1),
        dict(labels=None), dict(kl=FAR + 2), dict(lse=FAR + 1), dict(labels=FAR + 2)]),
    ("gcpsl_distill_grad", DISTILL_GRAD, TEACHER + [
        dict(dtype=-1), dict(rows=MIN32), dict(L=0), dict(z=None), dict(dz=None), dict(lddz=6), dict(ldz=8),
        dict(lse_t=None), dict(lse=None), dict(labels=None), dict(g_kl=None, g_logp=None), dict(g_kl=FAR + 2)]),
])
def test_bad_arguments_are_refused(name, good, bad):
    for change in bad:
        assert call(name, good, **change) == g.EINVAL, change
        assert g.lib().gcpsl_last_error(), change


@built
def test_too_many_rows_or_workgroups_are_refused():
    assert call("gcpsl_group_gated_forward", GATED, rows=2 ** 31 - 1) == g.EUNSUPPORTED
    assert call("gcpsl_group_gated_forward", GATED, rows=2 ** 31 - 2048, n=2 ** 27, k=1, ldy=2 ** 31 - 1,
                ldpre=2 ** 31 - 1) == g.EUNSUPPORTED
    assert call("gcpsl_group_residual_norm", NORM, rows=2 ** 31 - 1) == g.EUNSUPPORTED
    assert call("gcpsl_group_residual_norm_grad", NORM_GRAD, rows=2 ** 31 - 1) == g.EUNSUPPORTED
    assert call("gcpsl_group_residual_norm_grad", NORM_GRAD, rows=1, n=2 ** 28, G=1024, ldo=2 ** 28, ldgo=2 ** 28,
                ldgh=2 ** 28, lddx=2 ** 28, lddy=2 ** 28, lddgate=2 ** 28, dw_block_gs=2 ** 28,
                dw_next_gs=2 ** 28) == g.EUNSUPPORTED


@built
def test_no_rows_need_no_tensors():
    assert call("gcpsl_group_gated_forward", GATED, rows=0, x=None, y=None, pre=None) == g.OK
    assert call("gcpsl_group_gated_grad", GATED_GRAD, rows=0, dz=None, pre=None, dpre=None) == g.OK
    assert call("gcpsl_group_residual_norm", NORM, rows=0, x=None, y=None, out=None, h=None, r_block=None) == g.OK
    assert call("gcpsl_group_residual_norm_grad", NORM_GRAD, rows=0, out=None, dx=None, dy=None, dw_block=None,
                dw_next=None) == g.OK
    assert call("gcpsl_distill", DISTILL, rows=0, z=None, t_class=None, t_value=None, kl=None) == g.OK
    assert call("gcpsl_distill_grad", DISTILL_GRAD, rows=0, z=None, dz=None, lse_t=None, g_kl=None) == g.OK


@built
def test_workspaces():
    n = C.c_size_t(1)
    assert g.lib().gcpsl_group_residual_workspace_bytes(0, 2, 0, 4, C.byref(n)) == g.OK and n.value == 0
    assert g.lib().gcpsl_group_residual_workspace_bytes(0, 2, 0, 4, None) == g.EINVAL
    assert g.lib().gcpsl_group_residual_workspace_bytes(0, 0, 0, 4, C.byref(n)) == g.EINVAL
    assert g.lib().gcpsl_group_residual_workspace_bytes(0, 1, 2 ** 31 - 1, 4, C.byref(n)) == g.EUNSUPPORTED
    assert g.lib().gcpsl_distill_workspace_bytes(0, 1, 0, C.byref(n)) == g.EINVAL
    assert g.lib().gcpsl_distill_workspace_bytes(0, 1, 10, None) == g.EINVAL
    need = g.group_residual_workspace_bytes("f32", 2, 100000, 4)
    assert need > 0
    for change in (dict(workspace_bytes=need - 1), dict(workspace=None), dict(workspace=FAR + 4)):
        assert call("gcpsl_group_residual_norm_grad", NORM_GRAD, rows=100000, **{"workspace_bytes": need, **change}) == g.EINVAL
    need = g.distill_workspace_bytes("f32", 1, 100000)
    assert need > 0
    for change in (dict(workspace_bytes=need - 1), dict(workspace=None), dict(workspace=FAR + 4)):
        assert call("gcpsl_distill", DISTILL, rows=1, L=100000, ldz=100000, **{"workspace_bytes": need, **change}) == g.EINVAL


def leaf(gen, *shape, scale=1.0, add=0.0):
    return (torch.randn(*shape, generator=gen, dtype=torch.float64) * scale + add).requires_grad_()


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
def test_gated_definitions_against_autograd(name):
    gen = torch.Generator().manual_seed(3)
    x, w, b = leaf(gen, 7, 5), leaf(gen, 3, 8, 5), leaf(gen, 3, 8)
    v, dz = leaf(gen, 3, 6, 4).detach(), leaf(gen, 7, 6).detach()
    off = [0, 2, 2, 7]
    pre = torch.cat([x[i:j] @ w[k].T + b[k] for k, i, j in plain.parts(off)])
    pre.retain_grad()
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[name]
    y = f(pre[:, :4]) * pre[:, 4:]
    z = torch.cat([y[i:j] @ v[k].T for k, i, j in plain.parts(off)])
    (z * dz).sum().backward()
    got = blocks.gated_forward(x.detach(), off, w.detach(), b.detach(), name)
    assert torch.allclose(got[0], y) and torch.allclose(got[2], pre)
    assert torch.allclose(blocks.gated_grad(dz, off, v, pre.detach(), name)[0], pre.grad)


def test_residual_definitions_against_autograd():
    gen = torch.Generator().manual_seed(4)
    rows, n, off = 7, 6, [0, 2, 2, 7]
    x, y, gate = leaf(gen, rows, n), leaf(gen, rows, n), leaf(gen, rows, n)
    w1, w2 = leaf(gen, 3, n, add=1.0), leaf(gen, 3, n, add=1.0)
    go, gh = leaf(gen, rows, n).detach(), leaf(gen, rows, n).detach()
    which = [0, 0, 2, 2, 2, 2, 2]
    norm = torch.nn.functional.rms_norm
    new = 0.5 * x + 2.0 * torch.sigmoid(gate) * norm(y, (n,), eps=1e-3) * w1[which]
    h = norm(new, (n,), eps=1e-3) * w2[which]
    (new * go + h * gh).sum().backward()
    d = [t.detach() for t in (x, y, gate, w1, w2)]
    got, _ = blocks.residual(d[0], off, *d[1:], 0.5, 2.0, 1e-3)
    assert torch.allclose(got["out"][0], new) and torch.allclose(got["h"][0], h)
    res, _ = blocks.residual_grad(new.detach(), off, go, gh, *d[1:], got["r_block"][0], got["r_next"][0], 0.5, 2.0)
    for k, t in (("dx", x), ("dy", y), ("dgate", gate), ("dw_block", w1), ("dw_next", w2)):
        assert torch.allclose(res[k][0], t.grad), k


def test_distillation_definitions_against_autograd():
    gen = torch.Generator().manual_seed(5)
    z, T = leaf(gen, 6, 11), 1.7
    cls = torch.stack([torch.randperm(11, generator=gen)[:4] for _ in range(6)]).int()
    val = torch.randn(6, 4, generator=gen)
    labels = torch.randint(0, 11, (6,), generator=gen).int()
    a, b = torch.randn(6, generator=gen).double(), torch.randn(6, generator=gen).double()
    lp = torch.log_softmax(z / T, 1).gather(1, cls.long())
    kl = torch.nn.functional.kl_div(lp, torch.softmax(val.double() / T, 1), reduction="none").sum(1)
    logp = torch.log_softmax(z, 1).gather(1, labels.long()[:, None])[:, 0]
    (kl * a + logp * b).sum().backward()
    got = blocks.distill(z.detach(), cls, val, T, labels)
    assert torch.allclose(got["kl"][0], kl) and torch.allclose(got["logp"][0], logp)
    assert torch.allclose(got["lse_t"][0], torch.logsumexp(z / T, 1))
    dz, _ = blocks.distill_grad(z.detach(), cls, val, got["lse_t"][0], T, labels, got["lse"][0], a, b)
    assert torch.allclose(dz, z.grad)
