"""Gated layers, residual norms and distillation in 64 bits, from their definitions, and the error bounds that go with
them (ops_plain.py: unit roundoffs, grouped products).

exp, reciprocal, logarithm, erfc and square root are taken as off by at most 4 steps of 2^-23 of their result, next to
what the rounding of their argument makes of it: e^v of an argument off by 2^-24 |v| is off by 2^-24 |v| of itself, the
normal distribution's lower tail at g by g^2 2^-24 (its logarithm falls as -g^2 / 2).
"""
import math

import torch

import ops_plain as plain
from ops_plain import U32, UACC, parts, rounded


def act(g, name):
    """(f(g), f'(g), the magnitude that f' is summed from)."""
    if name == "silu":
        s = torch.sigmoid(g)
        rest = torch.sigmoid(-g)
        return g * s, s + g * s * rest, s + g.abs() * s * rest
    if name == "gelu":
        phi, pdf = torch.erfc(-g / math.sqrt(2)) / 2, torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return g * phi, phi + g * pdf, phi + g.abs() * pdf
    return g.clamp(min=0), (g > 0).double(), torch.ones_like(g)


def gated_forward(x, offsets, w, bias=None, name="silu"):
    """(y, its bound, pre, its bound, rows written)."""
    n = w.shape[1] // 2
    pre, _, written = plain.forward(x.double(), offsets, w.double(), None if bias is None else bias.double())
    mag = plain.forward(x.double().abs(), offsets, w.double().abs(), None if bias is None else bias.double().abs())[0]
    sums = (x.shape[1] + 8) * UACC * mag
    g, u, eg, eu = pre[:, :n], pre[:, n:], sums[:, :n], sums[:, n:]
    f = act(g, name)[0]
    # |f'| <= 1.13 for all three; f itself is off by its argument's rounding and a few steps
    bound = 1.13 * eg * (u.abs() + eu) + f.abs() * eu + (f * u).abs() * (g.abs() + g * g / 2 + 16) * UACC
    bound = bound + u.abs() * 1e-36  # (e^-|g| below fp32's normal numbers is 0)
    return f * u, rounded(bound, f * u, x.dtype), pre, rounded(sums, pre, x.dtype), written


def gated_grad(dz, offsets, w, pre, name="silu"):
    """(dpre, its bound, rows written)."""
    n = w.shape[2]
    dh, _, written = plain.forward(dz.double(), offsets, w.double().transpose(1, 2))
    mag = plain.forward(dz.double().abs(), offsets, w.double().abs().transpose(1, 2))[0]
    eh = (dz.shape[1] + 8) * UACC * mag
    g, u = pre[:, :n].double(), pre[:, n:].double()
    f, d, dmag = act(g, name)
    rel = (g.abs() + g * g / 2 + 16) * UACC
    ef, ed = f.abs() * rel + 1e-36, dmag * rel + 1e-36
    out = torch.cat((d * u * dh, f * dh), 1)
    bound = torch.cat((((d * u).abs() + ed * u.abs()) * eh + ed * (u * dh).abs() + 2 * U32 * (d * u * dh).abs(),
                       (f.abs() + ef) * eh + ef * dh.abs() + 2 * U32 * (f * dh).abs()), 1)
    return torch.where(written[:, None], out, 0.0), rounded(bound, out, dz.dtype), written


def by_row(w, offsets, rows):
    """[rows][n] of [G][n]; 1 outside the groups."""
    out = torch.ones(rows, w.shape[1], dtype=torch.float64)
    for g, a, b in parts(offsets):
        out[a:b] = w[g].double()
    return out


def _written(offsets, rows):
    t = torch.zeros(rows, dtype=torch.bool)
    t[offsets[0]:offsets[-1]] = True
    return t


def residual(x, offsets, y=None, gate=None, w_block=None, w_next=None, alpha=1.0, beta=1.0, eps=1e-6):
    """dict of (value, bound) of out, h, r_block, r_next (those the call has), and the rows written.

    A row's mean square is summed by 64 threads or more, each one after another, then in a tree: off by (n / 64 + 32)
    2^-24 of itself, its reciprocal root by half of that and a few steps."""
    rows, n = x.shape
    dtype = x.dtype
    x = x.double()
    srel = (n / 64 + 32) * U32 / 2 + 6 * U32
    got = {}
    new, e = x, torch.zeros_like(x)
    if y is not None:
        t, rel = y.double(), torch.zeros(rows, 1, dtype=torch.float64)
        if w_block is not None:
            r1 = 1 / torch.sqrt((t * t).mean(1) + eps)
            got["r_block"] = (r1, r1 * srel + 1e-37)
            t = by_row(w_block, offsets, rows) * t * r1[:, None]
            rel = rel + srel + 4 * U32
        if gate is not None:
            t = t * torch.sigmoid(gate.double())
            rel = rel + (gate.double().abs() + 12) * UACC
        new = alpha * x + beta * t
        e = (beta * t).abs() * (rel + 4 * U32) + (alpha * x).abs() * 4 * U32 + 1e-37
        got["out"] = (new, rounded(e, new, dtype))
    if w_next is not None:
        mean = (new * new).mean(1)
        r2 = 1 / torch.sqrt(mean + eps)
        rel2 = ((new.abs() * e + e * e).mean(1)) / (mean + eps) + srel
        got["r_next"] = (r2, r2 * rel2 + 1e-37)
        w = by_row(w_next, offsets, rows)
        h = w * new * r2[:, None]
        eh = (w * r2[:, None]).abs() * e + h.abs() * (rel2[:, None] + 4 * U32)
        got["h"] = (h, rounded(eh, h, dtype))
    return got, _written(offsets, rows)


def residual_grad(out, offsets, g_out=None, g_h=None, y=None, gate=None, w_block=None, w_next=None, r_block=None,
                  r_next=None, alpha=1.0, beta=1.0):
    """dict of (value, bound) of dx, dy, dgate, dw_block, dw_next (those the call has), and the rows written.  Every
    sum is off by its number of additions' roundings of the magnitudes it adds, every product by a few."""
    rows, n = out.shape
    dtype = out.dtype
    zero = torch.zeros(rows, n, dtype=torch.float64)
    k_row = (n / 64 + 40) * U32  # of a row's sums
    got = {}
    D = zero if g_out is None else g_out.double()
    eD, mD = zero, D.abs()  # error of D, magnitude of what it is made of
    o = a = r2 = zero
    if g_h is not None:
        gh, w2, r2 = g_h.double(), by_row(w_next, offsets, rows), r_next.double()[:, None]
        o, a = out.double() * r2, w2 * gh
        c2 = (a * o).mean(1, keepdim=True)
        e2 = (a * o).abs().mean(1, keepdim=True) * k_row
        D = D + r2 * (a - o * c2)
        mD = mD + (r2 * a).abs() + (r2 * o * c2).abs()
        eD = mD * 8 * U32 + (r2 * o).abs() * e2
        got["dw_next"] = _columns(gh * o, (gh * o).abs() * 4 * U32, offsets)
    else:
        e2 = torch.zeros(rows, 1, dtype=torch.float64)
    dx = alpha * D
    got["dx"] = (dx, rounded(abs(alpha) * eD + dx.abs() * 2 * U32, dx, dtype))
    if y is None:
        return got, _written(offsets, rows)
    s = rest = torch.ones_like(zero)
    rel_s = 0.0
    if gate is not None:
        s, rest = torch.sigmoid(gate.double()), torch.sigmoid(-gate.double())
        rel_s = (gate.double().abs() + 12) * UACC
    es = beta * D * s
    ee = (beta * s).abs() * eD + es.abs() * (rel_s + 4 * U32) + 1e-37
    t, v, w1 = y.double(), y.double(), torch.ones_like(zero)
    if w_block is not None:
        r1, w1 = r_block.double()[:, None], by_row(w_block, offsets, rows)
        v = t * r1
        t = w1 * v
        c = es * w1
        c1 = (c * v).mean(1, keepdim=True)
        # mean(c v) = (sum p (g_out + r2 a) - r2 c2 sum p o) / n with p = beta s w1 v
        p = (beta * s * w1 * v).abs()
        e1 = (p * mD * (k_row + rel_s)).mean(1, keepdim=True) + (p * o.abs()).mean(1, keepdim=True) * (r2 if g_h is not None else 0.0) * e2
        dy = r1 * (c - v * c1)
        edy = r1.abs() * (w1.abs() * ee + v.abs() * e1) + (r1 * c).abs() * 6 * U32 + (r1 * v * c1).abs() * 6 * U32
        got["dw_block"] = _columns(es * v, v.abs() * ee + (es * v).abs() * 4 * U32, offsets)
    else:
        dy, edy = es, ee
    got["dy"] = (dy, rounded(edy, dy, dtype))
    if gate is not None:
        dg = es * t * rest
        got["dgate"] = (dg, rounded((t * rest).abs() * ee + dg.abs() * (rel_s + 6 * U32), dg, dtype))
    return got, _written(offsets, rows)


def _columns(terms, errors, offsets):
    """(sums over each group's rows, their bounds): rows of a piece one after another, pieces one after another."""
    v, e = [], []
    for _, a, b in parts(offsets):
        v.append(terms[a:b].sum(0))
        e.append(errors[a:b].sum(0) + (b - a + 8) * U32 * terms[a:b].abs().sum(0) + 1e-37)
    return torch.stack(v), torch.stack(e)


def teacher(t_class, t_value, L, temperature):
    """(log q [rows][top], -inf where an entry is left out; rows with any)."""
    v = t_value.double() / temperature
    left = (t_class >= 0) & (t_class < L) & (t_value != -math.inf)
    v = torch.where(left, v, -math.inf)
    some = left.any(1)
    lse = torch.logsumexp(torch.where(some[:, None], v, 0.0), 1, keepdim=True)
    return torch.where(left, v - lse, -math.inf), some


def _log_softmax(z):
    """(log probabilities, lse); -inf throughout for a row of -inf, NaN with a NaN or +inf."""
    m = z.max(1, keepdim=True).values
    base = torch.where(m == -math.inf, 0.0, m)
    s = torch.exp(z - base).sum(1, keepdim=True)
    lse = base + torch.log(s)
    lp = (z - base) - torch.log(s)
    return torch.where(s == 0, -math.inf, lp), torch.where(s == 0, -math.inf, lse)[:, 0]


def distill(z, t_class, t_value, temperature=1.0, labels=None):
    """dict of (value, bound) of kl, lse_t and, with labels, logp and lse.

    The bounds of the sums are those of the scores (ops_plain.score_bounds) with d = (z - m) / T off by twice that, and
    a rebasing to a larger maximum for every 2,048 elements of a row."""
    rows, L = z.shape
    z = z.double()

    def lse_bound(v):
        m = v.max(1, keepdim=True).values
        d = torch.where(v == -math.inf, 0.0, v - m)
        far = (torch.softmax(v, 1) * d.abs()).sum(1)
        return (far + 4) * 4 * U32 + (L / 64 + L / 512 + 32) * U32 + 6 * U32 * (m[:, 0].abs() + math.log(L) + 1)

    lp_t, lse_t = _log_softmax(z / temperature)
    lq, some = teacher(t_class, t_value, L, temperature)
    q = lq.exp()
    own = lp_t.gather(1, t_class.clamp(0, L - 1).long())
    terms = torch.where(q == 0, 0.0, q * (lq - own))
    kl = torch.where(some, terms.sum(1), 0.0)
    e = lse_bound(z / temperature)
    far = torch.where(q == 0, 0.0, q * ((lq.abs() + own.abs() + 4) * 8 + (t_class.shape[1] + 8) * (lq - own).abs())).sum(1)
    got = {"kl": (kl, e + (far + 4 * math.log(t_class.shape[1]) + 8) * U32),
           "lse_t": (lse_t, e)}
    if labels is not None:
        lp, lse = _log_softmax(z)
        ok = (labels >= 0) & (labels < L)
        logp = torch.where(ok, lp.gather(1, labels.clamp(0, L - 1).long()[:, None])[:, 0], 0.0)
        e = lse_bound(z)
        got.update(lse=(lse, e), logp=(logp, e + logp.abs().clamp(max=1e30) * 4 * U32))
    return got


def distill_grad(z, t_class, t_value, lse_t, temperature=1.0, labels=None, lse=None, g_kl=None, g_logp=None):
    """(dz, bound)."""
    rows, L = z.shape
    dtype = z.dtype
    z = z.double()
    d, e = torch.zeros_like(z), torch.zeros_like(z)
    if g_kl is not None:
        lq, some = teacher(t_class, t_value, L, temperature)
        lt = lse_t.double()[:, None]
        alive = some[:, None] & ~(lt <= -2.0 ** 23)
        g = torch.where(alive, g_kl.double()[:, None] / temperature, 0.0)
        lt = torch.where(alive, lt, 0.0)
        p = torch.exp(z / temperature - lt)
        q = torch.zeros_like(z)
        eq = torch.zeros_like(z)
        for r in range(rows):
            for k in range(t_class.shape[1]):
                c = int(t_class[r, k])
                if 0 <= c < L and lq[r, k] != -math.inf:
                    q[r, c] += math.exp(lq[r, k])
                    eq[r, c] += math.exp(lq[r, k]) * (abs(float(lq[r, k])) * 2 + t_class.shape[1] + 12) * 2 * U32
        spread = torch.where(p == 0, 0.0, ((z / temperature).abs() + lt.abs()) * 2 + 8)
        d = d + g * (p - q)
        e = e + g.abs() * (p * spread * 2 * U32 + eq + (p + q) * 6 * U32)
    if g_logp is not None:
        l1 = lse.double()[:, None]
        ok = ((labels >= 0) & (labels < L))[:, None] & ~(l1 <= -2.0 ** 23)
        g = torch.where(ok, g_logp.double()[:, None], 0.0)
        l1 = torch.where(ok, l1, 0.0)
        p = torch.exp(z - l1)
        hot = torch.zeros_like(z)
        hot.scatter_(1, labels.clamp(0, L - 1).long()[:, None], 1.0)
        spread = torch.where(p == 0, 0.0, (z.abs() + l1.abs()) * 2 + 8)
        d = d + g * (hot - torch.where(g == 0, 0.0, p))
        e = e + g.abs() * (p * spread * 2 * U32 + (p + hot) * 6 * U32)
    return d, rounded(e, d, dtype)
