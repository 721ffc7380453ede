"""The operators on caller-owned tensors in 64 bits, from their definitions, and the error bounds that go with them.

Unit roundoffs: an fp32 operation is off by at most 2^-24 of its result, a rounding to bf16 by 2^-9.  A matrix core may
round a sum more than once on its way and need not round to nearest, so a sum's steps are taken at 2^-23 here.
"""
import numpy as np
import torch

U32, UACC, UBF16 = 2.0 ** -24, 2.0 ** -23, 2.0 ** -9


def mix64(z):
    z = np.asarray(z, dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def kept(rows, cols, p, seed):
    """bool [rows][cols]: which elements a dropout keeps."""
    words = -(-cols // 4)
    with np.errstate(over="ignore"):
        key = mix64(np.uint64((seed + 0x44524F50) % 2 ** 64))
        z = mix64(key + np.arange(1, rows * words + 1, dtype=np.uint64) * np.uint64(0x9E3779B97F4A7C15))
    draw = np.stack([(z >> np.uint64(16 * j)) & np.uint64(0xFFFF) for j in range(4)], axis=-1)
    return torch.from_numpy(draw.reshape(rows, 4 * words)[:, :cols] >= round(65536 * p))


def factor(p):
    return 65536.0 / (65536 - round(65536 * p))


def parts(offsets):
    return [(g, a, b) for g, (a, b) in enumerate(zip(offsets, offsets[1:]))]


def rounded(bound, value, dtype):
    """The bound with the last rounding to dtype."""
    return bound + (bound + value.abs()) * (2 * UBF16 if dtype == torch.bfloat16 else 2 * U32) + 1e-37


def forward(x, offsets, w, bias=None, relu=False, p=0.0, seed=0):
    """(y, bound, rows written); rows outside the groups are 0."""
    rows, n = x.shape[0], w.shape[1]
    y, mag = torch.zeros(rows, n, dtype=torch.float64), torch.zeros(rows, n, dtype=torch.float64)
    written = torch.zeros(rows, dtype=torch.bool)
    for g, a, b in parts(offsets):
        xg, wg = x[a:b].double(), w[g].double()
        y[a:b], mag[a:b] = xg @ wg.T, xg.abs() @ wg.abs().T
        if bias is not None:
            y[a:b] += bias[g].double()
            mag[a:b] += bias[g].double().abs()
        written[a:b] = True
    bound = (x.shape[1] + 8) * UACC * mag
    if relu:
        y = y.clamp(min=0)
    if p:
        y = torch.where(kept(rows, n, p, seed), y * factor(p), 0.0)
        bound = bound * factor(p) + y.abs() * 2 * U32
    return y, rounded(bound, y, x.dtype), written


def input_grad(dy, offsets, w, gate=None, p=0.0):
    dx, bound, written = forward(dy, offsets, w.transpose(1, 2))
    if gate is not None:
        dx = torch.where(gate > 0, dx * factor(p), 0.0)
        bound = bound * factor(p) * (1 + 4 * U32)
    return dx, bound, written


def weight_grad(dy, x, offsets):
    """(dw, db, their bounds)."""
    out = []
    for g, a, b in parts(offsets):
        d, v = dy[a:b].double(), x[a:b].double()
        out.append((d.T @ v, d.sum(0), (b - a + 8) * UACC * (d.abs().T @ v.abs()) + 1e-37,
                    (b - a + 8) * UACC * d.abs().sum(0) + 1e-37))
    return tuple(torch.stack(t) for t in zip(*out))


def score(z, labels, top):
    """(logp, entropy, lse, top_logp, top_class) in 64 bits."""
    z = z.double()
    rows, L = z.shape
    m = z.max(1).values
    base = torch.where(m == -np.inf, 0.0, m)[:, None]
    e = torch.exp(z - base)
    s = e.sum(1)
    lse = base[:, 0] + torch.log(s)
    empty = (m == -np.inf) & (s == 0)
    lse = torch.where(torch.isinf(m) & (m > 0), np.nan, lse)
    lp = (z - base) - torch.log(s)[:, None]  # z - lse, which would lose log s next to a large m
    p = torch.exp(lp)
    h = -(p * torch.where(p == 0, 0.0, lp)).sum(1)
    h = torch.where(empty, 0.0, torch.where(torch.isnan(lse), np.nan, h))
    lp = torch.where(empty[:, None], -np.inf, lp)
    lp = torch.where(torch.isnan(lse)[:, None], np.nan, lp)
    lp = torch.where(lp < -torch.finfo(torch.float32).max, -np.inf, lp)  # past what an fp32 result holds
    # by value, a NaN first, then by index: a stable sort of the negated values
    key = torch.where(torch.isnan(z), np.inf, z)
    rank = torch.where(torch.isnan(z), 1.0, 0.0)
    order = np.lexsort((np.broadcast_to(np.arange(L), (rows, L)), -key.numpy(), -rank.numpy()), axis=1)
    order = torch.from_numpy(order)[:, :top]
    given = None
    if labels is not None:
        ok = (labels >= 0) & (labels < L)
        given = torch.where(ok, lp.gather(1, labels.clamp(0, L - 1).long()[:, None])[:, 0], 0.0)
    return given, h, lse, lp.gather(1, order), order.int()


def score_bounds(z):
    """[rows] bounds of lse (and of a log probability, apart from the logit's own size) and of entropy.

    A term exp(d), d = z - m <= 0: d is off by U32 |d|, the exponential by a few U32, so the term by (|d| + 4) 2 U32 of
    itself, and sums of L positive terms in a tree of at least 64 lanes by (L / 64 + 32) U32 of themselves.  Terms
    below exp(-87) may be lost as subnormals: L 2^-126.
    """
    z = z.double()
    m = z.max(1, keepdim=True).values
    d = torch.where(z == -np.inf, 0.0, z - m)
    p = torch.softmax(z, 1)
    far = (p * d.abs()).sum(1)
    rel = (far + 4) * 2 * U32 + (z.shape[1] / 64 + 32) * U32
    lse = rel + 4 * U32 * (m[:, 0].abs() + np.log(z.shape[1]) + 1)
    far2 = (p * d * d).sum(1)
    h = rel * (1 + far) + 2 * U32 * (far2 + 8 * far) + 4 * U32 * (far + np.log(z.shape[1]) + 1)
    return lse, h


def score_grad(z, labels, lse, entropy, g_logp, g_entropy):
    z = z.double()
    rows, L = z.shape
    zero = torch.zeros(rows, dtype=torch.float64)
    gl = zero if g_logp is None else g_logp.double()
    gh = zero if g_entropy is None else g_entropy.double()
    h = zero if entropy is None else entropy.double()
    lse = lse.double()
    empty = lse < -1e30
    lp = z - torch.where(empty, 0.0, lse)[:, None]
    p = torch.exp(lp)
    if labels is not None:
        ok = (labels >= 0) & (labels < L)
        gl = torch.where(ok, gl, 0.0)
    d = -gl[:, None] * p - gh[:, None] * p * (torch.where(p == 0, 0.0, lp) + h[:, None])
    if labels is not None:
        r = torch.arange(rows)[ok]
        d[r, labels[ok].long()] += gl[ok]
    return torch.where(empty[:, None], 0.0, d)
