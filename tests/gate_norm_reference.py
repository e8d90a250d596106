"""Plain 64-bit forms of group norm, the gate and gradient clipping, and what
FP32 arithmetic may leave, for the tests.

E32 = 2^-24 is half a step of FP32 relative to the value, E16 = 2^-8 of BF16."""
import math

import torch

import ops_reference as ref
from ops_reference import E16, E32


def sample_spans(offsets, rows):
    return ref.spans(offsets, rows)


def group_norm(x, g, b, groups, spans, eps, kind):
    """y, mean, rstd, xh, z; rows of no sample are NaN."""
    n, c = x.shape
    y = torch.full_like(x, math.nan)
    xh, z = torch.zeros_like(x), torch.zeros_like(x)
    mean = torch.zeros(len(spans), groups, dtype=torch.float64)
    rstd = torch.zeros_like(mean)
    for s, (lo, hi) in enumerate(spans):
        if hi <= lo:
            continue
        v = x[lo:hi].view(hi - lo, groups, c // groups)
        mu = v.mean((0, 2))
        rs = 1 / torch.sqrt(((v - mu[None, :, None]) ** 2).mean((0, 2)) + eps)
        mean[s], rstd[s] = mu, rs
        xh[lo:hi] = ((v - mu[None, :, None]) * rs[None, :, None]).reshape(hi - lo, c)
        z[lo:hi] = xh[lo:hi] * g + b
        y[lo:hi] = ref.act(z[lo:hi], kind)
    return y, mean, rstd, xh, z


def per_row(stat, spans, rows, cg):
    """[samples, groups] spread over the rows and columns; 0 for rows of none."""
    out = torch.zeros(rows, stat.shape[1] * cg, dtype=torch.float64)
    for s, (lo, hi) in enumerate(spans):
        out[lo:hi] = stat[s].repeat_interleave(cg)
    return out


def group_norm_bounds(x, g, b, mean, rstd, xh, z, spans, eps, kind, dtype, terms=81, ratio=8):
    """Bounds of y, mean and rstd.

    Short samples: d = x - K and d^2 are summed in FP32, K the mean of at least
    1 / ratio of the sample's rows (8: 64 rows where 8 are held; others hold a
    quarter).  A sum passes at most `terms` additions: 3 in a vector, 64 rows
    of a thread, 6 between lanes and 8 between waves.  n_held (K - mean)^2 <= n
    var, and K's own sum is off by terms E32 max |x|, so that
        |K - mean| <= k = sqrt(ratio var) + terms E32 max |x|,
        mean |d| <= D = sqrt(var) + k,  mean d^2 = var + (K - mean)^2.
    The mean is off by (terms + 3) E32 D and its rounding, the variance by
    (terms + 6) E32 (var + k^2) and 2 k (terms + 3) E32 D, rstd by half of that
    relative to var + eps and a square root's and a quotient's rounding (8 E32
    in all).  Long samples are summed in FP64, which leaves less.  z passes the
    mean's error, the difference's, the products' and the sum's rounding, 12 of
    them; the activations, slope at most 1.13, are evaluated to 4 E32 |z|."""
    n, c = x.shape
    cg = c // mean.shape[1]
    top, var, some = torch.zeros_like(mean), torch.zeros_like(mean), torch.zeros_like(mean)
    for s, (lo, hi) in enumerate(spans):
        if hi > lo:
            v = x[lo:hi].view(hi - lo, -1, cg)
            top[s], some[s] = v.abs().amax((0, 2)), 1
            var[s] = ((v - v.mean((0, 2))[None, :, None]) ** 2).mean((0, 2))
    k = (ratio * var).sqrt() + terms * E32 * top
    d = var.sqrt() + k
    bm = (E32 * mean.abs() + (terms + 3) * E32 * d) * some
    noise = ((terms + 6) * E32 * (var + k ** 2) + 2 * k * (terms + 3) * E32 * d) * rstd ** 2 / 2
    br = rstd * (8 * E32 + noise)
    rs, er, em, mu = (per_row(a, spans, n, cg) for a in (rstd, noise, bm, mean))
    bz = rs * g.abs() * (em + 12 * E32 * (x - mu).abs()) + E32 * (2 * b.abs() + z.abs()) + (xh * g).abs() * er
    by = 1.13 * bz + (4 * E32 * z.abs() if kind not in ("none", "relu") else 0)
    if dtype == torch.bfloat16:
        by = by + E16 * (ref.act(z, kind).abs() + by)
    return by, bm, br, bz


def group_norm_backward(dy, x, g, b, mean, rstd, groups, spans, kind, dtype):
    """dx, dgamma, dbeta and their bounds.

    z is formed again from x with the FP32 mean and rstd: four roundings.  A
    slope's own evaluation leaves 16 E32 (1 + |z|), and the error of z times the
    slope's derivative (below 0.8); relu's slope may flip where z is within its
    error of 0.  A set's sums add 8 products in FP32, then in FP64; column sums
    add a thread's rows, the lanes, the blocks and 64 slices in FP32 (rows / 8 +
    150 terms)."""
    n, c = x.shape
    cg = c // groups
    mu, rs = per_row(mean, spans, n, cg), per_row(rstd, spans, n, cg)
    inside = torch.zeros(n, 1, dtype=torch.float64)
    for lo, hi in spans:
        inside[lo:hi] = 1
    xh = (x - mu) * rs
    z = xh * g + b
    dy = dy * inside
    dz = dy * (ref.slope(z, kind) if kind != "none" else 1.0)
    exh = 2 * E32 * xh.abs()
    ez = 2 * exh * g.abs() + E32 * z.abs()
    if kind == "none":
        edz = torch.zeros_like(dz)
    elif kind == "relu":
        edz = torch.where(z.abs() <= ez, dy.abs(), torch.zeros_like(dz))
    else:
        edz = dy.abs() * (0.8 * ez + 16 * E32 * (1 + z.abs()))
    a, ea = dz * g, edz * g.abs() + E32 * (dz * g).abs()
    dx, bdx = torch.full_like(x, math.nan), torch.zeros_like(x)
    for lo, hi in spans:
        if hi <= lo:
            continue
        v = lambda t: t[lo:hi].view(hi - lo, groups, cg)  # noqa: E731
        m = lambda t: t.mean((0, 2))[None, :, None]  # noqa: E731
        av, hv, r = v(a), v(xh), v(rs)
        m1, m2 = m(av), m(av * hv)
        em1 = m(v(ea)) + 12 * E32 * m(av.abs())
        em2 = m(v(ea) * hv.abs() + av.abs() * v(exh)) + 14 * E32 * m((av * hv).abs())
        d = r * (av - m1 - hv * m2)
        e = r * (v(ea) + em1 + hv.abs() * em2 + v(exh) * m2.abs() + 6 * E32 * (av.abs() + m1.abs() + (hv * m2).abs()))
        dx[lo:hi], bdx[lo:hi] = d.reshape(hi - lo, c), e.reshape(hi - lo, c)
    dg, db = (dz * xh).sum(0), dz.sum(0)
    k = (n / 8 + 150) * E32
    bdg = (edz * xh.abs() + dz.abs() * exh).sum(0) + k * (dz * xh).abs().sum(0)
    bdb = edz.sum(0) + k * dz.abs().sum(0)
    if dtype == torch.bfloat16:
        bdx, bdg, bdb = bdx * (1 + E16) + E16 * dx.abs().nan_to_num(0), bdg + E16 * dg.abs(), bdb + E16 * db.abs()
    return dx, dg, db, bdx, bdg, bdb


# ---- the gate ------------------------------------------------------------------
def gate(x, k, normalize):
    """weights, indices, counts, share, loss, rows with a head, p (x in 64 bits)."""
    n, h = x.shape
    some = (x > -math.inf).any(1)
    safe = torch.where(some[:, None], x, torch.zeros_like(x))
    p = torch.softmax(safe, 1) * some[:, None]
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    taken = x.gather(1, order) > -math.inf
    w = p.gather(1, order) * taken
    if normalize:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    idx = torch.where(taken, order, torch.full_like(order, -1))
    counts = torch.bincount(idx[taken], minlength=h)
    rows = int(some.sum())
    share = p.sum(0) / max(1, rows)
    loss = h * (counts.double() / max(1, int(counts.sum())) * share).sum()
    return w, idx.to(torch.int32), counts.to(torch.int32), share, loss, rows, p


def softmax_error(x):
    """Relative error of a softmax value: the exponent x - top is off by E32 of
    itself, exp by 4 E32, as the sum's terms, whose adding takes `heads` more;
    the quotient or product 4."""
    fin = torch.where(x > -math.inf, x, torch.full_like(x, math.inf))
    spread = (x.amax(1, keepdim=True) - fin.amin(1, keepdim=True)).clamp_min(0)
    spread = torch.where(spread.isfinite(), spread, torch.zeros_like(spread))
    return (2 * spread + x.shape[1] + 16) * E32


def gate_backward(x, dw, idx, counts, rows, normalize, balance):
    """dlogits and the sum of magnitudes that its error is relative to."""
    n, h = x.shape
    some = (x > -math.inf).any(1)
    p = torch.softmax(torch.where(some[:, None], x, torch.zeros_like(x)), 1) * some[:, None]
    taken = idx >= 0
    at = idx.long().clamp_min(0)
    d = torch.zeros_like(x)
    if dw is not None:
        d.scatter_add_(1, at, torch.where(taken, dw, torch.zeros_like(dw)))
    total = int(counts.sum())
    f = counts.double() * (balance * h / (max(1, rows) * max(1, total)))
    dp = f + (0 if normalize else d)
    dx = p * (dp - (p * dp).sum(1, keepdim=True))
    mag = p * (dp.abs() + (p * dp.abs()).sum(1, keepdim=True))
    if normalize:
        on = torch.zeros_like(x).scatter_add_(1, at, taken.double()).clamp_max(1)
        w = p * on
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
        dx = dx + w * (d - (w * d).sum(1, keepdim=True))
        mag = mag + w * (d.abs() + (w * d.abs()).sum(1, keepdim=True))
    return dx, mag
