"""Plain 64-bit forms of the head-tuning operators (torch.float64), and
the error that FP32 arithmetic may leave, for the tests."""
import math

import torch

E32, E16 = 2.0 ** -24, 2.0 ** -8        # half an ulp of 1: 24 significant bits in FP32, 8 in BF16
ACTS = ("none", "silu", "relu", "gelu")


def within(error, bound, what=""):
    """Every error within its bound; says how far the worst is off."""
    error, bound = error.abs().double(), bound.double().expand_as(error)
    bad = ~(error <= bound)
    if bool(bad.any()):
        worst = float((error / bound.clamp_min(1e-300)).nan_to_num(float("inf")).max())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values outside, the worst {worst:.3g} bounds off")


def act(z, kind):
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    return z.clone()


def slope(z, kind):
    if kind == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def norm(x, g, b, eps):
    mu = x.mean(1, keepdim=True)
    rs = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)
    return (x - mu) * rs * g + b, mu[:, 0], rs[:, 0]


def norm_backward(dy, x, g, mu, rs):
    xh = (x - mu[:, None]) * rs[:, None]
    a = dy * g
    dx = rs[:, None] * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def spans(offsets, rows):
    """Row ranges of the groups, bounds clamped as documented."""
    out = []
    for a, b in zip(offsets[:-1], offsets[1:]):
        a = min(max(a, 0), rows)
        out.append((a, min(max(b, a), rows)))
    return out


def sum_bound(k):
    """FP32 error of a sum of k products over the sum of their magnitudes:
    32 of them inside one matrix instruction, k / 32 of those in a row, and
    the split operands' dropped products (3 x 2^-24)."""
    return (k / 32 + 40) * E32


def linear(x, w, bias, kind, residual, ranges):
    """y, z and the magnitude sum |x| |w| + |b| of z; w [G, o, i], bias [G, o]."""
    n, o = x.shape[0], w.shape[1]
    z = torch.zeros(n, o, dtype=torch.float64, device=x.device)
    mag = torch.zeros_like(z)
    for g, (a, b) in enumerate(ranges):
        z[a:b] = x[a:b] @ w[g].t()
        mag[a:b] = x[a:b].abs() @ w[g].t().abs()
        if bias is not None:
            z[a:b] += bias[g]
            mag[a:b] += bias[g].abs()
    y = act(z, kind)
    if residual is not None:
        y = y + residual
    return y, z, mag


def linear_backward(dy, z, kind, x, w, xz, x_kind, ranges):
    """dx, dw, db, their magnitude sums (m...), and those with every slope
    replaced by its bound 1.13 (e...), which an error of the slope's own
    evaluation is relative to."""
    dz = dy * slope(z, kind) if kind != "none" else dy.clone()
    top = dy.abs() * (1.13 if kind != "none" else 1.0)
    out = {k: torch.zeros(s, dtype=torch.float64, device=x.device) for k, s in
           (("dx", x.shape), ("dw", w.shape), ("db", w.shape[:2]), ("mdx", x.shape), ("mdw", w.shape),
            ("mdb", w.shape[:2]), ("edx", x.shape), ("edw", w.shape), ("edb", w.shape[:2]))}
    for g, (a, b) in enumerate(ranges):
        d, v = dz[a:b], x[a:b]
        out["dx"][a:b], out["mdx"][a:b] = d @ w[g], d.abs() @ w[g].abs()
        out["dw"][g], out["mdw"][g] = d.t() @ v, d.t().abs() @ v.abs()
        out["db"][g], out["mdb"][g] = d.sum(0), d.abs().sum(0)
        u = top[a:b]
        out["edx"][a:b], out["edw"][g], out["edb"][g] = u @ w[g].abs(), u.t() @ v.abs(), u.sum(0)
    if x_kind != "none":
        s = slope(xz, x_kind)
        out["dx"], out["mdx"], out["edx"] = out["dx"] * s, out["mdx"] * s.abs(), out["edx"] * 1.13
    return out
