"""Plain 64-bit statements of the refiner's operators, on the CPU, with bounds
on how far a 32-bit evaluation may be from them.  Nothing here uses the
library.

The bounds.  u = 2^-24 is the rounding of one 32-bit operation.  Every value
that the kernels form goes through at most 16 such roundings beyond the ones
whose effect is written out (a statistic's rounding acts on the whole
difference x - mean; exp, erf and the reciprocal are good to a few units), so
32 u times the sum of the magnitudes involved bounds the 32-bit part; an
output rounded to a shorter type adds half a unit of that type, sums over n
terms add at most 64 terms in 32 bits in one thread before they are joined in
64, which the sum of magnitudes times 64 u covers."""
import math

import torch

U = 2.0 ** -24
HALF_UNIT = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
GROUP = 32


def act(z, kind):
    """(value, slope)."""
    if kind == "relu":
        return z.clamp(min=0), (z > 0).double()
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if kind == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def statistics(x, G, eps):
    """mean and 1 / deviation [N][G] of x [N][P][C] (float64)."""
    N, P, C = x.shape
    if P == 0:
        return torch.zeros((N, G)).double(), torch.full((N, G), 1 / math.sqrt(eps)).double()
    g = x.reshape(N, P, G, C // G).permute(0, 2, 1, 3).reshape(N, G, -1)
    mean = g.mean(2)
    var = ((g - mean[..., None]) ** 2).mean(2)
    return mean, 1 / torch.sqrt(var + eps)


def wide(v, P, C):
    """[N][G] spread over [N][P][C]."""
    N, G = v.shape
    return v[:, None, :, None].expand(N, P, G, C // G).reshape(N, P, C)


def norm(x, G, gamma, beta, eps, kind, dtype):
    """(y, bound on |error|, mean, rstd)."""
    x = x.double()
    N, P, C = x.shape
    mean, rstd = statistics(x, G, eps)
    m, r = wide(mean, P, C), wide(rstd, P, C)
    ga = torch.ones(C).double() if gamma is None else gamma.double()
    be = torch.zeros(C).double() if beta is None else beta.double()
    xh = (x - m) * r
    z = xh * ga + be
    y = act(z, kind)[0]
    big = ga.abs() * (r * (x.abs() + m.abs()) + xh.abs()) + be.abs() + z.abs() * (1 + z.abs())
    return y, 32 * U * big + HALF_UNIT[dtype] * y.abs() + TINY[dtype], mean, rstd


def norm_back(dy, x, stats, gamma, beta, kind, dtype):
    """({dx, dgamma, dbeta}, {the same: bound}) at the values x with given
    statistics [N][G][2]."""
    dy, x = dy.double(), x.double()
    N, P, C = x.shape
    G = stats.shape[1]
    m, r = wide(stats[..., 0].double(), P, C), wide(stats[..., 1].double(), P, C)
    ga = torch.ones(C).double() if gamma is None else gamma.double()
    be = torch.zeros(C).double() if beta is None else beta.double()
    xh = (x - m) * r
    z = xh * ga + be
    dz = dy * act(z, kind)[1]
    dbeta, dgamma = dz.sum((0, 1)), (dz * xh).sum((0, 1))
    M = max(1, P * (C // G))
    groups = lambda v: v.reshape(N, P, G, C // G).sum((1, 3)) / M  # noqa: E731
    a, b = groups(ga * dz), groups(ga * dz * xh)
    dx = r * (ga * dz - wide(a, P, C) - xh * wide(b, P, C))
    # magnitudes: the error of xh and z (of the size of the terms of x - m)
    # moves the slope by at most 1.2 times itself
    ex = r * (x.abs() + m.abs()) + xh.abs()
    ez = ga.abs() * ex + be.abs() + z.abs() * (1 + z.abs())
    edz = dy.abs() * (1.2 + 1.2 * ez)
    bb, bg = edz.sum((0, 1)), (edz * (1 + xh.abs()) + dy.abs() * 1.2 * ex).sum((0, 1))
    ea = groups(ga.abs() * edz)
    eb = groups(ga.abs() * (edz * (1 + xh.abs()) + dy.abs() * 1.2 * ex))
    ebx = r * (ga.abs() * edz + wide(ea, P, C) + xh.abs() * wide(eb, P, C)
               + ex * wide(b.abs(), P, C) + wide(a.abs(), P, C))
    return ({"dx": dx, "dgamma": dgamma, "dbeta": dbeta},
            {"dx": 96 * U * ebx + HALF_UNIT[dtype] * dx.abs() + TINY[dtype],
             "dgamma": 96 * U * bg + 1e-30, "dbeta": 96 * U * bb + 1e-30})


def keep(x):
    """(codes, exps, values) of x [rows][C], element by element from the rule."""
    rows, C = x.shape
    low = -24 if x.dtype == torch.float16 else -126
    most = float(torch.finfo(x.dtype).max)
    groups = -(-C // GROUP)
    codes = torch.zeros((rows, C), dtype=torch.int8)
    exps = torch.zeros((rows, groups), dtype=torch.uint8)
    values = torch.zeros((rows, C), dtype=torch.float64)
    for r in range(rows):
        for g in range(groups):
            part = x[r, g * GROUP:(g + 1) * GROUP].double()
            sl = slice(g * GROUP, g * GROUP + len(part))
            if not bool(torch.isfinite(part).all()):
                exps[r, g] = 255
                values[r, sl] = math.nan
                continue
            a, e = float(part.abs().max()), low
            while round(math.ldexp(a, -e)) > 127:   # Python rounds halves to even
                e += 1
            cap = 127 if math.ldexp(64.0, e) <= most else 63
            q = torch.round(part * math.ldexp(1.0, -e)).clamp(-cap, cap)
            codes[r, sl] = q.to(torch.int8)
            exps[r, g] = e + 127
            values[r, sl] = q * math.ldexp(1.0, e)
    return codes, exps, values


def turn(x, pos, freq, axis, layout, inverse, dtype):
    """(turned, bound) of x [T][heads][D]: the angle is one 32-bit product."""
    pairs = freq.shape[0]
    angle = (pos.float()[:, axis.long()] * freq.float()).double()[:, None, :]
    c, s = torch.cos(angle), torch.sin(angle) * (-1 if inverse else 1)
    x = x.double()
    y, big = x.clone(), torch.zeros_like(x)
    one, two = ((slice(0, pairs), slice(pairs, 2 * pairs)) if layout == "halves"
                else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)))
    a, b = x[..., one], x[..., two]
    y[..., one], y[..., two] = a * c - b * s, b * c + a * s
    big[..., one] = big[..., two] = a.abs() + b.abs()
    return y, 8 * U * big + HALF_UNIT[dtype] * y.abs() * (big > 0) + TINY[dtype]
