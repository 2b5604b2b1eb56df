"""Plain 64-bit statements of the refiner's attention and of its heads' norm, on
the CPU, with bounds on how far the kernels may be from them.  Nothing here uses
the library.

The bounds.  u = 2^-24 is the rounding of one 32-bit operation, h that of the
arrays' type (half a step, relative).

  score   scale q k + bias is a sum of D products and a few terms in 32 bits, and
          the exponent's argument and its subtraction add a few more: an error of
          at most e = (D + 32) u (scale sum |q k| + sum |bias| + |lse| + 1), which is
          a relative error of the weight.  A weight is divided by a sum whose terms
          have such errors too: its row's mean of e.
  sums    a sum over n rows in 32 bits is off by at most (n + 64) u times the sum of
          its terms' magnitudes (however it is split).
  weights the 16-bit types round a weight to h before the second product (serving),
          or to h^2 (training); dS is rounded to h before its products.
  delta   sum_d dout out from an output kept to h^2 (h of what rounding left).

An output rounded to its type adds h times its size, and half its smallest step."""
import math

import torch

U = 2.0 ** -24
HALF_UNIT = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


# --- heads normed and turned ----------------------------------------------------------

def turn(x, pos, freq, axis, layout, inverse=False):
    """x [tokens][heads][D] (float64), the angle as the kernels round it."""
    pairs = freq.numel()
    angle = (pos.float()[:, axis.long()] * freq.float()).double()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    s = -s if inverse else s
    out = x.clone()
    one, two = ((slice(0, pairs), slice(pairs, 2 * pairs)) if layout == "halves"
                else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)))
    out[..., one] = x[..., one] * c - x[..., two] * s
    out[..., two] = x[..., two] * c + x[..., one] * s
    return out


def _mates(x, pairs, layout):
    """|x1| + |x2| of each element's pair (|x| past the pairs)."""
    m = x.abs().clone()
    one, two = ((slice(0, pairs), slice(pairs, 2 * pairs)) if layout == "halves"
                else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)))
    m[..., one] = x[..., one].abs() + x[..., two].abs()
    m[..., two] = m[..., one]
    return m


def rotary_norm(x, w, pos, freq, axis, layout, eps, dtype):
    """(out, bound).  The mean of squares is a sum of D terms in 32 bits, the root,
    the products and the turn a few roundings more."""
    x = x.double()
    D = x.shape[-1]
    w = torch.ones(D).double() if w is None else w.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r * w
    y = turn(n, pos, freq, axis, layout)
    big = _mates(n, freq.numel(), layout)
    return y, (D + 32) * U * big + HALF_UNIT[dtype] * y.abs() + TINY[dtype]


def rotary_norm_back(dy, x, w, pos, freq, axis, layout, eps, dtype):
    """((dx, dw), their bounds)."""
    x, dy = x.double(), dy.double()
    T, H, D = x.shape
    w = torch.ones(D).double() if w is None else w.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xh = x * r
    u = turn(dy, pos, freq, axis, layout, True)
    size = _mates(dy, freq.numel(), layout)
    t = u * w
    along = (t * xh).mean(-1, keepdim=True)
    dx = r * (t - xh * along)
    e = (D + 64) * U
    most = (size * w.abs() * xh.abs()).mean(-1, keepdim=True)
    dx_bound = 3 * e * r * (size * w.abs() + xh.abs() * most)
    dw = (u * xh).sum((0, 1))
    # a lane's rows in 32 bits (at most 1100 of them), then a block's groups
    rows = min(T * H, 1100) + 64
    dw_bound = (e + rows * U) * (size * xh.abs()).sum((0, 1)) + TINY[torch.float32]
    return ((dx, dw), (dx_bound + HALF_UNIT[dtype] * dx.abs() + TINY[dtype], dw_bound))


# --- attention ---------------------------------------------------------------------

def bias_rows(buckets, q_pos, k_pos):
    """Bucket of each axis, query and key: [axes][queries][keys]."""
    reach = buckets.shape[1] // 2
    out = []
    for a in range(buckets.shape[0]):
        d = k_pos[:, a].long()[None] - q_pos[:, a].long()[:, None]
        out.append(buckets[a].long()[d.clamp(-reach, reach) + reach])
    return torch.stack(out)


def attention(q, k, v, dtype, lens=None, bias=None, scale=None, dout=None, train=False):
    """{o, and with dout dq, dk, dv, dtable: (value, bound)} of q [B][Tq][H][D],
    k, v [B][Tk][Hk][D].  bias: (table, buckets, q_pos, k_pos), the positions with an
    entry's own or not."""
    B, Tq, H, D = q.shape
    Tk, Hk = k.shape[1:3]
    scale = 1 / math.sqrt(D) if scale is None else scale
    h = HALF_UNIT[dtype]
    short = dtype != torch.float32
    train = train or dout is not None
    hp = (h * h if train else h) if short else 0.0
    zero = lambda *s: torch.zeros(s, dtype=torch.float64)  # noqa: E731
    val = {"o": zero(B, Tq, H, D)}
    err = {"o": zero(B, Tq, H, D)}
    names = [("dq", (B, Tq, H, D)), ("dk", (B, Tk, Hk, D)), ("dv", (B, Tk, Hk, D))]
    if bias is not None:
        names.append(("dtable", tuple(bias[0].shape)))
    if dout is not None:
        for n, s in names:
            val[n], err[n] = zero(*s), zero(*s)
    for b in range(B):
        n = Tk if lens is None else max(0, min(Tk, int(lens[b])))
        if n == 0 or Tq == 0:
            continue
        if bias is not None:
            table, buckets, qp, kp = bias
            at = bias_rows(buckets, qp[b] if qp.dim() == 3 else qp,
                           (kp[b] if kp.dim() == 3 else kp)[:n])
        for head in range(H):
            g = head // (H // Hk)
            Q, K, V = q[b, :, head].double(), k[b, :n, g].double(), v[b, :n, g].double()
            s = scale * Q @ K.T
            most = abs(scale) * Q.abs() @ K.abs().T
            if bias is not None:
                for a in range(at.shape[0]):
                    add = table[a, :, head].double()[at[a]]
                    s, most = s + add, most + torch.where(add.isinf(), 0.0, add.abs())
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
            total = p.sum(1, keepdim=True)
            some = total > 0
            p = torch.where(some, p / total, 0.0)
            lse = torch.where(some, top + torch.log(total), 0.0)
            e = (D + 32) * U * (most + lse.abs() + 1)
            e = e + (p * e).sum(1, keepdim=True)       # relative, of a weight
            o = p @ V
            val["o"][b, :, head] = o
            sums = (n + 64) * U
            o32 = (p * (e + hp + sums)) @ V.abs()
            # (a weight below the 16-bit types' smallest is rounded to it)
            tiny = TINY[dtype] * V.abs().sum(0) if short else 0.0
            err["o"][b, :, head] = o32 + tiny + h * o.abs() + TINY[dtype]
            if dout is None:
                continue
            dO = dout[b, :, head].double()
            dp = dO @ V.T
            dpe = (D + 4) * U * dO.abs() @ V.abs().T
            delta = (dO * o).sum(1, keepdim=True)
            held = (h * h if short else 0.0) + (D + 4) * U
            de = (dO.abs() * (o32 + tiny + held * o.abs() + TINY[dtype])).sum(1, keepdim=True)
            ds = p * (dp - delta)
            dse = p * (e * (dp - delta).abs() + dpe + de) + 4 * U * ds.abs()
            small = TINY[dtype] if short else 0.0
            val["dv"][b, :n, g] += p.T @ dO
            err["dv"][b, :n, g] += (p * (e + (h if short else 0) + (Tq * (H // Hk) + 64) * U)
                                    + small).T @ dO.abs()
            val["dq"][b, :, head] = scale * ds @ K
            wide = dse + ds.abs() * ((h if short else 0) + sums) + small
            err["dq"][b, :, head] = abs(scale) * wide @ K.abs()
            val["dk"][b, :n, g] += scale * ds.T @ Q
            wide = dse + ds.abs() * ((h if short else 0) + (Tq * (H // Hk) + 64) * U) + small
            err["dk"][b, :n, g] += abs(scale) * wide.T @ Q.abs()
            if bias is not None:
                # a lane sums at most 1024 keys, a block 256 lanes, then 64 bits
                for a in range(at.shape[0]):
                    flat = at[a].reshape(-1)
                    val["dtable"][a, :, head] += zero(table.shape[1]).index_add(
                        0, flat, ds.reshape(-1))
                    err["dtable"][a, :, head] += zero(table.shape[1]).index_add(
                        0, flat, (dse + (min(n, 1024) + 320) * U * ds.abs()).reshape(-1))
    for n in ("dq", "dk", "dv"):
        if n in val:
            err[n] += h * val[n].abs() + TINY[dtype]
    if "dtable" in val:
        err["dtable"] += U * val["dtable"].abs() + TINY[torch.float32]
    return {n: (val[n], err[n]) for n in val}
