"""Rotary positions and numbers held in 4 bits written plainly in 64 bits, on the CPU, and how far a correct kernel may be from them.

Bounds.  A rotation in fp32 (u = 2^-24): cosine and sine are rounded (u each), the product y s is, and their sum is:
  |d (x c - y s)| <= u (|x c| + 2 |y s| + |x c - y s|); bf16 results are rounded once more, by 2^-8 of their value.
A theta is a whole number of 2^-64 turns, so an angle is off by up to da = 2 pi |position| 2^-65 (1.8e-10 at 2^30, where a pair with x c close to 0 and a small y
shows it): another mscale da (|x| + |y|).
Keys on their way into 4 bits are turned in 64 bits and rounded once: equal.
"""
import decimal
import math

import torch

decimal.getcontext().prec = 50
TWO_PI = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510")
U = 2.0 ** -24
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def thetas(rot, base=10000.0):
    """To 50 digits."""
    return [(decimal.Decimal(base).ln() * -2 * i / rot).exp() for i in range(rot // 2)]


def angles(pos, theta):
    """pos[..., None] * theta modulo whole turns, to the last bit of 64: in 64 bits a product is off by position * theta * 2^-52, 2.4e-7 at 2^30."""
    at, back = torch.as_tensor(pos).unique(return_inverse=True)
    theta = [decimal.Decimal(t) for t in theta]
    rows = [[float((int(p) * t).remainder_near(TWO_PI)) for t in theta] for p in at]
    return torch.tensor(rows, dtype=torch.float64).reshape(len(at), len(theta))[back]


def pairs_of(rot, layout):
    """Indices of the pairs' first and second elements."""
    i = torch.arange(rot // 2)
    return (i, i + rot // 2) if layout == "halves" else (2 * i, 2 * i + 1)


def turn(x, pos, theta, layout, mscale=1.0, inverse=False):
    """x [..., d] turned at pos (whose sizes broadcast to x's leading ones), and the bound of the fp32 kernels."""
    x = x.double()
    rot = 2 * len(theta)
    a = angles(pos, theta)
    mscale = float(torch.tensor(mscale, dtype=torch.float32))
    c, s = a.cos() * mscale, a.sin() * (-mscale if inverse else mscale)
    da = mscale * (2 * math.pi * 2.0 ** -65 * torch.as_tensor(pos).double().abs()[..., None] + 2.0 ** -50)
    one, two = pairs_of(rot, layout)
    y, tol = x.clone(), torch.zeros_like(x)
    p, q = x[..., one], x[..., two]
    y[..., one], y[..., two] = p * c - q * s, p * s + q * c
    # either product may be the one that is rounded
    most = torch.maximum((p * c).abs() + 2 * (q * s).abs(), 2 * (p * c).abs() + (q * s).abs())
    tol[..., one] = 1.01 * U * (most + y[..., one].abs()) + da * (p.abs() + q.abs())
    most = torch.maximum((p * s).abs() + 2 * (q * c).abs(), 2 * (p * s).abs() + (q * c).abs())
    tol[..., two] = 1.01 * U * (most + y[..., two].abs()) + da * (p.abs() + q.abs())
    return y, tol


def rounded(y, tol, dtype):
    """The bound of what is stored in dtype."""
    return tol + (2.0 ** -8 * (y.abs() + tol) + 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149)


def quantise(x):
    """Codes and scale bytes of x [..., d] (float or double), number by number."""
    x = x.double()
    flat = x.reshape(-1, 32)
    codes, scales = torch.zeros(flat.shape, dtype=torch.uint8), torch.zeros(flat.shape[0], dtype=torch.uint8)
    top = flat.abs().amax(-1)
    ok = torch.isfinite(flat).all(-1)
    e = torch.full(top.shape, -120, dtype=torch.int64)
    live = ok & (top > 0)
    f, ex = torch.frexp(top[live])                                # f in [0.5, 1)
    e[live] = (ex.long() - 3 + (f > 7.25 / 8)).clamp(-120, 125)
    t = torch.where(ok[:, None], flat, torch.zeros(()).double()) * torch.exp2(-e.double())[:, None]
    levels = torch.tensor(LEVELS, dtype=torch.float64)
    far = (t.abs()[..., None] - levels).abs()
    near = far.amin(-1, keepdim=True)
    among = far == near                                          # one level, or two as near: the even code
    pick = torch.where(among, torch.where(torch.arange(8) % 2 == 0, 0, 1), 2).argmin(-1)
    codes = (pick + 8 * torch.signbit(t)).to(torch.uint8)
    codes[~ok] = 0
    scales = torch.where(ok, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales.reshape(*x.shape[:-1], -1)


def values(codes, scales):
    """What they stand for, in 64 bits."""
    levels = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64)
    x = torch.stack((levels[(codes & 15).long()], levels[(codes >> 4).long()]), -1).flatten(-2)
    unit = torch.where(scales == 255, torch.full((), math.nan, dtype=torch.float64), torch.exp2(scales.double() - 127))
    return x * unit.repeat_interleave(32, -1)


def positions(lens, row_start, seen=None):
    """(row, sequence, slot, position) of every packed row that has a slot."""
    out = []
    for b in range(len(lens)):
        r0, r1 = int(row_start[b]), int(row_start[b + 1])
        for r in range(r0, r1):
            slot = int(lens[b]) - (r1 - r)
            if slot >= 0:
                out.append((r, b, slot, slot if seen is None else int(seen[b]) - (r1 - r)))
    return out
