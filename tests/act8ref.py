"""Plain float64 forms of the 8-bit checkpoint and the RMS norm, for the tests of
the stand-alone operators (CPU tensors)."""
from __future__ import annotations

import torch

GROUP = 32
U32 = 2.0 ** -24        # half a float32 step, relative


def pitch(cols):
    return -(-cols // 16) * 16


def groups(cols):
    return -(-cols // GROUP)


def exponents(x):
    """s [rows][groups] of a float64 matrix, by the definition: the smallest power
    of two 2^(s-127) with rint(amax * 2^(133-s)) <= 127, within [7, 254]; 255
    where the group is not finite."""
    rows, cols = x.shape
    g = torch.zeros(rows, groups(cols) * GROUP, dtype=torch.float64)
    g[:, :cols] = x.abs()
    g = g.view(rows, groups(cols), GROUP)
    bad = ~torch.isfinite(g).all(2)
    amax = torch.where(bad, 0.0, torch.nan_to_num(g, 0, 0, 0).amax(2))
    s = torch.full(amax.shape, 254, dtype=torch.int64)
    for e in range(253, 6, -1):
        s = torch.where(torch.round(amax * 2.0 ** (133 - e)) <= 127, e, s)
    return torch.where(bad, 255, s)


def pack(x, keep_sign=False):
    """(codes [rows][pitch] int8, s [rows][groups] uint8) of a float64 matrix."""
    rows, cols = x.shape
    s = exponents(x)
    per = s.repeat_interleave(GROUP, 1)[:, :cols]
    fine = per != 255
    step = torch.exp2((per - 133).double())
    v = torch.where(fine, x, torch.zeros((), dtype=torch.float64))
    c = torch.round(v / step).clamp(-127, 127)
    if keep_sign:
        c = torch.where((c == 0) & (v != 0), torch.sign(v), c)
    codes = torch.zeros(rows, pitch(cols), dtype=torch.int8)
    codes[:, :cols] = c.to(torch.int8)
    return codes, s.to(torch.uint8)


def buffer(codes, s):
    return torch.cat([codes.reshape(-1).view(torch.uint8), s.reshape(-1)])


def split(q, rows, cols):
    p = pitch(cols)
    return q[:rows * p].view(torch.int8).view(rows, p), q[rows * p:].view(rows, groups(cols))


def values(codes, s, cols):
    per = s.long().repeat_interleave(GROUP, 1)[:, :cols]
    v = codes[:, :cols].double() * torch.exp2((per - 133).double())
    return torch.where(per == 255, torch.nan, v)


def norm(x, gamma, eps, res=None, dtype=None):
    """(h, rstd, y) in float64; h rounded to dtype after a residual addition."""
    h = x if res is None else (x + res).to(dtype).double()
    rstd = 1 / torch.sqrt((h * h).mean(1) + eps)
    return h, rstd, h * rstd[:, None] * gamma


def norm_bwd(dy, h, rstd, gamma):
    """(dx, dgamma) and the sums of their terms' magnitudes."""
    r = rstd[:, None]
    g = dy * gamma
    dx = r * (g - h * (r * r * (g * h).mean(1, keepdim=True)))
    size = r * (g.abs() + h.abs() * (r * r * (g * h).abs().mean(1, keepdim=True)))
    return dx, (dy * h * r).sum(0), size, (dy * h * r).abs().sum(0)
