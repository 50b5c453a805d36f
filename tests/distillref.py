"""Top logits and distillation in float64, with bounds of the error that float32 sums can
make."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
INF = float("inf")


def top(z, k):
    """(values, index) of the k largest of each row; equal values: the lowest class first, a
    NaN above everything."""
    key = z.double() + 0.0
    key = torch.where(torch.isnan(key), torch.full_like(key, INF), key)
    nan = torch.isnan(z.double())
    index = torch.empty(z.shape[0], k, dtype=torch.int32)
    for r in range(z.shape[0]):
        order = sorted(range(z.shape[1]), key=lambda c: (not bool(nan[r, c]), -float(key[r, c]), c))
        index[r] = torch.tensor(order[:k], dtype=torch.int32)
    return z.float().gather(1, index.long()), index


def rest(z, index, T):
    """log of the sum of exp(z / T) over the classes that are not in index"""
    taken = torch.zeros(z.shape, dtype=torch.bool).scatter_(1, index.long(), True)
    return torch.logsumexp((z.double() / T).masked_fill(taken, -INF), 1)


def path(C):
    """Additions on the longest way of a sum over a row: 64 values a thread, then at most 12 of
    lanes and waves, and of pieces (of 8192 values at least) for longer rows."""
    return 64 + 12 + C // 8192


def rest_bound(z, index, T):
    """An exponent carries two roundings of |z / T - max| log2 e and 2^x one unit in the
    last place; log adds one, and the largest value its own.  The largest value may be
    replaced by a bound above it, relative to which the sum is at least 1, so that it is at most
    T log C higher: every exponent is that much longer.  The exponents are relative to a rounded
    bound / T; what the rounding left out is one more power and product of the sum, 3 units."""
    taken = torch.zeros(z.shape, dtype=torch.bool).scatter_(1, index.long(), True)
    u = (z.double() / T).masked_fill(taken, -INF)
    m = u.amax(1, keepdim=True)
    p = torch.softmax(u, 1)
    spread = torch.where(p > 0, p * (m - u), 0.0).sum(1)
    r = torch.logsumexp(u, 1)
    return (3 * spread + 3 * math.log(z.shape[1]) + path(z.shape[1]) + 9) * U + 4 * U * (m[:, 0].abs() + (r - m[:, 0]).abs())


def distill(z, values, index, rest=None, labels=None, weight=None, alpha=1.0, T=1.0, scale=1.0):
    """(loss, dz, bound of loss, bound of dz) in float64"""
    rows, C = z.shape
    z = z.double()
    used = (index >= 0) & (index < C)
    at = torch.where(used, index, torch.zeros_like(index)).long()
    t = (values.double() / T).masked_fill(~used, -INF)
    if rest is not None:
        t = torch.cat([t, rest.double().unsqueeze(1)], 1)
    tm = t.amax(1, keepdim=True)
    empty = (tm[:, 0] == -INF)
    p = torch.softmax(t, 1)
    p = torch.where(empty.unsqueeze(1), torch.zeros_like(p), p)
    logp = torch.log_softmax(t, 1)
    m = z.amax(1, keepdim=True)
    u = z / T
    logq = torch.log_softmax(u, 1)
    q = logq.exp()
    k = index.shape[1]
    mine = logq.gather(1, at)
    target = torch.zeros_like(z)
    for i in range(k):
        target.scatter_add_(1, at[:, i:i + 1], torch.where(used[:, i:i + 1], p[:, i:i + 1], 0.0))
    hit = torch.zeros(z.shape, dtype=torch.int32).scatter_add_(1, at, used.int()) > 0
    qr = torch.zeros(rows, 1, dtype=torch.float64)
    if rest is not None:
        tail = torch.logsumexp(logq.masked_fill(hit, -INF), 1, keepdim=True)
        mine = torch.cat([mine, tail], 1)
        qr = tail.exp()
        target = target + torch.where(hit, 0.0, q) / torch.where(qr > 0, qr, 1.0) * p[:, k:]
    soft = torch.where(p > 0, p * (logp - mine), 0.0).sum(1)
    log1 = torch.log_softmax(z, 1)
    q1 = log1.exp()
    y = torch.full((rows,), -1) if labels is None else labels.long()
    known = ((y >= 0) & (y < C))
    y0 = torch.where(known, y, 0).unsqueeze(1)
    hard = torch.where(known, -log1.gather(1, y0)[:, 0], 0.0)
    w = torch.ones(rows, dtype=torch.float64) if weight is None else weight.double()
    a1 = torch.where(known, 1 - alpha, 0.0)
    aT = torch.where(empty, 0.0, alpha * T)
    if alpha == 0:
        soft = torch.zeros_like(soft)
    if alpha == 1:
        hard = torch.zeros_like(hard)
    loss = w * (a1 * hard + aT * T * torch.where(empty, 0.0, soft))
    onehot = torch.zeros_like(z).scatter_(1, y0, known.double().unsqueeze(1))
    dz = (w * scale).unsqueeze(1) * (a1.unsqueeze(1) * (q1 - onehot) + aT.unsqueeze(1) * (q - target))
    skip = (w == 0) | ((a1 == 0) & (aT == 0))
    loss, dz = torch.where(w == 0, 0.0, loss), torch.where(skip.unsqueeze(1), 0.0, dz)
    # bounds.  A probability: its exponent's roundings and the sum's.
    S = (path(C) + k + 24) * U
    # (a class of -inf has no probability and adds no error)
    d1 = torch.where(z > -INF, m - z, 0.0)
    dT = d1 / T
    b1 = torch.where(q1 > 0, q1 * (3 * d1 * U + S), 0.0) + torch.where(q1 > 0, (q1 * 3 * d1).sum(1, keepdim=True) * U, 0.0) * q1
    e = torch.where(q > 0, q * 3 * dT * U, 0.0)
    bq = e + q * (S + e.sum(1, keepdim=True))
    tt = torch.where(p > 0, p * 3 * (tm - t) * U, 0.0)
    bp = tt + p * (S + tt.sum(1, keepdim=True))
    btarget = torch.zeros_like(z)
    for i in range(k):
        btarget.scatter_add_(1, at[:, i:i + 1], torch.where(used[:, i:i + 1], bp[:, i:i + 1], 0.0))
    if rest is not None:
        # the others' share: relative to the smaller of the list's and the rest's weights
        small = torch.minimum((target * hit).sum(1, keepdim=True) + (q * hit).sum(1, keepdim=True), p[:, k:] + qr)
        small = torch.where(p[:, k:] > 0.5, (target * hit).sum(1, keepdim=True) + (q * hit).sum(1, keepdim=True),
                            p[:, k:] + qr)
        spread = (e.sum(1, keepdim=True) + tt.sum(1, keepdim=True)) + 2 * S
        bo = torch.where(hit, 0.0, q) / torch.where(qr > 0, qr, 1.0) * small * 3 * spread
        bq = torch.where(hit, bq, bo + (q - target).abs() * (bq / torch.where(q > 0, q, 1.0)))
    bdz = (w * scale).abs().unsqueeze(1) * (a1.unsqueeze(1) * (b1 + 2 * U * (q1 + onehot))
                                            + aT.unsqueeze(1) * (bq + btarget + 3 * U * (q + target)))
    bdz = bdz + 3 * U * dz.abs()
    # logs: of sums, and differences of numbers of the list's and the logits' size
    fin = lambda v: torch.where(torch.isfinite(v), v, torch.zeros_like(v))   # noqa: E731
    size = fin((tm - t)).abs() + fin(logp).abs() + fin(mine).abs()
    size[:, :k] += (m - z).gather(1, at) / T * 2
    delta = 4 * U * (size + fin((values.double().abs().amax(1, keepdim=True) / T)) + 2) + 2 * S \
        + e.sum(1, keepdim=True) + tt.sum(1, keepdim=True)
    bsoft = torch.where(p > 0, (p + fin(mine).exp() * (p > 0)) * delta + fin(p * (logp - mine)).abs() * (S + 8 * U)
                        + bp * fin(logp - mine).abs(), 0.0).sum(1)
    bsoft = bsoft + (2 * S + 2 * e.sum(1) + 2 * tt.sum(1)) * (0 if rest is None else 1)
    bhard = 4 * U * (hard.abs() + d1.gather(1, y0)[:, 0]) + S + (q1 * 3 * d1).sum(1) * U
    bloss = w.abs() * (a1 * fin(bhard) + aT * T * bsoft) + 4 * U * fin(loss).abs()
    return loss, dz, bloss, bdz
