"""Group norm with an activation function, and its gradient, in float64, with bounds of
the error that float32 sums can make."""
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def wide(v, C):
    """[images][groups] -> [images][1][C]"""
    return v.repeat_interleave(C // v.shape[1], 1).unsqueeze(1)


def forward(x, images, groups, gamma, beta, eps, name):
    """(y, mean, rstd) of x [rows][C]"""
    n, C = images, x.shape[1]
    xg = x.double().reshape(n, -1, groups, C // groups)
    mean = xg.mean((1, 3))
    var = (xg - mean[:, None, :, None]).square().mean((1, 3))
    rstd = 1 / torch.sqrt(var + eps)
    u = (x.double().reshape(n, -1, C) - wide(mean, C)) * wide(rstd, C)
    return act(u * gamma.double() + beta.double(), name).reshape(x.shape), mean, rstd


def backward(dy, x, images, groups, gamma, beta, mean, rstd, name):
    """(dx, dgamma, dbeta) from given statistics"""
    n, C = images, x.shape[1]
    x3, dy3 = x.double().reshape(n, -1, C), dy.double().reshape(n, -1, C)
    r = wide(rstd.double(), C)
    u = (x3 - wide(mean.double(), C)) * r
    dz = dy3 * act_grad(u * gamma.double() + beta.double(), name)
    g = dz * gamma.double()

    def group_mean(t):
        return wide(t.reshape(n, -1, groups, C // groups).mean((1, 3)), C)
    dx = r * (g - (group_mean(g) + u * group_mean(g * u)))
    return dx.reshape(x.shape), (dz * u).sum((0, 1)), dz.sum((0, 1))


def thread_rows(pixels, C):
    """Rows that a thread of the kernels sums at most: 256 threads, a power of two of them, 64
    at most, to a row."""
    lanes = 1
    while lanes < 64 and lanes * 4 < C:
        lanes *= 2
    return min(1025, -(-pixels * lanes // 256))


def forward_bounds(x, images, groups, gamma, beta, eps, name):
    """(y, mean, rstd): how far float32 results may be off.

    A thread adds n differences from a value k of the group, and their squares; means and
    squared deviations of about 40 parts are merged after that, two roundings each.
    With d the largest |x - mean|, |x - k| <= 2 d: the mean is off by (n + 80) U 2 d and
    its own rounding, twice (k + e, merges), the variance by (n + 80) U times the mean of
    (x - k)^2 <= 2 (var + d^2)."""
    n, C = images, x.shape[1]
    y, mean, rstd = forward(x, images, groups, gamma, beta, eps, name)
    xg = x.double().reshape(n, -1, groups, C // groups)
    dev = (xg - mean[:, None, :, None]).abs()
    d, var = dev.amax((1, 3)), dev.square().mean((1, 3))
    L = thread_rows(xg.shape[1], C) + 80
    bm = (2 * L * d + 3 * mean.abs()) * U
    # (the mean's own error reaches the variance in its square only)
    bv = L * U * 2 * (var + d * d) + bm * bm
    br = rstd * (bv / 2 * rstd * rstd + 4 * U)
    r = wide(rstd, C)
    u = (x.double().reshape(n, -1, C) - wide(mean, C)) * r
    gamma, beta = gamma.double(), beta.double()
    bz = gamma.abs() * (u.abs() * (wide(br, C) / r + 3 * U) + wide(bm, C) * r) + (u * gamma + beta).abs() * U
    # (no activation function is steeper than 1.1; SiLU's own roundings: 6)
    by = 1.1 * bz + 6 * U * y.reshape(u.shape).abs() + HALF[x.dtype] * (y.reshape(u.shape).abs() + 1.1 * bz)
    return by.reshape(x.shape) + 1e-38, bm + 1e-38, br


def pre_activation(x, images, groups, gamma, beta, mean, rstd):
    """z, and how far a float32 z may be off"""
    n, C = images, x.shape[1]
    u = (x.double().reshape(n, -1, C) - wide(mean.double(), C)) * wide(rstd.double(), C)
    z = u * gamma.double() + beta.double()
    return z.reshape(x.shape), ((3 * (u * gamma.double()).abs() + z.abs()) * U).reshape(x.shape)


def backward_bounds(dy, x, images, groups, gamma, beta, mean, rstd, name):
    """(dx, dgamma, dbeta): u carries two roundings, dz SiLU's (its derivative moves by at most
    half of z's error; 8 of its own); a sum adds those of its n terms a thread, then of the
    waves, of the group's channels and of the splits."""
    n, C = images, x.shape[1]
    pixels = x.shape[0] // n
    x3, dy3 = x.double().reshape(n, -1, C), dy.double().reshape(n, -1, C)
    r, gamma = wide(rstd.double(), C), gamma.double()
    u = (x3 - wide(mean.double(), C)) * r
    z, bz = pre_activation(x, images, groups, gamma, beta, mean, rstd)
    z, bz = z.reshape(u.shape), bz.reshape(u.shape)
    dz = dy3 * act_grad(z, name)
    bdz = dy3.abs() * (0.5 * bz + 8 * U * (1 + z.abs())) if name == "silu" else torch.zeros_like(dz)
    L = (thread_rows(pixels, C) + C // groups + 300) * U

    def group_mean(t):
        return wide(t.reshape(n, -1, groups, C // groups).mean((1, 3)), C)
    g = dz * gamma
    b1 = group_mean(bdz * gamma.abs() + L * g.abs())
    b2 = group_mean((bdz * gamma.abs() + (L + 3 * U) * g.abs()) * u.abs())
    s1, s2 = group_mean(g), group_mean(g * u)
    bdx = r * (bdz * gamma.abs() + 3 * U * g.abs() + b1 + u.abs() * (b2 + 4 * U * s2.abs()) + 2 * U * s1.abs())
    dx = r * (g - (s1 + u * s2))
    bdx = bdx + 3 * U * dx.abs()
    K = L + n / 16 * U
    return (bdx.reshape(x.shape), ((bdz + (K + 3 * U) * dz.abs()) * u.abs()).sum((0, 1)) + 1e-38,
            (bdz + K * dz.abs()).sum((0, 1)) + 1e-38)
