"""Group norm and distillation from a teacher's top logits, as cases to be timed.

Activations are matrices of rows (the pixels of a batch, image after image) by
channels; logits are matrices of samples by classes.

  norm        group norm of a channels-last activation with an activation
              function behind it: the normalised rows and every group's mean
              and reciprocal deviation
  norm_bwd    its gradient: of the input, and of the scale and the shift
  top         what is kept of a teacher's answers: each row's k largest logits,
              their classes, and the log of what the other classes weigh
  distill     a student's loss against them (and against the labels), and the
              gradient of its logits

`run` computes them with elementary torch operations, or, with `own`, through
the library.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5


# ---------------------------------------------------------------------------
# the cases

def _norm(name, images, pixels, channels, groups, dtype, act, pitch=0):
    """pitch: elements between rows, where the activation is a slice of channels."""
    return {"name": name, "kind": "norm", "images": images, "pixels": pixels, "channels": channels, "groups": groups,
            "dtype": dtype, "act": act, "pitch": max(pitch, channels)}


def _norm_bwd(name, images, pixels, channels, groups, dtype, act, residual=False):
    """residual: the gradient that reaches the norm's input by another path is added."""
    return {"name": name, "kind": "norm_bwd", "images": images, "pixels": pixels, "channels": channels,
            "groups": groups, "dtype": dtype, "act": act, "residual": residual}


def _top(name, rows, classes, k, dtype, temperature=1.0):
    return {"name": name, "kind": "top", "rows": rows, "classes": classes, "k": k, "dtype": dtype,
            "temperature": temperature}


def _distill(name, rows, classes, k, dtype, temperature=2.0, alpha=0.7, rest=True, padded=False):
    """rest: what the teacher's other classes weigh is known (otherwise the k stand
    for all); padded: the last rows fill a batch up and count for nothing, and
    some rows list fewer than k classes."""
    return {"name": name, "kind": "distill", "rows": rows, "classes": classes, "k": k, "dtype": dtype,
            "temperature": temperature, "alpha": alpha, "rest": rest, "padded": padded}


def listed():
    return [
        # one image's 8 x 8 map: launches and latency only
        _norm("norm_one_image", 1, 8 * 8, 64, 8, "fp32", "relu"),
        # the first stage of a residual network, batch 32 at 56 pixels, mixed precision
        _norm("norm_56px_256_bf16", 32, 56 * 56, 256, 32, "bf16", "relu"),
        # 90 of the 96 channels of a full-precision map in 9 groups, an odd batch at 27 pixels
        _norm("norm_27px_slice_fp32", 75, 27 * 27, 90, 9, "fp32", "silu", pitch=96),
        # the gradient for a batch of 128 at 32 pixels, 4 channels a group, mixed precision
        _norm_bwd("norm_bwd_32px_128_bf16", 128, 32 * 32, 128, 32, "bf16", "relu"),
        # groups of 25 channels, which end inside every vector, added to a shortcut's gradient
        _norm_bwd("norm_bwd_28px_250_fp32", 32, 28 * 28, 250, 10, "fp32", "silu", residual=True),
        # a small batch's gradient: latency
        _norm_bwd("norm_bwd_8px_64", 8, 8 * 8, 64, 16, "fp32", "none"),
        # a teacher's answers to a batch of 128, 1000 classes
        _top("top_128x1000", 128, 1000, 10, "fp32"),
        # to a large batch with very many classes, mixed precision
        _top("top_4096x20000_bf16", 4096, 20000, 32, "bf16", 2.0),
        # few samples, long rows
        _top("top_8x131072", 8, 131072, 64, "fp32", 2.0),
        # a step's loss, 10 classes: latency
        _distill("distill_128x10", 128, 10, 5, "fp32", 4.0, 0.9),
        # 1000 classes, the batch filled up, short lists in it, no rest
        _distill("distill_1024x1000_padded", 1024, 1000, 16, "fp32", rest=False, padded=True),
        # a large batch with very many classes, mixed precision
        _distill("distill_4096x20000_bf16", 4096, 20000, 32, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "top", "distill"])
    dtype = rng.choice(["fp32", "bf16"])
    if kind in ("norm", "norm_bwd"):
        groups = rng.choice([1, 2, 3, 5, 8, 10, 16, 32, 32])
        channels = groups * _log(rng, 1, 2048 // groups)
        if rng.random() < 0.6:
            channels = -(-channels // (8 * groups)) * 8 * groups
        most = (25 if kind == "norm" else 16) * 10 ** 6 // channels
        least = -(-16 * groups // channels)      # pixels of a group of 16 values, the smallest that say something
        pixels = _log(rng, least, min(most, 112 * 112))
        images = _log(rng, 1, max(1, min(512, most // pixels)))
        act = rng.choice(["none", "relu", "relu", "silu"])
        if kind == "norm":
            c = _norm("", images, pixels, channels, groups, dtype, act, channels + rng.choice([0, 0, 8, 3]))
        else:
            c = _norm_bwd("", images, pixels, channels, groups, dtype, act, rng.random() < 0.4)
    else:
        classes = _log(rng, 2, 131072)
        k = _log(rng, 1, min(classes, 128))
        rows = _log(rng, 1, min(16384, 8 * 10 ** 7 // classes))
        temperature = rng.choice([1.0, 2.0, 4.0, 3.5])
        if kind == "top":
            c = _top("", rows, classes, k, dtype, temperature)
        else:
            c = _distill("", rows, classes, k, dtype, temperature, rng.choice([1.0, 0.9, 0.5]), rng.random() < 0.6,
                         rng.random() < 0.4)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs

def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _generator(seed, k):
    return torch.Generator("cuda").manual_seed(int(seed) * 1000003 + k)


def _normal(seed, k, *shape):
    return torch.randn(*shape, generator=_generator(seed, k), device="cuda")


def _activation(c, seed, k, cols):
    """N(0, 1) rows, the channels scaled by e^N(0, 0.3) and shifted by N(0, 0.5)."""
    x = _normal(seed, k, c["images"] * c["pixels"], cols)
    x *= torch.exp(0.3 * _normal(seed, k + 100, cols))
    x += 0.5 * _normal(seed, k + 200, cols)
    return x.to(_type(c))


def _logits(c, seed, k):
    """Logits as a trained classifier gives them: spread by 2, its favourite well above."""
    z = 2 * _normal(seed, k, c["rows"], c["classes"])
    best = torch.randint(c["classes"], (c["rows"], 1), generator=_generator(seed, k + 100), device="cuda")
    return z.scatter_add_(1, best, torch.full_like(best, 6, dtype=torch.float32)), best


def prepare(case, seed):
    c = dict(case)
    if c["kind"] in ("norm", "norm_bwd"):
        ch = c["channels"]
        c["gamma"] = 1 + 0.1 * _normal(seed, 3, ch)
        c["beta"] = 0.1 * _normal(seed, 4, ch)
        if c["kind"] == "norm":
            c["x"] = _activation(c, seed, 1, c["pitch"])[:, :ch]
            return c
        c["x"] = _activation(c, seed, 1, ch)
        d = c["x"].double().view(c["images"], c["pixels"], c["groups"], -1)
        mean = d.mean((1, 3), keepdim=True)
        rstd = 1 / torch.sqrt((d - mean).square().mean((1, 3), keepdim=True) + EPS)
        dy = _normal(seed, 2, c["images"] * c["pixels"], ch) * 1e-3
        if c["act"] == "relu":
            # no gradient where the ReLU's input is so near 0 that 32 and 64 bits may decide differently
            dy[(((d - mean) * rstd).view(-1, ch) * c["gamma"] + c["beta"]).abs() < 1e-4] = 0
        c["mean"], c["rstd"] = mean.float().view(c["images"], -1), rstd.float().view(c["images"], -1)
        c["dy"] = dy.to(_type(c))
        c["dres"] = (_normal(seed, 5, *dy.shape) * 1e-3).to(_type(c)) if c["residual"] else None
        return c
    z, best = _logits(c, seed, 1)
    if c["kind"] == "top":
        c["z"] = z.to(_type(c))
        return c
    # the teacher's list, and a student that half agrees with it
    rows, t = c["rows"], c["temperature"]
    values, index = torch.topk(z, c["k"], 1)
    c["z"] = (0.5 * z + _normal(seed, 2, *z.shape)).to(_type(c))
    c["values"], c["index"] = values, index.int()
    others = z.scatter_(1, index, float("-inf"))
    c["rest_mass"] = torch.logsumexp(others / t, 1) if c["rest"] else None
    c["labels"] = best[:, 0].int()
    c["weight"] = None
    if c["padded"]:
        c["weight"] = (torch.arange(rows, device="cuda") < rows - rows // 8).float()
        c["index"][::7, (c["k"] + 1) // 2:] = -1
    return c


# ---------------------------------------------------------------------------
# one pass

def _empty(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _space(n):
    """A workspace of n floats, where one is wanted."""
    return _empty(n) if n else None


def _own(c):
    from paper_2203_06638_amd import lpp
    if c["kind"] in ("norm", "norm_bwd"):
        act = {"none": lpp.ACT_NONE, "relu": lpp.ACT_RELU, "silu": lpp.ACT_SILU}[c["act"]]
        sizes = c["images"], c["pixels"], c["channels"], c["groups"]
        n, g = c["images"], c["groups"]
        out = _empty(n * c["pixels"], c["channels"], dtype=_type(c))
        if c["kind"] == "norm":
            mean, rstd = _empty(n, g), _empty(n, g)
            lpp.kernel_groupnorm(c["x"], n, g, c["gamma"], c["beta"], out, mean, rstd, _space(lpp.groupnorm_ws(*sizes)),
                                 eps=EPS, act=act)
            return {"y": out, "mean": mean, "rstd": rstd}
        dgamma, dbeta = _empty(c["channels"]), _empty(c["channels"])
        lpp.kernel_groupnorm_bwd(c["dy"], c["x"], n, g, c["gamma"], c["beta"], c["mean"], c["rstd"], out, dgamma, dbeta,
                                 _space(lpp.groupnorm_bwd_ws(*sizes)), dres=c["dres"], act=act)
        return {"dx": out, "dgamma": dgamma, "dbeta": dbeta}
    rows, classes, k = c["rows"], c["classes"], c["k"]
    if c["kind"] == "top":
        values, index, rest = _empty(rows, k), _empty(rows, k, dtype=torch.int32), _empty(rows)
        lpp.kernel_top_logits(c["z"], values, index, rest, c["temperature"], _space(lpp.top_logits_ws(rows, classes, k)))
        return {"values": values, "index": index, "rest": rest}
    loss, dz = _empty(rows), _empty(rows, classes, dtype=_type(c))
    lpp.kernel_distill(c["z"], c["values"], c["index"], loss, dz, c["rest_mass"], c["labels"], c["weight"],
                       alpha=c["alpha"], temperature=c["temperature"], scale=1 / rows,
                       ws=_space(lpp.distill_ws(rows, classes)))
    return {"loss": loss, "dz": dz}


def _per_channel(v, c):
    """[images][groups] as a factor of [images][pixels][channels]"""
    return v.repeat_interleave(c["channels"] // c["groups"], 1).unsqueeze(1)


def _lse(x):
    """log of the sum of e^x over a row; -inf for a row of -inf"""
    m = x.amax(1, keepdim=True).clamp(min=torch.finfo(x.dtype).min)
    return torch.log(torch.exp(x - m).sum(1, keepdim=True)) + m


def run(state):
    c = state
    if own:
        return _own(c)
    t = _type(c)
    if c["kind"] in ("norm", "norm_bwd"):
        n, p, ch, g = c["images"], c["pixels"], c["channels"], c["groups"]
        x = c["x"].float().reshape(n, p, ch)
        if c["kind"] == "norm":
            xg = x.view(n, p, g, ch // g)
            mean = xg.mean((1, 3))
            d = x - _per_channel(mean, c)
            var = (d * d).view(n, p, g, ch // g).mean((1, 3))
            rstd = 1 / torch.sqrt(var + EPS)
            y = d * _per_channel(rstd, c) * c["gamma"] + c["beta"]
            if c["act"] == "relu":
                y = torch.where(y > 0, y, 0)
            if c["act"] == "silu":
                y = y / (1 + torch.exp(-y))
            return {"y": y.view(n * p, ch).to(t), "mean": mean, "rstd": rstd}
        rstd = _per_channel(c["rstd"], c)
        u = (x - _per_channel(c["mean"], c)) * rstd
        dz = c["dy"].float().view(n, p, ch)
        if c["act"] != "none":
            z = u * c["gamma"] + c["beta"]
            if c["act"] == "relu":
                dz = torch.where(z > 0, dz, 0)
            else:
                s = 1 / (1 + torch.exp(-z))
                dz = dz * (s * (1 + z * (1 - s)))
        a, b = dz.sum(1), (dz * u).sum(1)
        size = p * ch // g
        s1 = (a * c["gamma"]).view(n, g, -1).sum(2) / size
        s2 = (b * c["gamma"]).view(n, g, -1).sum(2) / size
        dx = rstd * (dz * c["gamma"] - (_per_channel(s1, c) + u * _per_channel(s2, c)))
        dx = dx.view(n * p, ch)
        if c["dres"] is not None:
            dx = dx + c["dres"].float()
        return {"dx": dx.to(t), "dgamma": b.sum(0), "dbeta": a.sum(0)}
    k, temp = c["k"], c["temperature"]
    z = c["z"].float()
    if c["kind"] == "top":
        values, index = torch.sort(z, dim=1, descending=True, stable=True)   # ties: the lowest class first
        return {"values": values[:, :k].contiguous(), "index": index[:, :k].int(),
                "rest": _lse(values[:, k:] / temp)[:, 0] if k < c["classes"] else
                torch.full_like(values[:, 0], float("-inf"))}
    rows, alpha = c["rows"], c["alpha"]
    valid = c["index"] >= 0
    at = torch.where(valid, c["index"], 0).long()
    u = z / temp
    m = u.amax(1, keepdim=True)
    e = torch.exp(u - m)
    size = e.sum(1, keepdim=True)
    # the teacher's probabilities of its list, and of all other classes together
    teacher = torch.where(valid, c["values"] / temp, float("-inf"))
    if c["rest_mass"] is not None:
        teacher = torch.cat([teacher, c["rest_mass"].unsqueeze(1)], 1)
    teacher = teacher - teacher.amax(1, keepdim=True)
    logp = teacher - torch.log(torch.exp(teacher).sum(1, keepdim=True))
    p = torch.exp(logp)
    logq = (u - m).gather(1, at) - torch.log(size)
    target = torch.zeros_like(z).scatter_add_(1, at, torch.where(valid, p[:, :k], 0))
    if c["rest_mass"] is not None:
        hits = torch.zeros_like(z).scatter_add_(1, at, valid.float())
        others = torch.where(hits > 0, 0, e)
        theirs = others.sum(1, keepdim=True)
        logq = torch.cat([logq, torch.log(theirs / size)], 1)
        target = target + others / torch.where(theirs > 0, theirs, 1) * p[:, k:]
        # both sides' probabilities add up to 1: p log(p / q) - p + q, which stays exact where p is near q
        d = logp - logq
        soft = torch.where(p > 0, p * (d + torch.expm1(-d)), 0).sum(1)
    else:
        soft = torch.where(p > 0, p * (logp - logq), 0).sum(1)
    y = c["labels"].long().unsqueeze(1)
    lse = _lse(z)
    hard = (lse - z.gather(1, y))[:, 0]
    dz = torch.exp(z - lse).scatter_add_(1, y, torch.full_like(hard, -1).unsqueeze(1))
    dz = (1 - alpha) * dz + alpha * temp * (e / size - target)
    w = torch.ones_like(hard) if c["weight"] is None else c["weight"]
    return {"loss": w * ((1 - alpha) * hard + alpha * temp * temp * soft), "dz": (dz * (w / rows).unsqueeze(1)).to(t)}


def work(case):
    """Each input and output once."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] in ("norm", "norm_bwd"):
        n = c["images"] * c["pixels"] * c["channels"]
        stats = 8 * c["images"] * c["groups"]
        if c["kind"] == "norm":
            return {"bytes": 2 * n * e + stats + 8 * c["channels"], "flops": 8 * n}
        return {"bytes": n * e * (3 + c["residual"]) + stats + 16 * c["channels"], "flops": 16 * n}
    n, lists = c["rows"] * c["classes"], 8 * c["rows"] * c["k"]
    if c["kind"] == "top":
        return {"bytes": n * e + lists + 4 * c["rows"], "flops": 4 * n}
    return {"bytes": 2 * n * e + lists + c["rows"] * (8 + 4 * c["rest"] + 4 * c["padded"]), "flops": 10 * n}


# ---------------------------------------------------------------------------
# the definition in 64 bits; gradients are those that the definition's loss has

def _group_norm(x, gamma, beta, c):
    """(y, mean, rstd) of a [rows][channels] matrix of doubles"""
    n, g = c["images"], c["groups"]
    groups = x.reshape(n, c["pixels"], g, -1).transpose(1, 2).reshape(n, g, -1)
    var, mean = torch.var_mean(groups, 2, correction=0)
    rstd = torch.rsqrt(var + EPS)
    unit = ((groups - mean.unsqueeze(2)) * rstd.unsqueeze(2)).view(n, g, c["pixels"], -1).transpose(1, 2)
    y = torch.addcmul(beta, unit.reshape(x.shape), gamma)
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "silu":
        y = y * torch.sigmoid(y)
    return y, mean, rstd


def _distilled(z, c):
    """The loss of every row of a matrix of doubles, by the definition."""
    t, a = c["temperature"], c["alpha"]
    listed_ = c["index"] >= 0
    at = c["index"].clamp(min=0).long()
    teacher = (c["values"].double() / t).masked_fill(~listed_, float("-inf"))
    logq = torch.log_softmax(z / t, 1)
    mine = logq.gather(1, at)
    if c["rest_mass"] is not None:
        teacher = torch.cat([teacher, c["rest_mass"].double().unsqueeze(1)], 1)
        known = torch.zeros(z.shape, dtype=torch.int32, device=z.device).scatter_add_(1, at, listed_.int()) > 0
        tail = torch.logsumexp(logq.masked_fill(known, float("-inf")), 1, keepdim=True)
        mine = torch.cat([mine, tail], 1)
    p = torch.softmax(teacher, 1)
    soft = torch.where(p > 0, torch.xlogy(p, p) - p * mine, 0).sum(1)
    hard = -torch.log_softmax(z, 1).gather(1, c["labels"].long().unsqueeze(1)).squeeze(1)
    return (1 - a) * hard + a * t * t * soft


def exact(case, seed):
    c = prepare(case, seed)
    if c["kind"] == "norm":
        y, mean, rstd = _group_norm(c["x"].double(), c["gamma"].double(), c["beta"].double(), c)
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["kind"] == "norm_bwd":
        x, gamma, beta = (c[k].double().requires_grad_() for k in ("x", "gamma", "beta"))
        dx, dgamma, dbeta = torch.autograd.grad(_group_norm(x, gamma, beta, c)[0], (x, gamma, beta), c["dy"].double())
        return {"dx": dx if c["dres"] is None else dx + c["dres"].double(), "dgamma": dgamma, "dbeta": dbeta}
    if c["kind"] == "top":
        # the k-th largest value, and of those that equal it the first ones
        z, k = c["z"].double(), c["k"]
        border = torch.topk(z, k, 1).values[:, -1:]
        above, equal = z > border, z == border
        taken = above | (equal & (equal.cumsum(1) <= k - above.sum(1, keepdim=True)))
        index = taken.nonzero()[:, 1].view(-1, k)
        values = z.gather(1, index)
        values, order = torch.sort(values, dim=1, descending=True, stable=True)
        rest = torch.logsumexp(z.masked_fill(taken, float("-inf")) / c["temperature"], 1)
        return {"values": values, "index": index.gather(1, order).int(), "rest": rest}
    z = c["z"].double().requires_grad_()
    w = 1.0 if c["weight"] is None else c["weight"].double()
    loss = w * _distilled(z, c)
    dz, = torch.autograd.grad(loss.sum() / c["rows"], z)
    return {"loss": loss.detach(), "dz": dz}
