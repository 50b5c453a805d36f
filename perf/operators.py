"""8-bit activation checkpoints and RMS norm, as cases to be timed.

Activations are matrices of rows (pixels of a batch, or samples) by channels.

  checkpoint  an activation packed into 8 bits (groups of 32 channels of a row
              share a power-of-two scale) and unpacked again
  wgrad       the weight gradient dY^T X of a 1x1 conv or linear layer, X read
              from its checkpoint
  norm        RMS norm over the channels, after a residual addition if there
              is one: the sum, the normalised rows, their 8-bit checkpoint and
              the reciprocal root mean squares
  norm_bwd    its gradient, from the stored input or from that input's
              checkpoint

`run` computes them with elementary torch operations, or, with `own`, through
the library.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32      # channels that share a scale
EPS = 1e-5


# ---------------------------------------------------------------------------
# the cases

def _checkpoint(name, rows, cols, dtype, keep_sign=False, pitch=0):
    """pitch: elements between rows, where the activation is a slice of
    channels; keep_sign: a nonzero value never becomes zero (ReLU outputs)."""
    return {"name": name, "kind": "checkpoint", "rows": rows, "cols": cols, "dtype": dtype, "keep_sign": keep_sign,
            "pitch": max(pitch, cols)}


def _wgrad(name, rows, cin, cout, dtype):
    return {"name": name, "kind": "wgrad", "rows": rows, "cin": cin, "cout": cout, "dtype": dtype}


def _norm(name, rows, cols, dtype, residual=True, out=True, packed=True):
    """out: the normalised rows are wanted in the activation type; packed:
    their checkpoint is."""
    return {"name": name, "kind": "norm", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual,
            "out": out, "packed": packed}


def _norm_bwd(name, rows, cols, dtype, residual=True, packed=False):
    """residual: the gradient that reaches the norm's input by the residual
    path is added; packed: the input is read from its checkpoint."""
    return {"name": name, "kind": "norm_bwd", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual,
            "packed": packed}


def listed():
    return [
        # one sample's pooled features: launches and latency only
        _checkpoint("checkpoint_one_row", 1, 64, "fp32"),
        # a ReLU output of a batch of 32 at 56 pixels, 256 channels, mixed precision
        _checkpoint("checkpoint_56px_256_bf16", 32 * 56 * 56, 256, "bf16", keep_sign=True),
        # 90 of the 96 channels of a full-precision map, an odd batch at 27 pixels
        _checkpoint("checkpoint_slice_fp32", 75 * 27 * 27, 90, "fp32", pitch=96),
        # one row of a residual stream (a single sample at inference)
        _norm("norm_one_row_bf16", 1, 512, "bf16"),
        # the residual stream of a batch of 128 at 32 pixels, 128 channels: sum, output and checkpoint
        _norm("norm_32px_128_bf16", 128 * 32 * 32, 128, "bf16"),
        # a full-precision norm without a residual whose output is kept only as a checkpoint, odd channels
        _norm("norm_28px_250_fp32", 32 * 28 * 28, 250, "fp32", residual=False, out=False),
        # its gradient for the mixed-precision residual stream
        _norm_bwd("norm_bwd_32px_128_bf16", 128 * 32 * 32, 128, "bf16"),
        # wide rows in full precision, few of them, the input read from its checkpoint
        _norm_bwd("norm_bwd_wide_fp32", 1000, 2048, "fp32", packed=True),
        # a small batch's gradient: latency
        _norm_bwd("norm_bwd_8px_64", 8 * 8 * 8, 64, "fp32", residual=False),
        # the expanding 1x1 conv of a pointwise unit, batch 128 at 32 pixels, mixed precision
        _wgrad("wgrad_32px_128_512_bf16", 128 * 32 * 32, 128, 512, "bf16"),
        # a bottleneck's reducing 1x1 conv at 14 pixels in full precision
        _wgrad("wgrad_14px_1024_256_fp32", 32 * 14 * 14, 1024, 256, "fp32"),
        # few rows, sizes that fill no tile
        _wgrad("wgrad_odd", 333, 100, 36, "fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["checkpoint", "wgrad", "norm", "norm_bwd"])
    dtype = rng.choice(["fp32", "bf16"])
    if kind == "wgrad":
        cin, cout = _log(rng, 8, 1024), _log(rng, 8, 1024)
        if rng.random() < 0.7:
            cin, cout = -(-cin // 8) * 8, -(-cout // 8) * 8
        rows = _log(rng, 1, min(131072, 8 * 10 ** 9 // (cin * cout), 4 * 10 ** 7 // (cin + cout)))
        c = _wgrad("", rows, cin, cout, dtype)
    else:
        cols = _log(rng, 8, 4096)
        if rng.random() < 0.7:
            cols = -(-cols // 8) * 8
        rows = _log(rng, 1, 10 ** 7 // cols)
        if kind == "checkpoint":
            c = _checkpoint("", rows, cols, dtype, rng.random() < 0.5, cols + rng.choice([0, 0, 8, 3]))
        elif kind == "norm":
            out, packed = rng.choice([(True, True), (True, False), (False, True)])
            c = _norm("", rows, cols, dtype, rng.random() < 0.7, out, packed)
        else:
            c = _norm_bwd("", rows, cols, dtype, rng.random() < 0.7, rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs

def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _pitch8(cols):
    """bytes between rows of codes"""
    return -(-cols // 16) * 16


def _normal(c, seed, k, rows, cols, spread=0.0):
    """N(0, 1) rows, the channels scaled by e^N(0, spread)."""
    g = torch.Generator("cuda").manual_seed(int(seed) * 1000003 + k)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    if spread:
        x *= torch.exp(spread * torch.randn(cols, generator=g, device="cuda"))
    return x.to(_type(c))


def _groups(x):
    """[rows][groups][32] of a matrix, missing channels 0."""
    rows, cols = x.shape
    n = -(-cols // GROUP)
    return torch.nn.functional.pad(x, (0, n * GROUP - cols)).view(rows, n, GROUP)


def _quantise(x, keep_sign):
    """Codes [rows][cols] (as floats) and scales [rows][groups] (biased
    exponents) of a float32 matrix of finite values."""
    g = _groups(x)
    amax = g.abs().amax(-1)
    s = (((amax.view(torch.int32) + 0x10000) >> 23).clamp(7, 254))
    code = torch.round(g * ((260 - s) << 23).view(torch.float32).unsqueeze(-1)).clamp(-127, 127)
    if keep_sign:
        code = torch.where((code == 0) & (g != 0), torch.sign(g), code)
    return code.reshape(x.shape[0], -1)[:, :x.shape[1]], s


def _values(code, s):
    """What codes and scales stand for, float32."""
    scale = ((s.int() - 6) << 23).view(torch.float32)
    return (_groups(code) * scale.unsqueeze(-1)).reshape(code.shape[0], -1)[:, :code.shape[1]]


def _checkpoint_of(x, keep_sign):
    """The library's buffer: codes [rows][pitch], then scales [rows][groups]."""
    code, s = _quantise(x.float(), keep_sign)
    code = torch.nn.functional.pad(code, (0, _pitch8(x.shape[1]) - x.shape[1]))
    return torch.cat([code.to(torch.int8).view(torch.uint8).reshape(-1), s.to(torch.uint8).reshape(-1)])


def _split(q, rows, cols):
    """Codes (floats) and scales of such a buffer."""
    p = _pitch8(cols)
    return q[:rows * p].view(torch.int8).view(rows, p)[:, :cols].float(), q[rows * p:].view(rows, -1)


def prepare(case, seed):
    c = dict(case)
    rows = c["rows"]
    if c["kind"] == "wgrad":
        x = _normal(c, seed, 1, rows, c["cin"], 0.3).relu()
        c["q"] = _checkpoint_of(x, True)
        c["dy"] = _normal(c, seed, 2, rows, c["cout"], 0.3) * 1e-3
        return c
    cols = c["cols"]
    if c["kind"] == "checkpoint":
        x = _normal(c, seed, 1, rows, c["pitch"], 0.3)
        c["x"] = (x.relu() if c["keep_sign"] else x)[:, :cols]
        return c
    c["gamma"] = 1 + 0.1 * _normal({"dtype": "fp32"}, seed, 3, 1, cols)[0]
    if c["kind"] == "norm":
        c["x"] = _normal(c, seed, 1, rows, cols, 0.3)
        c["res"] = _normal(c, seed, 2, rows, cols, 0.3) * 2 if c["residual"] else None
        return c
    h = _normal(c, seed, 1, rows, cols, 0.3) * 2
    c["rstd"] = 1 / torch.sqrt((h.double() ** 2).mean(1) + EPS).float()
    c["h"] = None if c["packed"] else h
    c["q"] = _checkpoint_of(h, False) if c["packed"] else None
    c["dy"] = _normal(c, seed, 2, rows, cols) * 1e-3
    c["dres"] = _normal(c, seed, 4, rows, cols) * 1e-3 if c["residual"] else None
    return c


# ---------------------------------------------------------------------------
# one pass

def _empty(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _own(c):
    from paper_2203_06638_amd import lpp
    t, rows = _type(c), c["rows"]
    if c["kind"] == "checkpoint":
        x = c["x"]
        q = _empty(lpp.act8_bytes(rows, c["cols"]), dtype=torch.uint8)
        out = _empty(rows, c["cols"], dtype=t)
        lpp.kernel_act8_pack(x, q, keep_sign=c["keep_sign"])
        lpp.kernel_act8_unpack(q, out)
        return {"values": out}
    if c["kind"] == "wgrad":
        dw = _empty(c["cout"], c["cin"])
        lpp.kernel_act8_wgrad(c["dy"], c["q"], dw, _empty(lpp.act8_wgrad_ws(rows, c["cout"], c["cin"])))
        return {"dw": dw}
    cols = c["cols"]
    if c["kind"] == "norm":
        h = _empty(rows, cols, dtype=t) if c["residual"] else None
        y = _empty(rows, cols, dtype=t) if c["out"] else None
        q = _empty(lpp.act8_bytes(rows, cols), dtype=torch.uint8) if c["packed"] else None
        rstd = _empty(rows)
        lpp.kernel_rmsnorm(c["x"], c["gamma"], rstd, EPS, res=c["res"], h=h, y=y, q=q)
        values = None
        if c["packed"]:
            values = _empty(rows, cols, dtype=torch.bfloat16)
            lpp.kernel_act8_unpack(q, values)
        return {"h": h, "y": y, "values": values, "rstd": rstd}
    dx, dgamma = _empty(rows, cols, dtype=t), _empty(cols)
    lpp.kernel_rmsnorm_bwd(c["dy"], c["gamma"], c["rstd"], dx, dgamma, _empty(lpp.rmsnorm_bwd_ws(rows, cols)), h=c["h"],
                           q=c["q"], dres=c["dres"])
    return {"dx": dx, "dgamma": dgamma}


def run(state):
    c = state
    if own:
        return _own(c)
    t = _type(c)
    if c["kind"] == "checkpoint":
        return {"values": _values(*_quantise(c["x"].float(), c["keep_sign"])).to(t)}
    if c["kind"] == "wgrad":
        return {"dw": c["dy"].float().t() @ _values(*_split(c["q"], c["rows"], c["cin"]))}
    if c["kind"] == "norm":
        h = c["x"] if c["res"] is None else (c["x"].float() + c["res"].float()).to(t)
        hf = h.float()
        rstd = 1 / torch.sqrt((hf * hf).mean(1) + EPS)
        y = hf * rstd.unsqueeze(1) * c["gamma"]
        return {"h": None if c["res"] is None else h, "y": y.to(t) if c["out"] else None,
                "values": _values(*_quantise(y, False)).to(torch.bfloat16) if c["packed"] else None, "rstd": rstd}
    h = _values(*_split(c["q"], c["rows"], c["cols"])) if c["packed"] else c["h"].float()
    dy, rstd = c["dy"].float(), c["rstd"].unsqueeze(1)
    g = dy * c["gamma"]
    dx = rstd * (g - h * (rstd * rstd * (g * h).mean(1, keepdim=True)))
    if c["dres"] is not None:
        dx = dx + c["dres"].float()
    return {"dx": dx.to(t), "dgamma": (dy * (h * rstd)).sum(0)}


def work(case):
    """Each input and output once; a checkpoint is a byte a channel and one a group."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    rows = c["rows"]

    def q(cols):
        return rows * (cols + -(-cols // GROUP))

    if c["kind"] == "wgrad":
        return {"bytes": rows * c["cout"] * e + q(c["cin"]) + 4 * c["cout"] * c["cin"],
                "flops": 2 * rows * c["cout"] * c["cin"]}
    cols = c["cols"]
    n = rows * cols
    if c["kind"] == "checkpoint":     # packed, and unpacked
        return {"bytes": 2 * (n * e + q(cols)), "flops": 8 * n}
    if c["kind"] == "norm":           # a checkpoint is written, and unpacked into the values it stands for
        return {"bytes": n * e * (1 + 2 * c["residual"] + c["out"]) + 4 * (rows + cols)
                + (2 * q(cols) + 2 * n if c["packed"] else 0), "flops": 6 * n}
    return {"bytes": n * e * (2 + c["residual"]) + (q(cols) if c["packed"] else n * e) + 4 * rows + 8 * cols,
            "flops": 12 * n}


# ---------------------------------------------------------------------------
# the definition in 64 bits

def _decoded(q, rows, cols):
    """What a checkpoint stands for: code * 2^(s - 133)."""
    pitch, n = _pitch8(cols), -(-cols // GROUP)
    code = q[:rows * pitch].view(torch.int8).view(rows, pitch)[:, :cols].double()
    s = q[rows * pitch:].view(rows, n).double().repeat_interleave(GROUP, 1)[:, :cols]
    return code * torch.exp2(s - 133)


def _rounded(x, keep_sign):
    """A matrix of doubles after packing and unpacking.  The step of a group is
    the smallest power of two in which its largest magnitude rounds to 127
    steps at most; that is 2^-7 or 2^-6 of the power of two above it."""
    rows, cols = x.shape
    n = -(-cols // GROUP)
    g = torch.zeros(rows, n * GROUP, dtype=torch.float64, device=x.device)
    g[:, :cols] = x
    g = g.view(rows, n, GROUP)
    top, e = torch.frexp(g.abs().amax(2))
    e = (e - torch.where(top * 128 < 127.5, 7, 6)).clamp(-126, 121)
    step = torch.exp2(e.double()).unsqueeze(2)
    steps = torch.round(g / step)
    if keep_sign:
        steps = torch.where(steps == 0, torch.sign(g), steps)
    return (steps * step).view(rows, n * GROUP)[:, :cols]


def exact(case, seed):
    c = prepare(case, seed)
    if c["kind"] == "checkpoint":
        return {"values": _rounded(c["x"].double(), c["keep_sign"])}
    if c["kind"] == "wgrad":
        x, dy = _decoded(c["q"], c["rows"], c["cin"]), c["dy"].double()
        return {"dw": torch.mm(dy.t().contiguous(), x)}
    if c["kind"] == "norm":
        h = c["x"].double()
        if c["res"] is not None:
            h = (h + c["res"].double()).to(_type(c)).double()
        size = torch.sqrt(h.square().sum(1) / c["cols"] + EPS)
        y = h / size.unsqueeze(1) * c["gamma"].double()
        return {"h": h if c["residual"] else None, "y": y if c["out"] else None,
                "values": _rounded(y, False) if c["packed"] else None, "rstd": 1 / size}
    h = _decoded(c["q"], c["rows"], c["cols"]) if c["packed"] else c["h"].double()
    rstd, dy = c["rstd"].double().unsqueeze(1), c["dy"].double()
    unit = h * rstd
    grad = dy * c["gamma"].double()
    dx = (grad - unit * (grad * unit).sum(1, keepdim=True) / c["cols"]) * rstd
    if c["dres"] is not None:
        dx = dx + c["dres"].double()
    return {"dx": dx, "dgamma": (dy * unit).sum(0)}
