"""8-bit checkpoints and RMS norm on the GPU against plain float64 forms.

Tolerances.  A checkpoint is exact: codes, exponents and values equal the
definition's bit for bit.  The weight gradient multiplies exactly (a code has 7
bits, a bf16 dY 8, a float32 dY is three terms of 8 bits) and adds in float32: at
most one rounding of 2^-23 (an MFMA may truncate) of the running sum per added
term, so |error| <= (rows + splits) 2^-23 sum |dy x|.  The norm's mean of C
squares takes at most C + 2 roundings of 2^-24, half of which reaches rstd,
which adds three of its own; y two more; a bf16 result 2^-8 more.  The
gradient's terms carry those of their factors.
"""
import math
import sys

import pytest

from paper_2203_06638_amd import lpp
from tests import act8ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    torch.cuda.init()


def rand(seed, rows, cols, dtype="fp32", spread=1.0):
    """Normal values, the channels scaled by e^N(0, spread); on the CPU in the
    given type."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(cols, generator=g))
    return x.to(DT[dtype])


def placed(x, layout):
    """x on the GPU: contiguous, with wider rows, or at an address and row
    distance that fit no vector load; and the whole buffer behind it."""
    rows, cols = x.shape
    ld, off = {"tight": (cols, 0), "wide": (-(-cols // 8) * 8 + 8, 0), "odd": (cols + 3, 1)}[layout]
    buf = torch.full((rows * ld + off + 8,), 7.0, dtype=x.dtype, device="cuda")
    v = buf[off:off + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(x)
    return v, buf


def empty_like(x, layout):
    v, buf = placed(torch.full(x.shape, 5.0, dtype=x.dtype), layout)
    return v, buf


def untouched(v, buf):
    """The elements of buf outside the matrix v are still 7."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    off = v.storage_offset()
    rows, cols = v.shape
    mask[off:off + rows * v.stride(0)].view(rows, -1)[:, :cols] = False
    return bool((buf[mask] == 7).all())


SHAPES = [(1, 1), (1, 64), (3, 4), (700, 8), (900, 11), (5, 17), (5, 31), (7, 32), (9, 33), (4, 48),
          (300, 16), (1000, 90), (257, 250), (33, 1000), (2, 5000), (4097, 64)]


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_pack_unpack_exact(dtype, layout, keep):
    for k, (rows, cols) in enumerate(SHAPES):
        x = rand(k, rows, cols, dtype, 2.0)
        if k % 2:
            x = x.relu()
        x[::3] *= 1e-4
        xd, _ = placed(x, layout)
        n = lpp.act8_bytes(rows, cols)
        q = torch.full((n + 32,), 99, dtype=torch.uint8, device="cuda")
        lpp.kernel_act8_pack(xd, q[:n], keep_sign=keep)
        codes, s = R.pack(x.double(), keep)
        assert torch.equal(q[:n].cpu(), R.buffer(codes, s)), (rows, cols)
        assert (q[n:] == 99).all()
        for to in ("fp32", "bf16"):
            out, buf = empty_like(x.to(DT[to]), layout)
            lpp.kernel_act8_unpack(q[:n], out)
            assert torch.equal(out.cpu().double(), R.values(codes, s, cols)), (rows, cols, to)
            assert untouched(out, buf)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_pack_extreme_values(dtype):
    f = torch.finfo(DT[dtype])
    rows = []
    for v in (0.0, f.tiny, f.tiny / 4, 2.0 ** -120, 2.0 ** -119, 1.0, 127.0, 127.5, 127.25, 1.9921875, 1.984375, f.max,
              f.max / 2, math.inf, math.nan):
        for w in (0.0, 1.0, -v if v == v and v != math.inf else 1.0):
            rows.append([v, w, v / 3 if math.isfinite(v) else 0.5] * 15)
    x = torch.tensor(rows, dtype=torch.float64).to(DT[dtype])
    x[3::7, 44] = -math.inf
    for keep in (False, True):
        q = torch.empty(lpp.act8_bytes(*x.shape), dtype=torch.uint8, device="cuda")
        lpp.kernel_act8_pack(x.cuda(), q, keep_sign=keep)
        codes, s = R.pack(x.double(), keep)
        assert torch.equal(q.cpu(), R.buffer(codes, s))
        out = torch.empty_like(x, device="cuda")
        lpp.kernel_act8_unpack(q, out)
        want = R.values(codes, s, x.shape[1])
        got = out.cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_pack_no_rows():
    x = torch.empty(0, 40, device="cuda")
    q = torch.empty(0, dtype=torch.uint8, device="cuda")
    lpp.kernel_act8_pack(x, q)
    lpp.kernel_act8_unpack(q, x)


def test_offsets_beyond_32_bits():
    """2^31 elements and more, and (one-column rows, whole groups of lanes each)
    more than 2^31 chunks."""
    for rows, cols, dtype in ((70000, 32768, torch.bfloat16), (270000000, 1, torch.float32)):
        say("pack", rows, cols)
        x = torch.zeros(rows, cols, dtype=dtype, device="cuda")
        x[-200:] = torch.randn(200, cols, device="cuda").to(dtype)
        q = torch.empty(lpp.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        lpp.kernel_act8_pack(x, q)
        out = torch.full_like(x, 3.0)
        lpp.kernel_act8_unpack(q, out)
        codes, s = R.pack(x[-200:].cpu().double())
        p, n = R.pitch(cols), R.groups(cols)
        assert torch.equal(q[(rows - 200) * p:rows * p].cpu(), codes.reshape(-1).view(torch.uint8))
        assert torch.equal(q[rows * p + (rows - 200) * n:].cpu(), s.reshape(-1))
        assert torch.equal(out[-200:].cpu().double(), R.values(codes, s, cols))
        assert bool((out[:200] == 0).all()) and bool((out[rows // 2:rows // 2 + 200] == 0).all())
        del x, q, out
        torch.cuda.empty_cache()


# -- weight gradient -------------------------------------------------------------

def checkpoint(x, keep=False):
    codes, s = R.pack(x.double(), keep)
    return R.buffer(codes, s).cuda(), R.values(codes, s, x.shape[1])


def wgrad(dy, q, rows, cin):
    cout = dy.shape[1]
    dw = torch.full((cout, cin), 9.0, device="cuda")
    n = lpp.act8_wgrad_ws(rows, cout, cin)
    ws = torch.full((n,), math.nan, device="cuda") if n else None
    lpp.kernel_act8_wgrad(dy, q, dw, ws)
    return dw.cpu().double()


@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_wgrad(dtype, layout):
    shapes = [(0, 8, 8), (1, 1, 1), (1, 40, 24), (31, 64, 64), (33, 65, 63), (257, 16, 128), (512, 129, 130),
              (1000, 90, 36), (999, 250, 7), (300, 512, 200), (5000, 33, 250), (20000, 128, 64), (4096, 64, 64),
              (16384, 128, 512)]
    for k, (rows, cin, cout) in enumerate(shapes):
        x, dy = rand(k, rows, cin).relu(), rand(100 + k, rows, cout, dtype)
        q, xv = checkpoint(x, True)
        got = wgrad(placed(dy, layout)[0], q, rows, cin)
        want, size = dy.double().t() @ xv, dy.double().abs().t() @ xv.abs()
        err = (got - want).abs() - (rows + 64) * 2.0 ** -23 * size
        assert (err <= 1e-30).all(), (rows, cin, cout, float(err.max()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_wgrad_is_reproducible_and_small_sums_exact(dtype):
    """Integer dY and codes: every sum below 2^24 is exact, so the result equals
    the definition's bit for bit; and two calls agree bit for bit."""
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-60, 61, (700, 200), generator=g).double()
    x[:, 0::32] = 127                                   # every group's step is 1
    dy = torch.randint(-90, 91, (700, 150), generator=g).to(DT[dtype])
    q, xv = checkpoint(x)
    assert torch.equal(xv, x)
    got = wgrad(dy.cuda(), q, 700, 200)
    assert torch.equal(got, dy.double().t() @ x)
    assert torch.equal(got, wgrad(dy.cuda(), q, 700, 200))


def test_wgrad_float32_terms():
    """A float32 dY keeps all its 24 bits: one row, so that each entry is one
    product, exact to the product's own rounding."""
    dy = rand(5, 1, 300) * math.pi
    x = torch.full((1, 64), 1.0, dtype=torch.float64)
    q, xv = checkpoint(x)
    got = wgrad(dy.cuda(), q, 1, 64)
    want = dy.double().t() @ xv
    assert ((got - want).abs() <= 2 * 2.0 ** -23 * want.abs()).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_wgrad_infinities_and_nan(dtype):
    """A not finite dY reaches its own output channel only, a group of X that is
    not finite its own input channels."""
    rows, cin, cout = 100, 70, 66
    x, dy = rand(1, rows, cin), rand(2, rows, cout, dtype)
    x[:, 3] = x[:, 3].abs() + 1
    dy[17, 5], dy[40, 9], dy[41, 11] = math.inf, math.nan, -math.inf
    x[50, 40] = math.nan
    q, xv = checkpoint(x)
    got = wgrad(dy.cuda(), q, rows, cin)
    want = dy.double().t() @ xv
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    assert got[5, 3] == math.inf and got[11, 3] == -math.inf and torch.isnan(got[9]).all()
    assert torch.isnan(got[:, 32:64]).all()
    fine = torch.isfinite(want)
    size = torch.nan_to_num(dy.double(), 0, 0, 0).abs().t() @ torch.nan_to_num(xv).abs()
    assert ((got - want)[fine].abs() <= ((rows + 64) * 2.0 ** -23 * size)[fine]).all()


# -- RMS norm ------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (1, 64), (3, 7), (5, 33), (70, 128), (300, 250), (17, 500), (9, 1000), (6, 2000), (7, 3000),
               (5, 4100), (3, 9000), (2, 16384), (9000, 48), (9000, 8), (7000, 13), (3000, 20)]


def check_norm(x, gamma, eps, dtype, res, want_y, want_q, layout):
    rows, cols = x.shape
    xd = placed(x, layout)[0]
    rd = placed(res, layout)[0] if res is not None else None
    h, hb = empty_like(x, layout) if res is not None else (None, None)
    y, yb = empty_like(x, layout) if want_y else (None, None)
    q = torch.empty(lpp.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda") if want_q else None
    rstd = torch.full((rows,), 3.0, device="cuda")
    lpp.kernel_rmsnorm(xd, gamma.cuda(), rstd, eps, res=rd, h=h, y=y, q=q)
    hr, rr, yr = R.norm(x.double(), gamma.double(), eps, None if res is None else res.double(), DT[dtype])
    if res is not None:
        assert torch.equal(h.cpu().double(), hr) and untouched(h, hb)
    tol = (cols / 2 + 6) * U
    assert ((rstd.cpu().double() - rr).abs() <= tol * rr).all()
    if want_y:
        assert ((y.cpu().double() - yr).abs() <= (tol + 3 * U + HALF[dtype]) * yr.abs() + 1e-44).all()
        assert untouched(y, yb)
    if want_q:
        codes, s = R.split(q.cpu(), rows, cols)
        assert (codes[:, cols:] == 0).all()
        # the exponent is the definition's, up to magnitudes within tol of a border
        lo, hi = R.exponents(yr * (1 - 2 * tol)), R.exponents(yr * (1 + 2 * tol))
        assert ((s.long() >= lo) & (s.long() <= hi)).all()
        step = torch.exp2(s.double() - 133).repeat_interleave(32, 1)[:, :cols]
        err = (R.values(codes, s, cols) - yr).abs()
        assert (err <= step * 0.5 + 3 * tol * yr.abs()).all()


@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rmsnorm(dtype, layout):
    for k, (rows, cols) in enumerate(NORM_SHAPES):
        x, res = rand(k, rows, cols, dtype), rand(50 + k, rows, cols, dtype)
        gamma = rand(90 + k, 1, cols)[0]
        for r, wy, wq in ((None, True, False), (res, True, True), (res, False, True)):
            check_norm(x, gamma, 1e-5, dtype, r, wy, wq, layout)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rmsnorm_values(dtype):
    """Rows of zeros, of one value, of tiny and of huge values, rows that hold an
    infinity or NaN (which stay in their row), no rows; h in place of x; no rstd."""
    x = rand(1, 9, 70, dtype, 0.1)
    x[1] = 0
    x[2] = 1
    x[3] *= 1e-18
    x[4] *= 1e15
    x[5, 3] = math.inf
    x[6, 40] = math.nan
    gamma = torch.ones(70)
    xd = x.cuda()
    y, q = torch.empty_like(xd), torch.empty(lpp.act8_bytes(9, 70), dtype=torch.uint8, device="cuda")
    lpp.kernel_rmsnorm(xd, gamma.cuda(), None, 1e-5, y=y, q=q)
    _, rr, yr = R.norm(x.double(), gamma.double(), 1e-5)
    got, tol = y.cpu().double(), 64 * U + HALF[dtype]
    for r in (0, 1, 2, 3, 4, 7, 8):
        assert ((got[r] - yr[r]).abs() <= tol * yr[r].abs()).all(), r
    # an infinity makes rstd 0 and itself NaN; the others 0
    assert torch.isnan(got[5, 3]) and (got[5, :3] == 0).all() and torch.isnan(got[6]).all()
    v = torch.empty_like(xd)
    lpp.kernel_act8_unpack(q, v)
    v = v.cpu()
    assert torch.isnan(v[5, :32]).all() and (v[5, 32:] == 0).all() and torch.isnan(v[6]).all()
    assert torch.isfinite(v[[0, 1, 2, 3, 4, 7, 8]]).all()
    # the sum in place of either input
    a, b = rand(3, 40, 70, dtype), rand(4, 40, 70, dtype)
    want = (a.double() + b.double()).to(DT[dtype])
    for into in (0, 1):
        t = [a.cuda(), b.cuda()]
        lpp.kernel_rmsnorm(t[0], gamma.cuda(), None, 1e-5, res=t[1], h=t[into], y=torch.empty_like(t[0]))
        assert torch.equal(t[into].cpu(), want)
    e = torch.empty(0, 70, dtype=DT[dtype], device="cuda")
    lpp.kernel_rmsnorm(e, gamma.cuda(), torch.empty(0, device="cuda"), 1e-5, y=e)


def check_bwd(rows, cols, dtype, packed, dres, layout, seed, want=(True, True)):
    h, dy = rand(seed, rows, cols, dtype), rand(seed + 1, rows, cols, dtype)
    gamma, rs = rand(seed + 2, 1, cols)[0], rand(seed + 3, rows, cols, dtype) if dres else None
    hv = h.double()
    q = None
    if packed:
        q, hv = checkpoint(h)
    rstd = (1 / torch.sqrt((h.double() ** 2).mean(1) + 1e-5)).float()
    dx, xb = empty_like(dy, layout) if want[0] else (None, None)
    dg = torch.full((cols,), 9.0, device="cuda") if want[1] else None
    ws = torch.full((lpp.rmsnorm_bwd_ws(rows, cols),), math.nan, device="cuda") if want[1] else None
    lpp.kernel_rmsnorm_bwd(placed(dy, layout)[0], gamma.cuda(), rstd.cuda(), dx, dg, ws,
                           h=None if packed else placed(h, layout)[0], q=q,
                           dres=placed(rs, layout)[0] if dres else None)
    wx, wg, sx, sg = R.norm_bwd(dy.double(), hv, rstd.double(), gamma.double())
    if want[0]:
        tol = (cols + 12) * U * sx
        if dres:
            wx = wx + rs.double()
            tol = tol + 2 * U * rs.double().abs()
        err = (dx.cpu().double() - wx).abs() - tol - HALF[dtype] * (wx.abs() + tol)
        assert (err <= 1e-44).all(), (rows, cols, float(err.max()))
        assert untouched(dx, xb)
    if want[1]:
        err = (dg.cpu().double() - wg).abs() - (rows + 8) * U * sg
        assert (err <= 1e-44).all(), (rows, cols, float(err.max()))


@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rmsnorm_bwd(dtype, packed, layout):
    for k, (rows, cols) in enumerate(NORM_SHAPES):
        check_bwd(rows, cols, dtype, packed, k % 2 == 0, layout, 10 * k)
    check_bwd(30, 100, dtype, packed, True, layout, 7, (True, False))
    check_bwd(30, 100, dtype, packed, True, layout, 8, (False, True))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rmsnorm_bwd_edges(dtype):
    """No rows: dgamma is zero.  dx in place of dy or of dres.  A row that is not
    finite stays in its own dx."""
    t = DT[dtype]
    gamma = torch.ones(70, device="cuda")
    e = torch.empty(0, 70, dtype=t, device="cuda")
    dg, ws = torch.full((70,), 5.0, device="cuda"), torch.empty(lpp.rmsnorm_bwd_ws(0, 70), device="cuda")
    lpp.kernel_rmsnorm_bwd(e, gamma, torch.empty(0, device="cuda"), e, dg, ws, h=e)
    assert (dg == 0).all()
    h, dy, rs = (rand(k, 50, 70, dtype).cuda() for k in (1, 2, 3))
    rstd = (1 / torch.sqrt((h.double() ** 2).mean(1) + 1e-5)).float()
    dx = torch.empty_like(dy)
    lpp.kernel_rmsnorm_bwd(dy, gamma, rstd, dx, h=h, dres=rs)
    for into in (0, 1):
        a, b = dy.clone(), rs.clone()
        lpp.kernel_rmsnorm_bwd(a, gamma, rstd, (a, b)[into], h=h, dres=b)
        assert torch.equal((a, b)[into], dx)
    dy2 = dy.clone()
    dy2[7, 3], dy2[9, 0] = math.nan, math.inf
    dx2 = torch.empty_like(dy)
    lpp.kernel_rmsnorm_bwd(dy2, gamma, rstd, dx2, h=h, dres=rs)
    keep = [r for r in range(50) if r not in (7, 9)]
    assert torch.equal(dx2[keep], dx[keep]) and torch.isnan(dx2[7]).all() and not torch.isfinite(dx2[9]).any()


def test_rmsnorm_gradient_against_differences():
    """The kernel's gradient of sum(y * dy) against central differences of the
    kernel's own forward pass: the differences carry the forward's float32 error
    U |y dy| / e, the gradient its own."""
    rows, cols, e = 20, 96, 1e-2
    x, gamma, dy = rand(1, rows, cols, spread=0.2), rand(2, 1, cols, spread=0.2)[0], rand(3, rows, cols, spread=0.2)
    xd, gd, dyd = x.cuda(), gamma.cuda(), dy.cuda()
    rstd, y = torch.empty(rows, device="cuda"), torch.empty_like(xd)
    lpp.kernel_rmsnorm(xd, gd, rstd, 1e-5, y=y)
    dx, dg = torch.empty_like(xd), torch.empty(cols, device="cuda")
    lpp.kernel_rmsnorm_bwd(dyd, gd, rstd, dx, dg, torch.empty(lpp.rmsnorm_bwd_ws(rows, cols), device="cuda"), h=xd)

    def loss(xx, gg):
        out = torch.empty_like(xd)
        lpp.kernel_rmsnorm(xx, gg, None, 1e-5, y=out)
        return (out.double() * dyd.double()).sum().item()
    g = torch.Generator().manual_seed(9)
    size = (y.double() * dyd.double()).abs().sum().item()
    for _ in range(4):
        vx = torch.randn(rows, cols, generator=g).cuda()
        vg = torch.randn(cols, generator=g).cuda()
        num = (loss(xd + e * vx, gd + e * vg) - loss(xd - e * vx, gd - e * vg)) / (2 * e)
        ana = ((dx.double() * vx.double()).sum() + (dg.double() * vg.double()).sum()).item()
        # rounding of the four roundings of y and of x + e v, and e^2 / 6 of a third derivative of the size of the
        # loss (rows of unit size moved by e)
        assert abs(num - ana) <= size * (60 * U / e + 10 * e * e), (num, ana)


def test_more_than_2_31_elements():
    """Norm, its gradient and the weight gradient over matrices of 2^31 elements and
    more: everything but the last rows is zero, so that the last rows are the whole
    result."""
    t, last = torch.bfloat16, 150
    rows, cols = 140000, 16384
    assert rows * cols > 2 ** 31
    h, dy = rand(1, last, cols, "bf16"), rand(2, last, cols, "bf16")
    gamma = rand(3, 1, cols)[0]
    big = [torch.zeros(rows, cols, dtype=t, device="cuda") for _ in range(3)]
    big[0][-last:], big[1][-last:] = h.cuda(), dy.cuda()
    rstd = torch.empty(rows, device="cuda")
    q = torch.empty(lpp.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    say("norm", rows, cols)
    lpp.kernel_rmsnorm(big[0], gamma.cuda(), rstd, 1e-5, y=big[2], q=q)
    yr = R.norm(h.double(), gamma.double(), 1e-5)[2]
    tol = (cols / 2 + 9) * U + HALF["bf16"]
    assert ((big[2][-last:].cpu().double() - yr).abs() <= tol * yr.abs()).all()
    assert not big[2][:-last].any()
    lpp.kernel_act8_unpack(q, big[2])
    back = big[2][-last:].cpu().double()
    assert ((back - yr).abs() <= (0.5 / 63.5 + 1e-3) * yr.abs().amax(1, keepdim=True)).all()
    say("norm gradient", rows, cols)
    dg, ws = torch.empty(cols, device="cuda"), torch.empty(lpp.rmsnorm_bwd_ws(rows, cols), device="cuda")
    lpp.kernel_rmsnorm_bwd(big[1], gamma.cuda(), rstd, big[2], dg, ws, h=big[0])
    wx, wg, sx, sg = R.norm_bwd(dy.double(), h.double(), rstd[-last:].cpu().double(), gamma.double())
    tol = (cols + 12) * U * sx
    assert ((big[2][-last:].cpu().double() - wx).abs() <= tol + HALF["bf16"] * (wx.abs() + tol)).all()
    assert ((dg.cpu().double() - wg).abs() <= (last + 600) * U * sg + 1e-44).all()
    assert not big[2][:-last].any()
    del big, q, rstd
    torch.cuda.empty_cache()
    rows, cout, cin = 17000000, 130, 24
    assert rows * cout > 2 ** 31
    say("weight gradient", rows, cout, cin)
    d = rand(4, last, cout, "bf16")
    x = rand(5, last, cin)
    dyb = torch.zeros(rows, cout, dtype=t, device="cuda")
    dyb[-last:] = d.cuda()
    xb = torch.zeros(rows, cin, device="cuda")
    xb[-last:] = x.cuda()
    q = torch.empty(lpp.act8_bytes(rows, cin), dtype=torch.uint8, device="cuda")
    lpp.kernel_act8_pack(xb, q)
    got = wgrad(dyb, q, rows, cin)
    xv = R.values(*R.pack(x.double()), cin)
    want, size = d.double().t() @ xv, d.double().abs().t() @ xv.abs()
    assert ((got - want).abs() <= (last + 600) * 2.0 ** -23 * size).all()


# -- streams and graphs ------------------------------------------------------------

def chain(t, stream=None):
    """norm (sum, checkpoint) -> weight gradient from the checkpoint -> norm's
    gradient from h's checkpoint, as a training step uses them."""
    lpp.kernel_rmsnorm(t["x"], t["gamma"], t["rstd"], 1e-5, res=t["res"], h=t["h"], y=t["y"], q=t["q"], stream=stream)
    lpp.kernel_act8_pack(t["h"], t["hq"], stream=stream)
    lpp.kernel_act8_wgrad(t["dout"], t["q"], t["dw"], t["ws"], stream=stream)
    lpp.kernel_rmsnorm_bwd(t["dy"], t["gamma"], t["rstd"], t["dx"], t["dgamma"], t["ws2"], q=t["hq"], dres=t["dres"],
                           stream=stream)
    return [t[k] for k in ("h", "y", "q", "dw", "dx", "dgamma", "rstd")]


def chain_tensors(seed, rows=3000, cols=96, cout=40, dtype="bf16"):
    t = {k: rand(seed + i, rows, cols, dtype, 0.3).cuda() for i, k in enumerate(("x", "res", "dy", "dres"))}
    t["gamma"] = rand(seed + 9, 1, cols)[0].cuda()
    t["dout"] = rand(seed + 10, rows, cout, dtype, 0.3).cuda()
    for k in ("h", "y", "dx"):
        t[k] = torch.zeros_like(t["x"])
    for k in ("q", "hq"):
        t[k] = torch.zeros(lpp.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    t["rstd"], t["dw"], t["dgamma"] = (torch.zeros(*n, device="cuda") for n in ((rows,), (cout, cols), (cols,)))
    t["ws"] = torch.zeros(lpp.act8_wgrad_ws(rows, cout, cols), device="cuda")
    t["ws2"] = torch.zeros(lpp.rmsnorm_bwd_ws(rows, cols), device="cuda")
    return t


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_chain_against_definition(dtype):
    t = chain_tensors(1, dtype=dtype)
    chain(t)
    c = {k: v.cpu() for k, v in t.items()}
    rows, cols = c["x"].shape
    h, rr, yr = R.norm(c["x"].double(), c["gamma"].double(), 1e-5, c["res"].double(), DT[dtype])
    assert torch.equal(c["h"].double(), h)
    assert torch.equal(c["hq"], R.buffer(*R.pack(h)))
    xv = R.values(*R.split(c["q"], rows, cols), cols)
    d = c["dout"].double()
    assert ((c["dw"].double() - d.t() @ xv).abs() <= (rows + 64) * 2.0 ** -23 * (d.abs().t() @ xv.abs())).all()
    # and against the gradient from the exact y: half a step (at most amax / 127) a value
    amax = yr.abs().amax(1, keepdim=True)
    far = d.abs().t() @ (amax / 127).expand(rows, cols)
    assert ((c["dw"].double() - d.t() @ yr).abs() <= 1.01 * far).all()
    hv = R.values(*R.split(c["hq"], rows, cols), cols)
    wx, wg, sx, sg = R.norm_bwd(c["dy"].double(), hv, c["rstd"].double(), c["gamma"].double())
    wx = wx + c["dres"].double()
    tol = (cols + 12) * U * (sx + c["dres"].double().abs())
    assert ((c["dx"].double() - wx).abs() <= tol + HALF[dtype] * (wx.abs() + tol)).all()
    assert ((c["dgamma"].double() - wg).abs() <= (rows + 8) * U * sg).all()


def test_chain_on_streams_and_in_graphs():
    """Two streams at once, and a captured graph replayed with eager work between
    the replays, give the bits of the eager default-stream call."""
    a, b = chain_tensors(1), chain_tensors(50, dtype="fp32")
    want = [[v.clone() for v in chain(t)] for t in (a, b)]
    torch.cuda.synchronize()

    def clear():
        for t in (a, b):
            for v in chain_out(t):
                v.zero_()
        torch.cuda.synchronize()

    def chain_out(t):
        return [t[k] for k in ("h", "y", "q", "dw", "dx", "dgamma", "rstd")]

    def same():
        torch.cuda.synchronize()
        return all(torch.equal(x, y) for t, w in zip((a, b), want) for x, y in zip(chain_out(t), w))
    clear()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for t, s in zip((a, b), streams):
            chain(t, s)
    assert same()
    graphs = []
    for t in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            chain(t, torch.cuda.current_stream())
        graphs.append(g)
    other = chain_tensors(99)
    for _ in range(4):
        clear()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        assert same()
        chain(other)
        torch.cuda.synchronize()


def test_binding_refusals():
    x = torch.zeros(8, 40, device="cuda")
    n = lpp.act8_bytes(8, 40)
    q, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(64, device="cuda")
    calls = [lambda: lpp.kernel_act8_pack(x.half(), q), lambda: lpp.kernel_act8_pack(x.t(), q),
             lambda: lpp.kernel_act8_pack(x[0], q), lambda: lpp.kernel_act8_pack(x, q[:-1]),
             lambda: lpp.kernel_act8_pack(x, q.cpu()), lambda: lpp.kernel_act8_pack(x, v),
             lambda: lpp.kernel_act8_pack(x[:1].expand(8, 40), q),
             lambda: lpp.kernel_act8_pack(x, torch.zeros(n + 1, dtype=torch.uint8, device="cuda")[1:]),
             lambda: lpp.kernel_act8_wgrad(x, q, torch.zeros(8, 40, device="cuda")),
             # (checkpoints of 33 .. 48 columns have the same bytes)
             lambda: lpp.kernel_act8_wgrad(x, q, torch.zeros(40, 49, device="cuda")),
             lambda: lpp.kernel_rmsnorm(x, v[:39], v, y=x), lambda: lpp.kernel_rmsnorm(x, v, v[:7], y=x),
             lambda: lpp.kernel_rmsnorm(x, v, v), lambda: lpp.kernel_rmsnorm(x, v, v, y=x.bfloat16()),
             lambda: lpp.kernel_rmsnorm(x, v, v, y=x[:4]), lambda: lpp.kernel_rmsnorm(x, v.cpu(), v, y=x),
             lambda: lpp.kernel_rmsnorm_bwd(x, v, v, x), lambda: lpp.kernel_rmsnorm_bwd(x, v, v, x, h=x, q=q),
             lambda: lpp.kernel_rmsnorm_bwd(x, v, v, x, v, h=x),
             lambda: lpp.kernel_rmsnorm_bwd(x, v, v, x, v, v[:8], h=x)]
    for k, f in enumerate(calls):
        with pytest.raises(lpp.LppError) as e:
            f()
        assert e.value.code == lpp.EINVAL, k
    with pytest.raises(lpp.LppError) as e:
        y = torch.zeros(2, 16385, device="cuda")
        lpp.kernel_rmsnorm(y, torch.zeros(16385, device="cuda"), None, y=y)
    assert e.value.code == lpp.EUNSUPPORTED
