"""Group norm with an activation function on the GPU against float64 (tests/gnref.py, where
the tolerances are derived)."""
import math
import sys

import pytest

from paper_2203_06638_amd import lpp
from tests import gnref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
ACT = {"none": lpp.ACT_NONE, "relu": lpp.ACT_RELU, "silu": lpp.ACT_SILU}
EPS = 1e-5


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    torch.cuda.init()


# (images, pixels, channels, groups): groups of one value, of channels that end inside
# a vector, that cross slabs, rows that several workgroups share
SHAPES = [(1, 1, 1, 1), (2, 1, 4, 4), (3, 2, 5, 5), (3, 7, 6, 2), (1, 64, 64, 8), (2, 33, 96, 32), (5, 50, 90, 9),
          (3, 49, 250, 10), (1, 17, 2048, 1), (2, 9, 1100, 4), (2, 40, 1536, 3), (1, 3136, 16, 4), (300, 4, 32, 4),
          (4, 1024, 128, 32), (1, 2000, 3, 1), (7, 130, 34, 17), (2, 600, 520, 520)]


def make(seed, images, pixels, C, dtype, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(images * pixels, C, generator=g) * torch.exp(0.3 * torch.randn(C, generator=g))
    x = (x + 0.5 * torch.randn(C, generator=g) + offset).to(DT[dtype])
    gamma = 1 + 0.2 * torch.randn(C, generator=g)
    beta = 0.3 * torch.randn(C, generator=g)
    dy = (torch.randn(images * pixels, C, generator=g) * 0.01).to(DT[dtype])
    dres = (torch.randn(images * pixels, C, generator=g) * 0.01).to(DT[dtype])
    return x, gamma, beta, dy, dres


def placed(x, layout):
    """x on the GPU: contiguous, with wider rows, or at an address and row distance that
    fit no vector load; and the whole buffer behind it."""
    rows, cols = x.shape
    ld, off = {"tight": (cols, 0), "wide": (-(-cols // 8) * 8 + 8, 0), "odd": (cols + 3, 1)}[layout]
    buf = torch.full((rows * ld + off + 8,), 7.0, dtype=x.dtype, device="cuda")
    v = buf[off:off + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(x)
    return v, buf


def untouched(v, buf):
    """The elements of buf outside the matrix v are still 7."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    off = v.storage_offset()
    rows, cols = v.shape
    mask[off:off + rows * v.stride(0)].view(rows, -1)[:, :cols] = False
    return bool((buf[mask] == 7).all())


def space(n):
    """A workspace of n floats between two guards."""
    b = torch.full((n + 8,), 7.0, device="cuda")
    return b, b[:n] if n else None


def guarded(b):
    return bool((b[-8:] == 7).all())


def near(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(err[bad].max()), float((err / bound).max()))


def run_forward(x, images, groups, gamma, beta, act, layout="tight", eps=EPS):
    n, C = images, x.shape[1]
    xd, _ = placed(x, layout)
    yd, ybuf = placed(torch.full(x.shape, 5.0, dtype=x.dtype), layout)
    mean, rstd = torch.empty(n, groups, device="cuda"), torch.empty(n, groups, device="cuda")
    b, ws = space(lpp.groupnorm_ws(n, x.shape[0] // n, C, groups))
    lpp.kernel_groupnorm(xd, n, groups, gamma.cuda(), beta.cuda(), yd, mean, rstd, ws, eps=eps, act=ACT[act])
    assert untouched(yd, ybuf) and guarded(b)
    return yd, mean, rstd


@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_forward(dtype, act, layout):
    for i, (n, p, C, G) in enumerate(SHAPES):
        say("groupnorm", dtype, act, layout, n, p, C, G)
        x, gamma, beta, _, _ = make(i, n, p, C, dtype)
        y, mean, rstd = run_forward(x, n, G, gamma, beta, act, layout)
        want = R.forward(x, n, G, gamma, beta, EPS, act)
        bounds = R.forward_bounds(x, n, G, gamma, beta, EPS, act)
        for k, what in enumerate(("y", "mean", "rstd")):
            near((y, mean, rstd)[k], want[k], bounds[k], (what, n, p, C, G))


def gradient_inputs(seed, n, p, C, G, dtype, act, offset=0.0):
    x, gamma, beta, dy, dres = make(seed, n, p, C, dtype, offset)
    _, mean, rstd = R.forward(x, n, G, gamma, beta, EPS, act)
    mean, rstd = mean.float(), rstd.float()
    if act == "relu":     # no gradient where float32 and float64 may decide differently
        z, bound = R.pre_activation(x, n, G, gamma, beta, mean, rstd)
        dy[z.abs() <= bound] = 0
    return x, gamma, beta, dy, dres, mean, rstd


@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_backward(dtype, act, layout):
    for i, (n, p, C, G) in enumerate(SHAPES):
        say("groupnorm_bwd", dtype, act, layout, n, p, C, G)
        x, gamma, beta, dy, dres, mean, rstd = gradient_inputs(i, n, p, C, G, dtype, act)
        res = i % 2 == 1
        xd, yd, rd = (placed(t, layout)[0] for t in (x, dy, dres))
        dx, dbuf = placed(torch.full(x.shape, 5.0, dtype=x.dtype), layout)
        dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        b, ws = space(lpp.groupnorm_bwd_ws(n, p, C, G))
        lpp.kernel_groupnorm_bwd(yd, xd, n, G, gamma.cuda(), beta.cuda(), mean.cuda(), rstd.cuda(), dx, dg, db, ws,
                                 dres=rd if res else None, act=ACT[act])
        assert untouched(dx, dbuf) and guarded(b)
        want = list(R.backward(dy, x, n, G, gamma, beta, mean, rstd, act))
        bounds = list(R.backward_bounds(dy, x, n, G, gamma, beta, mean, rstd, act))
        if res:
            want[0] = want[0] + dres.double()
            bounds[0] = bounds[0] + R.U * want[0].abs()
        bounds[0] = bounds[0] + R.HALF[x.dtype] * (want[0].abs() + bounds[0]) + 1e-38
        for k, what in enumerate(("dx", "dgamma", "dbeta")):
            near((dx, dg, db)[k], want[k], bounds[k], (what, n, p, C, G))


@pytest.mark.parametrize("what", ["dx", "dgamma", "dbeta", "params"])
def test_backward_parts(what):
    """Each gradient alone is the same to the bit; the others are not needed."""
    n, p, C, G = 3, 70, 40, 5
    x, gamma, beta, dy, _, mean, rstd = (t.cuda() for t in gradient_inputs(1, n, p, C, G, "fp32", "silu"))

    def run(want):
        out = {"dx": torch.zeros_like(x), "dgamma": torch.zeros_like(gamma), "dbeta": torch.zeros_like(beta)}
        ws = torch.empty(lpp.groupnorm_bwd_ws(n, p, C, G), device="cuda")
        lpp.kernel_groupnorm_bwd(dy, x, n, G, gamma, beta, mean, rstd, ws=ws, act=ACT["silu"],
                                 **{k: out[k] for k in want})
        return out
    whole = run(("dx", "dgamma", "dbeta"))
    names = ("dgamma", "dbeta") if what == "params" else (what,)
    part = run(names)
    for k in whole:
        assert torch.equal(part[k], whole[k] if k in names else torch.zeros_like(whole[k])), k


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_far_mean(dtype):
    """Values about 1000 with a spread of 1: squares of values would lose the variance."""
    n, p, C, G = 2, 500, 24, 3
    x, gamma, beta, _, _ = make(3, n, p, C, dtype, 1000.0)
    got = run_forward(x, n, G, gamma, beta, "none")
    want = R.forward(x, n, G, gamma, beta, EPS, "none")
    bounds = R.forward_bounds(x, n, G, gamma, beta, EPS, "none")
    for k in range(3):
        near(got[k], want[k], bounds[k], k)
    assert float(((got[2].double().cpu() - want[2]) / want[2]).abs().max()) < 1e-4


def test_integer_sums_are_whole():
    """Small whole numbers, of which every sum is exact: one row more or less would show."""
    for n, p, C, G in [(2, 3136, 64, 4), (1, 1111, 24, 24), (3, 515, 520, 2)]:
        x = torch.randint(-3, 4, (n * p, C), generator=torch.Generator().manual_seed(p)).float()
        _, mean, rstd = run_forward(x, n, G, torch.ones(C), torch.zeros(C), "none")
        _, m, r = R.forward(x, n, G, torch.ones(C), torch.zeros(C), EPS, "none")
        # (exact sums a thread; then about 40 merges, each off by three roundings of values under 6)
        near(mean, m, 40 * 3 * R.U * 6 * torch.ones_like(m), "mean")
        near(rstd, r, 60 * 3 * R.U * r, "rstd")


def test_constant_groups_and_eps():
    n, p, C, G = 2, 90, 16, 4
    x = torch.full((n * p, C), 3.25)
    beta = torch.linspace(-1, 1, C)
    y, mean, rstd = run_forward(x, n, G, torch.ones(C), beta, "none")
    assert torch.equal(y.cpu(), beta.expand(n * p, C)) and (mean == 3.25).all()
    near(rstd, torch.full((n, G), 1 / math.sqrt(EPS), dtype=torch.float64),
         torch.full((n, G), 4 * R.U / math.sqrt(EPS), dtype=torch.float64), "rstd")
    # with eps = 0 such a group has an infinite rstd, and 0 * inf is NaN
    y, mean, rstd = run_forward(x, n, G, torch.ones(C), beta, "none", eps=0.0)
    assert torch.isinf(rstd).all() and torch.isnan(y).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_not_finite(bad):
    """An infinity or NaN makes its own group NaN (under a ReLU 0), no other."""
    n, p, C, G = 2, 300, 24, 3
    for act in ("none", "relu", "silu"):
        x, gamma, beta, _, _ = make(5, n, p, C, "fp32")
        clean = run_forward(x, n, G, gamma, beta, act)[0].cpu()
        x[p + 250, 11] = bad                       # image 1, group 1
        y, mean, rstd = run_forward(x, n, G, gamma, beta, act)
        hit = torch.zeros(n * p, C, dtype=torch.bool)
        hit[p:, 8:16] = True
        assert torch.equal(y.cpu()[~hit], clean[~hit])
        assert (y.cpu()[hit] == 0).all() if act == "relu" else torch.isnan(y.cpu()[hit]).all()
        assert torch.isnan(rstd[1, 1]) and int(torch.isnan(rstd).sum()) == 1


def test_squares_past_float32():
    n, p, C, G = 1, 600, 8, 2
    x, gamma, beta, _, _ = make(6, n, p, C, "fp32")
    x[:, :4] *= 1e25
    y, mean, rstd = run_forward(x, n, G, gamma, beta, "none")
    assert rstd[0, 0] == 0 and rstd[0, 1] > 0
    assert torch.equal(y.cpu()[:, :4], beta[:4].expand(p, 4))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_in_place(dtype):
    n, p, C, G = 3, 700, 90, 9
    x, gamma, beta, dy, dres, mean, rstd = gradient_inputs(2, n, p, C, G, dtype, "silu")
    want = run_forward(x, n, G, gamma, beta, "silu")[0]
    g, b = gamma.cuda(), beta.cuda()
    buf = x.cuda()
    lpp.kernel_groupnorm(buf, n, G, g, b, buf, ws=torch.empty(lpp.groupnorm_ws(n, p, C, G), device="cuda"),
                         act=ACT["silu"])
    assert torch.equal(buf, want)

    def back(xd, yd, rd, out):
        ws = torch.empty(lpp.groupnorm_bwd_ws(n, p, C, G), device="cuda")
        dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        lpp.kernel_groupnorm_bwd(yd, xd, n, G, g, b, mean.cuda(), rstd.cuda(), out, dg, db, ws, dres=rd,
                                 act=ACT["silu"])
        return out, dg, db
    want = back(x.cuda(), dy.cuda(), dres.cuda(), torch.empty_like(x, device="cuda"))
    for which in range(3):
        t = [x.cuda(), dy.cuda(), dres.cuda()]
        got = back(*t, t[which])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), which


# maps that take every shape of workgroup: many images, groups inside a vector, whole vectors, any
LARGE = [(100, 3136, 16, 4), (100, 3136, 32, 4), (100, 3136, 16, 16), (260, 100, 64, 2), (600, 49, 64, 32),
         (24, 784, 100, 4), (300, 196, 48, 16), (64, 1000, 40, 8), (1100, 16, 32, 8), (40, 600, 64, 32), (270, 1024, 16, 2),
         (60, 900, 24, 8), (60, 400, 24, 3), (60, 400, 32, 16), (2000, 100, 16, 2), (560, 1500, 8, 4), (520, 800, 16, 2),
         (600, 700, 16, 4)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", LARGE, ids=lambda s: "x".join(map(str, s)))
def test_large(shape, dtype):
    n, p, C, G = shape
    act = ("relu", "silu", "none")[(n + G) % 3]
    x, gamma, beta, dy, dres, mean, rstd = gradient_inputs(n, n, p, C, G, dtype, act)
    got = run_forward(x, n, G, gamma, beta, act)
    want = R.forward(x, n, G, gamma, beta, EPS, act)
    bounds = R.forward_bounds(x, n, G, gamma, beta, EPS, act)
    for k in range(3):
        near(got[k], want[k], bounds[k], ("forward", k))
    dx, dg, db = torch.empty_like(x, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    b, ws = space(lpp.groupnorm_bwd_ws(n, p, C, G))
    lpp.kernel_groupnorm_bwd(dy.cuda(), x.cuda(), n, G, gamma.cuda(), beta.cuda(), mean.cuda(), rstd.cuda(), dx, dg, db, ws,
                             act=ACT[act])
    assert guarded(b)
    want = R.backward(dy, x, n, G, gamma, beta, mean, rstd, act)
    bounds = list(R.backward_bounds(dy, x, n, G, gamma, beta, mean, rstd, act))
    bounds[0] = bounds[0] + R.HALF[x.dtype] * (want[0].abs() + bounds[0]) + 1e-38
    for k in range(3):
        near((dx, dg, db)[k], want[k], bounds[k], ("gradient", k))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_decides_as_the_forward_pass(dtype):
    """Where a ReLU let nothing through its gradient does not either, also next to 0: the output
    itself says, and dy = 1 without the statistics' terms (one value a group)."""
    n, p, C, G = 2, 1500, 16, 4
    x, gamma, beta, _, _ = make(8, n, p, C, "fp32")
    beta = -gamma * 0.25
    x = x.to(DT[dtype])
    y, mean, rstd = run_forward(x, n, G, gamma, beta, "relu")
    db = torch.empty(C, device="cuda")
    for c in range(0, C, 5):      # dbeta of a one-hot column counts its open decisions
        dy = torch.zeros_like(x)
        dy[:, c] = 1
        ws = torch.empty(lpp.groupnorm_bwd_ws(n, p, C, G), device="cuda")
        lpp.kernel_groupnorm_bwd(dy.cuda(), x.cuda(), n, G, gamma.cuda(), beta.cuda(), mean, rstd, dbeta=db, ws=ws,
                                 act=ACT["relu"])
        assert db[c] == (y[:, c] > 0).sum() and int((db != 0).sum()) <= 1


def test_no_images():
    dg, db = torch.full((12,), 5.0, device="cuda"), torch.full((12,), 5.0, device="cuda")
    z, v = torch.empty(0, 12, device="cuda"), torch.ones(12, device="cuda")
    none = torch.empty(0, 3, device="cuda")
    lpp.kernel_groupnorm(z, 0, 3, v, v, z, none, none)
    ws = torch.empty(max(1, lpp.groupnorm_bwd_ws(0, 1, 12, 3)), device="cuda")
    lpp.kernel_groupnorm_bwd(z, z, 0, 3, v, v, none, none, z, dg, db, ws)
    assert (dg == 0).all() and (db == 0).all()


def test_stream_capture_and_replays():
    """Both directions captured on a stream of their own and replayed on new inputs, with eager
    calls on another stream and another workspace in between."""
    n, p, C, G = 4, 900, 48, 6
    s = torch.cuda.Stream()
    sets = [[t.cuda() for t in gradient_inputs(k, n, p, C, G, "bf16", "relu")] for k in range(3)]
    x, gamma, beta, dy, dres, _, _ = [t.clone() for t in sets[0]]

    def run(x, gamma, beta, dy, dres, ws, wb, stream=None):
        out = [torch.empty_like(x), torch.empty(n, G, device="cuda"), torch.empty(n, G, device="cuda"),
               torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)]
        call(x, gamma, beta, dy, dres, ws, wb, out, stream)
        return out

    def call(x, gamma, beta, dy, dres, ws, wb, out, stream):
        lpp.kernel_groupnorm(x, n, G, gamma, beta, *out[:3], ws, act=ACT["relu"], stream=stream)
        lpp.kernel_groupnorm_bwd(dy, x, n, G, gamma, beta, *out[1:], wb, dres=dres, act=ACT["relu"], stream=stream)

    def spaces():
        return (torch.empty(lpp.groupnorm_ws(n, p, C, G), device="cuda"),
                torch.empty(lpp.groupnorm_bwd_ws(n, p, C, G), device="cuda"))
    eager = [run(*t[:5], *spaces()) for t in sets]
    torch.cuda.synchronize()
    out, own = [torch.empty_like(t) for t in eager[0]], spaces()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        graph.capture_begin()
        call(x, gamma, beta, dy, dres, *own, out, s)
        graph.capture_end()
    for k in (1, 0, 2, 1):
        for a, b in zip((x, gamma, beta, dy, dres), sets[k]):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        other = run(*sets[(k + 1) % 3][:5], *spaces())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[k])), k
        assert all(torch.equal(a, b) for a, b in zip(other, eager[(k + 1) % 3])), k


def test_past_two_to_31_elements():
    n, p, C, G = 33, 65536, 1000, 8
    assert n * p * C > 2 ** 31
    x = torch.empty(n * p, C, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator("cuda").manual_seed(1)
    for i in range(n):
        x[i * p:(i + 1) * p] = torch.randn(p, C, generator=g, device="cuda")
    y = torch.empty_like(x)
    gamma, beta = torch.full((C,), 1.5, device="cuda"), torch.full((C,), 0.25, device="cuda")
    mean, rstd = torch.empty(n, G, device="cuda"), torch.empty(n, G, device="cuda")
    ws = torch.empty(lpp.groupnorm_ws(n, p, C, G), device="cuda")
    lpp.kernel_groupnorm(x, n, G, gamma, beta, y, mean, rstd, ws, act=ACT["relu"])
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    last = slice((n - 1) * p, n * p)
    xd = x[last].float()
    m, r = mean[-1].repeat_interleave(C // G), rstd[-1].repeat_interleave(C // G)
    ref = xd.double().view(p, G, -1)
    assert torch.allclose(mean[-1].double(), ref.mean((0, 2)), atol=1e-6, rtol=0)
    assert torch.allclose(rstd[-1].double(), 1 / torch.sqrt(ref.var((0, 2), unbiased=False) + EPS), atol=1e-5, rtol=0)
    want = torch.relu((xd - m) * r * 1.5 + 0.25)
    assert ((y[last].float() - want).abs() <= 2.0 ** -8 * want + 1e-5).all()
    # the gradient of y in y's place
    ws = torch.empty(lpp.groupnorm_bwd_ws(n, p, C, G), device="cuda")
    lpp.kernel_groupnorm_bwd(y, x, n, G, gamma, beta, mean, rstd, y, dg, db, ws, act=ACT["relu"])
    u = (xd - m) * r
    z = u * 1.5 + 0.25
    dz = torch.where(z > 0, want.bfloat16().float(), torch.zeros_like(z))
    gz = (dz * 1.5).view(p, G, -1)
    s1 = gz.mean((0, 2)).repeat_interleave(C // G)
    s2 = (gz * u.view(p, G, -1)).mean((0, 2)).repeat_interleave(C // G)
    ref = r * (dz * 1.5 - s1 - u * s2)
    assert ((y[last].float() - ref).abs() <= 2.0 ** -8 * ref.abs() + 0.02).all()
    assert torch.isfinite(dg).all() and torch.isfinite(db).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_groups_across_slabs(dtype):
    """A group that lies in two workgroups' channels has one mean and one rstd: equal values with equal
    gamma and beta give equal outputs on both sides, those of the stored statistics, and the
    gradient's ReLU decides as the forward pass did.  (Slabs end at channel 256 and 512.)"""
    C, G, edge = (320, 32, 256) if dtype == "fp32" else (640, 32, 512)
    for n, p in ((1, 2300), (3, 3000), (2, 5001)):
        say("across slabs", dtype, n, p)
        x, gamma, beta, _, _ = make(n, n, p, C, dtype)
        beta = -0.25 * gamma
        a, b = edge - 2, edge + 1
        assert a // (C // G) == b // (C // G)
        x[:, b], gamma[b], beta[b] = x[:, a], gamma[a], beta[a]
        for act in ("none", "relu"):
            y, mean, rstd = run_forward(x, n, G, gamma, beta, act)
            assert torch.equal(y[:, a], y[:, b])
        db = torch.empty(C, device="cuda")
        ws = torch.empty(lpp.groupnorm_bwd_ws(n, p, C, G), device="cuda")
        for c in range(a - 8, edge + 8):
            dy = torch.zeros_like(x, device="cuda")
            dy[:, c] = 1
            dx = torch.empty_like(dy)
            lpp.kernel_groupnorm_bwd(dy, x.cuda(), n, G, gamma.cuda(), beta.cuda(), mean, rstd, dx, dbeta=db, ws=ws,
                                     act=ACT["relu"])
            assert db[c] == (y[:, c] > 0).sum() and int((db != 0).sum()) <= 1
            if c != a and c != b:       # (no gradient of its own: what the group's means take from both is the same)
                assert torch.equal(dx[:, a], dx[:, b])


@pytest.mark.parametrize("pixels", [40, 4000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_silu_of_large_values(dtype, pixels):
    """z / (1 + e^-z) and its derivative where e^-z, or z log2 e, is past float32: SiLU of an infinity is
    itself, of a very negative number -0, and the derivative 1 and 0.  Both kernels."""
    n, C, G = 2, 32, 4
    x, gamma, beta, dy, _ = make(4, n, pixels, C, dtype)
    big = torch.tensor([87.0, 89.0, 104.0, 1e4, 1e30, 2.3e38, 2.5e38, 3e38, math.inf])
    high, low = slice(2, 2 + len(big)), slice(16, 16 + len(big))
    beta[high], beta[low] = big, -big
    y, mean, rstd = run_forward(x, n, G, gamma, beta, "silu")
    y = y.float().cpu()
    want, _, _ = R.forward(x, n, G, gamma, beta, EPS, "silu")
    # (at 87 and more SiLU is its argument to 2^-120, whose own roundings the bounds have)
    by = R.forward_bounds(x, n, G, gamma, beta, EPS, "silu")[0]
    finite = torch.isfinite(want)
    finite[:, low] = False
    near(torch.where(finite, y, 0.0), torch.where(finite, want, 0.0), by.nan_to_num(0.0, 0.0), "y")
    assert (y[:, 2 + len(big) - 1] == math.inf).all()
    # (z is within 7 of beta; |z e^z| < 1e-32 from -80 on)
    assert (y[:, 16:16 + len(big) - 1].abs() < 1e-30).all()
    # -inf / (1 + inf)
    assert torch.isnan(y[:, 16 + len(big) - 1]).all()
    dx = torch.empty_like(x, device="cuda")
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.empty(max(1, lpp.groupnorm_bwd_ws(n, pixels, C, G)), device="cuda")
    lpp.kernel_groupnorm_bwd(dy.cuda(), x.cuda(), n, G, gamma.cuda(), beta.cuda(), mean, rstd, dx, dg, db, ws, act=ACT["silu"])
    assert torch.isfinite(dx).all() and torch.isfinite(dg).all()
    sums = dy.double().sum(0)
    # (float32 sums of 2 * pixels values)
    bound = (R.backward_bounds(dy, x, n, G, gamma, torch.zeros(C), mean.cpu(), rstd.cpu(), "none")[2])
    near(db[high], sums[high], bound[high], "dbeta")
    assert (db[low].abs() < 1e-30).all()


@pytest.mark.parametrize("pixels", [600, 6000])
def test_values_past_float32_sums(pixels):
    """Values whose sum, and whose squared deviations, float32 does not hold: the mean is theirs and
    rstd 0.  Both kernels."""
    n, C, G = 2, 8, 2
    for size in (1e34, 3e36, 1.5e38):
        x, gamma, beta, _, _ = make(6, n, pixels, C, "fp32")
        x[:, :4] = size * (1 - 0.5 * torch.rand(n * pixels, 4, generator=torch.Generator().manual_seed(1)))
        x[pixels:, :4] *= torch.where(torch.arange(pixels) % 3 == 0, -1.0, 1.0).unsqueeze(1)
        y, mean, rstd = run_forward(x, n, G, gamma, beta, "none")
        want, bound = R.forward(x, n, G, gamma, beta, EPS, "none"), R.forward_bounds(x, n, G, gamma, beta, EPS, "none")
        near(mean, want[1], bound[1], ("mean", size))
        assert (rstd[:, 0] == 0).all() and (rstd[:, 1] > 0).all()
        assert torch.equal(y.cpu()[:, :4], beta[:4].expand(n * pixels, 4))
        assert torch.isfinite(y).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(20000, 16, 32, 8), (30001, 5, 24, 3), (9000, 1, 64, 16)], ids=lambda s: "x".join(map(str, s)))
def test_many_images(shape, dtype):
    """dgamma and dbeta of tens of thousands of images, and every image's own statistics."""
    test_large(shape, dtype)
