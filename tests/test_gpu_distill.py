"""Top logits and distillation on the GPU against float64 (tests/distillref.py, where the
tolerances are derived).  Values and classes of the top logits are exact."""
import math
import sys

import pytest

from paper_2203_06638_amd import lpp
from tests import distillref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
INF = math.inf


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    torch.cuda.init()


def logits(seed, rows, C, dtype, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    z = spread * torch.randn(rows, C, generator=g)
    best = torch.randint(C, (rows, 1), generator=g)
    return z.scatter_add(1, best, torch.full((rows, 1), 5.0)).to(DT[dtype]), best[:, 0].int()


def placed(x, layout):
    """x on the GPU: contiguous, with wider rows, or at an address and row distance that
    fit no vector load; and the whole buffer behind it."""
    rows, cols = x.shape
    ld, off = {"tight": (cols, 0), "wide": (-(-cols // 8) * 8 + 8, 0), "odd": (cols + 3, 1)}[layout]
    buf = torch.full((rows * ld + off + 8,), 99.0, dtype=x.dtype, device="cuda")
    v = buf[off:off + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(x)
    return v, buf


def untouched(v, buf):
    """The elements of buf outside the matrix v are still 99."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    off = v.storage_offset()
    rows, cols = v.shape
    mask[off:off + rows * v.stride(0)].view(rows, -1)[:, :cols] = False
    return bool((buf[mask] == 99).all())


def near(got, want, bound, what):
    got = got.double().cpu()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    err = (got - want).abs()
    bad = ~(same | (err <= bound))
    assert not bad.any(), (what, int(bad.sum()), got[bad][:3], want[bad][:3], float((err / bound)[bad].max()))


def run_top(z, k, T=1.0, layout="tight", with_rest=True):
    rows, C = z.shape
    zd, _ = placed(z, layout)
    n = lpp.top_logits_ws(rows, C, k)
    ws = torch.full((n + 8,), 7.0, device="cuda")
    values, index = torch.empty(rows, k, device="cuda"), torch.empty(rows, k, dtype=torch.int32, device="cuda")
    rest = torch.empty(rows, device="cuda") if with_rest else None
    lpp.kernel_top_logits(zd, values, index, rest, T, ws[:n] if n else None)
    assert (ws[-8:] == 7).all()
    return values.cpu(), index.cpu(), rest.cpu() if with_rest else None


def check_top(z, k, T=1.0, layout="tight"):
    values, index, rest = run_top(z, k, T, layout)
    v, i = R.top(z, k)
    assert torch.equal(index, i), (z.shape, k, (index != i).nonzero()[:3])
    assert torch.equal(torch.nan_to_num(values, nan=5e30), torch.nan_to_num(v, nan=5e30))
    near(rest, R.rest(z, i, T), R.rest_bound(z, i, T), ("rest", z.shape, k))


TOPS = [(1, 1, 1), (3, 2, 1), (5, 10, 5), (9, 100, 10), (4, 10, 10), (33, 17, 3), (7, 64, 16), (3, 128, 128), (2, 129, 128),
        (5, 100, 33), (9, 1000, 10), (3, 1000, 128), (4, 1025, 32), (2, 4097, 64), (2, 8192, 7), (2, 8193, 128),
        (1, 20000, 32), (2, 50001, 1)]


@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_top(dtype, layout):
    for n, (rows, C, k) in enumerate(TOPS):
        say("top", dtype, layout, rows, C, k)
        check_top(logits(n, rows, C, dtype)[0], k, (1.0, 2.0, 3.5)[n % 3], layout)


@pytest.mark.parametrize("T", [1e-30, 0.02, 300.0, 1e30])
def test_top_temperatures(T):
    """z / T far from 0, where its rounding is many times the distance of two logits."""
    for n, (rows, C, k) in enumerate([(9, 100, 10), (3, 1000, 40), (2, 8192, 7), (1, 60000, 32)]):
        say("top", T, rows, C, k)
        check_top(logits(n, rows, C, "fp32")[0] + 5000.0, k, T)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [10, 700, 1500, 9000, 20000])
def test_top_orders(dtype, C):
    """Ties, sorted rows, and rows laid out against the threads: all large values in a few
    threads' chunks."""
    k = min(C, 31)
    V = 4 if dtype == "fp32" else 8
    z = torch.zeros(8, C)
    z[1] = torch.arange(C).float()
    z[2] = -torch.arange(C).float()
    z[3] = (torch.arange(C) % 5).float()
    z[4] = -0.0
    z[4, C // 2:] = 0.0
    chunk = torch.arange(C) // V
    z[5] = torch.where(chunk % 64 < 16, 100.0 + (torch.arange(C) % 77), -(torch.arange(C) % 9).float())
    z[6] = torch.where(chunk % 256 < 20, 100.0 + (torch.arange(C) % 101), -(torch.arange(C) % 7).float())
    z[7] = torch.where(chunk % 64 == 5, 50.0, 0.0)
    check_top(z.to(DT[dtype]), k)
    check_top(z.to(DT[dtype]), min(C, 128))


@pytest.mark.parametrize("C", [12, 1000, 20000])
def test_top_not_finite(C):
    z = logits(1, 6, C, "fp32")[0]
    z[0] = -INF
    z[1, C // 2:] = -INF
    z[2, [3, C - 1]] = math.nan
    z[3, [2, C - 3]] = INF
    z[4, :] = -INF
    z[4, 5] = 1.0
    z[5, :11] = -math.nan
    values, index, rest = run_top(z, 10)
    v, i = R.top(z, 10)
    assert torch.equal(index, i)
    assert torch.equal(torch.nan_to_num(values, nan=5e30), torch.nan_to_num(v, nan=5e30))
    want = R.rest(z, i, 1.0)
    assert want[0] == -INF and rest[0] == -INF and rest[4] == -INF
    near(rest, want, R.rest_bound(z, i, 1.0).nan_to_num(1e-5), "rest")
    assert math.isnan(rest[5]) and not torch.isnan(rest[:5]).any()
    z[1, :] = INF        # more infinities than the list holds
    assert run_top(z, 10)[2][1] == INF


def test_top_far_favourites():
    """The others' weight is computed from their own largest value: favourites far above them do
    not make it vanish."""
    for C in (100, 3000, 30000):
        z = logits(2, 4, C, "fp32")[0]
        z[:, 7:12] += 500.0
        check_top(z, 5)


def test_top_without_rest():
    z = logits(3, 5, 12000, "bf16")[0]
    a, b = run_top(z, 9), run_top(z, 9, with_rest=False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# -- distillation ----------------------------------------------------------------

def teacher(seed, rows, C, k, T, rest):
    """A teacher's list of k classes (and rest), and the logits of a student that half agrees."""
    z, best = logits(seed, rows, C, "fp32")
    values, index = torch.topk(z, min(k, C), 1)
    others = z.scatter(1, index, -INF)
    r = torch.logsumexp(others / T, 1) if rest else None
    g = torch.Generator().manual_seed(seed + 1000)
    return 0.5 * z + torch.randn(rows, C, generator=g), values, index.int(), r, best


def run_distill(z, values, index, rest=None, labels=None, weight=None, layout="tight", grad=True, place=False, **kw):
    rows, C = z.shape
    zd, zbuf = placed(z, layout)
    dz, dbuf = (zd, zbuf) if place else placed(torch.full(z.shape, 5.0, dtype=z.dtype), layout)
    n = lpp.distill_ws(rows, C)
    ws = torch.full((n + 8,), 7.0, device="cuda")
    loss = torch.full((rows + 8,), 7.0, device="cuda")
    dev = lambda t: None if t is None else t.cuda()      # noqa: E731
    lpp.kernel_distill(zd, values.cuda(), index.cuda(), loss[:rows], dz if grad else None, dev(rest), dev(labels),
                       dev(weight), ws=ws[:n] if n else None, **kw)
    assert (ws[-8:] == 7).all() and (loss[rows:] == 7).all() and untouched(dz, dbuf)
    return loss[:rows].cpu(), dz.cpu()


def check_distill(z, values, index, rest=None, labels=None, weight=None, alpha=1.0, T=1.0, scale=1.0, layout="tight"):
    loss, dz = run_distill(z, values, index, rest, labels, weight, layout, alpha=alpha, temperature=T, scale=scale)
    want, wdz, bl, bd = R.distill(z, values, index, rest, labels, weight, alpha, T, scale)
    near(loss, want, bl + 1e-38, ("loss", z.shape, index.shape))
    near(dz, wdz, bd + R.HALF[z.dtype] * (wdz.abs() + bd) + 1e-38, ("dz", z.shape, index.shape))
    return loss, dz


DISTILLS = [(1, 1, 1), (3, 2, 1), (128, 10, 5), (5, 17, 17), (4, 64, 3), (3, 65, 20), (2, 250, 128), (6, 1000, 16),
            (3, 1001, 128), (2, 4100, 32), (2, 8192, 7), (3, 8200, 64), (1, 20000, 32), (2, 50001, 5)]


@pytest.mark.parametrize("layout", ["tight", "wide", "odd"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_distill(dtype, rest, layout):
    for n, (rows, C, k) in enumerate(DISTILLS):
        T, alpha = (1.0, 2.0, 4.0, 3.5)[n % 4], (1.0, 0.7, 0.0, 0.9, 0.5)[n % 5]
        say("distill", dtype, rest, layout, rows, C, k, T, alpha)
        z, values, index, r, best = teacher(n, rows, C, k, T, rest)
        weight = None if n % 3 else torch.linspace(-0.5, 2, rows)
        check_distill(z.to(DT[dtype]), values, index, r, best if n % 4 != 1 else None, weight, alpha, T, 1 / rows, layout)


@pytest.mark.parametrize("C", [10, 300, 3000, 20000])
@pytest.mark.parametrize("rest", [False, True])
def test_lists_of_every_kind(rest, C):
    """Entries that are not used (and hold anything), empty lists, classes listed twice, entries of
    -inf, labels inside, outside and beyond the list, rows of weight 0."""
    rows, k, T = 12, 6, 2.0
    z, values, index, r, best = teacher(5, rows, C, k, T, rest)
    index[0, 1] = -1
    values[0, 1] = math.nan
    index[1, 3:] = torch.tensor([C, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    index[2] = -1
    index[3] = -1
    index[4, 4] = index[4, 1]
    index[5, :] = index[5, 0]
    values[6, 2:] = -INF
    values[7] = -INF
    if rest:
        r[3] = -INF
        r[7] = -INF
        r[8] = -INF
    labels = best.clone()
    labels[1], labels[3], labels[9] = -1, C, -100
    labels[4] = index[4, 1]
    weight = torch.ones(rows)
    weight[10] = 0
    z[10, 3] = math.nan
    for alpha in (0.6, 1.0, 0.0):
        loss, dz = check_distill(z, values, index, r, labels, weight, alpha, T, 0.25)
        assert loss[10] == 0 and (dz[10] == 0).all()
        if alpha == 1.0:
            assert (loss[3] == 0 and (dz[3] == 0).all()) and (loss[7] == 0 and (dz[7] == 0).all())
    # all rows without labels: alpha's share alone
    check_distill(z, values, index, r, None, weight, 0.6, T, 0.25)


def test_whole_list_and_rest_of_nothing():
    """A list of all classes: the rest's student has none; it matters only if the teacher's has weight."""
    z, values, index, _, best = teacher(6, 4, 8, 8, 1.0, False)
    r = torch.tensor([-INF, -INF, 0.5, -INF])
    loss, dz = run_distill(z, values, index, r, best, alpha=0.5)
    want, wdz, bl, bd = R.distill(z, values, index, r, best, alpha=0.5)
    assert torch.isinf(loss[2]) and torch.isinf(want[2]) and torch.isfinite(dz).all()
    keep = torch.tensor([0, 1, 3])
    near(loss[keep], want[keep], bl[keep], "loss")
    near(dz, wdz, bd + R.U * wdz.abs() + 1e-38, "dz")


@pytest.mark.parametrize("C", [12, 1000, 20000])
def test_masked_and_not_finite_logits(C):
    z, values, index, r, best = teacher(7, 6, C, 4, 2.0, True)
    free = torch.ones(6, C, dtype=torch.bool).scatter_(1, index.long(), False).scatter_(1, best.long().unsqueeze(1), False)
    z[1] = torch.where(free[1] & (torch.arange(C) % 2 == 0), -INF, z[1])     # masked classes
    z[2] = torch.where(free[2], -INF, z[2])                                  # all others masked: the rest has no student
    z[3, index[3, 2].long()] = -INF                                          # a listed class masked
    z[4, C // 2] = math.nan
    z[5, C // 3] = INF
    loss, dz = run_distill(z, values, index, r, best, alpha=0.5, temperature=2.0)
    want, wdz, bl, bd = R.distill(z, values, index, r, best, alpha=0.5, T=2.0)
    # (row 2's loss is infinite unless its label, which is not masked, is one of the others)
    assert loss[3] == INF and torch.equal(torch.isinf(loss[2:4]), torch.isinf(want[2:4]))
    near(loss[:4], want[:4], bl[:4], "loss")
    assert torch.isnan(loss[4:]).all()
    near(dz[:2], wdz[:2], (bd + R.U * wdz.abs())[:2] + 1e-38, "dz")
    assert torch.isfinite(dz[2:4]).all() and torch.isnan(dz[4:]).all()
    assert (dz[1][z[1] == -INF] == 0).all() and (dz[2][z[2] == -INF] == 0).all()
    none = torch.full((2, C), -INF)
    loss, dz = run_distill(none, values[:2], index[:2], r[:2], best[:2], alpha=0.5)
    assert torch.isnan(loss).all() and torch.isnan(dz).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("C", [10, 2000, 20000])
def test_student_is_teacher(C, rest):
    """Where the student's answer is the teacher's own, loss and gradient vanish: the loss keeps
    to the square of the rounding errors where the list and the rest cover every class."""
    z, values, index, r, _ = teacher(8, 5, C, 6, 3.0, True)
    full = z * 2
    values, index = torch.topk(full, 6, 1)
    r = torch.logsumexp(full.scatter(1, index, -INF) / 3.0, 1) if rest else None
    if not rest:
        full = torch.full_like(full, -INF).scatter(1, index, values)
    loss, dz = check_distill(full, values, index.int(), r, alpha=1.0, T=3.0)
    assert loss.abs().max() < (1e-9 if rest else 1e-5)


def test_gradient_against_differences():
    """The loss's own differences along random directions, in float64 of the float32 kernel's
    losses: a step of 2^-6 leaves e^2 / 6 of the third derivative (under 1) and rounding 2^-20 / e."""
    z, values, index, r, best = teacher(9, 64, 30, 5, 2.0, True)
    kw = dict(alpha=0.6, temperature=2.0)
    _, dz = run_distill(z, values, index, r, best, **kw)
    g = torch.Generator().manual_seed(2)
    e = 2.0 ** -6
    for _ in range(4):
        v = torch.randn(z.shape, generator=g)
        v /= v.norm(dim=1, keepdim=True)
        up, down = (run_distill(z + s * e * v, values, index, r, best, **kw)[0].double() for s in (1, -1))
        err = ((up - down) / (2 * e) - (dz.double() * v).sum(1)).abs().max()
        assert err < e * e + 2.0 ** -19 / e, err


@pytest.mark.parametrize("C", [10, 1000, 20000, 70000])
def test_in_place_and_loss_alone(C):
    z, values, index, r, best = teacher(11, 6, C, 9, 2.0, True)
    for dtype in ("fp32", "bf16"):
        x = z.to(DT[dtype])
        kw = dict(alpha=0.7, temperature=2.0, scale=0.5)
        loss, dz = run_distill(x, values, index, r, best, layout="odd", **kw)
        again, same = run_distill(x, values, index, r, best, layout="odd", place=True, **kw)
        assert torch.equal(loss, again) and torch.equal(dz, same)
        only, kept = run_distill(x, values, index, r, best, layout="odd", grad=False, **kw)
        assert torch.equal(loss, only) and (kept == 5).all()


@pytest.mark.parametrize("C", [70, 6000, 12001, 16000, 30000, 32768])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_of_every_length(dtype, C):
    """Lengths between the others' that take other shapes of workgroups, in few rows and in many;
    rows of the same content have the same answer, to the bit."""
    z, values, index, r, best = teacher(12, 3, C, 12, 2.0, True)
    z = z.to(DT[dtype])
    check_top(z, 12, 2.0)
    many = (torch.arange(2051 if C < 20000 else 2048) * 7) % 3
    zd = z[many].cuda()
    v, i, rest = (torch.empty(len(many), 12, device="cuda"), torch.empty(len(many), 12, dtype=torch.int32, device="cuda"),
                  torch.empty(len(many), device="cuda"))
    n = lpp.top_logits_ws(len(many), C, 12)
    lpp.kernel_top_logits(zd, v, i, rest, 2.0, torch.empty(n, device="cuda") if n else None)
    tv, ti = R.top(z, 12)
    assert torch.equal(i.cpu(), ti[many]) and torch.equal(v.cpu(), tv[many])
    near(rest, R.rest(z, ti, 2.0)[many], R.rest_bound(z, ti, 2.0)[many], "rest")
    for T, alpha in ((2.0, 0.6), (4.0, 0.6), (3.0, 0.6), (2.5, 1.0)):
        check_distill(z, values, index, r, best, None, alpha, T, 0.5)
        loss, dz = torch.empty(len(many), device="cuda"), torch.empty_like(zd)
        n = lpp.distill_ws(len(many), C)
        lpp.kernel_distill(zd, values[many].cuda(), index[many].cuda(), loss, dz, r[many].cuda(), best[many].cuda(),
                           alpha=alpha, temperature=T, scale=0.5, ws=torch.empty(n, device="cuda") if n else None)
        want, wdz, bl, bd = R.distill(z, values, index, r, best, None, alpha, T, 0.5)
        near(loss, want[many], bl[many], "loss")
        for k in range(3):
            same = dz[(many == k).cuda()]
            assert (same == same[0]).all()
            near(same[0], wdz[k], bd[k] + R.HALF[z.dtype] * (wdz[k].abs() + bd[k]) + 1e-38, "dz")


def test_no_rows():
    z, v, i = torch.empty(0, 9, device="cuda"), torch.empty(0, 3, device="cuda"), torch.empty(0, 3, dtype=torch.int32, device="cuda")
    e = torch.empty(0, device="cuda")
    lpp.kernel_top_logits(z, v, i, e)
    lpp.kernel_distill(z, v, i, e, z, e)


@pytest.mark.parametrize("C", [100, 30000])
def test_teacher_to_student_captured(C):
    """A teacher's top logits and the student's loss on them, as they are used together: captured on
    a stream of their own and replayed on new logits, with eager calls on others in between."""
    rows, k, T = 12, 20, 2.0
    s = torch.cuda.Stream()
    sets = [(logits(n, rows, C, "fp32")[0].cuda(), logits(n + 50, rows, C, "bf16")[0].cuda()) for n in range(3)]
    labels = logits(0, rows, C, "fp32")[1].cuda()

    def spaces():
        return [torch.empty(max(1, n), device="cuda") for n in (lpp.top_logits_ws(rows, C, k), lpp.distill_ws(rows, C))]

    def outputs():
        return [torch.empty(rows, k, device="cuda"), torch.empty(rows, k, dtype=torch.int32, device="cuda"),
                torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"),
                torch.empty(rows, C, dtype=torch.bfloat16, device="cuda")]

    def call(t, z, out, ws, stream=None):
        lpp.kernel_top_logits(t, *out[:3], temperature=T, ws=ws[0], stream=stream)
        lpp.kernel_distill(z, out[0], out[1], out[3], out[4], out[2], labels, alpha=0.8, temperature=T, scale=1 / rows,
                           ws=ws[1], stream=stream)
        return out
    eager = [call(*t, outputs(), spaces()) for t in sets]
    torch.cuda.synchronize()
    # the first set against float64
    t, z = (x.cpu() for x in sets[0])
    v, i = R.top(t, k)
    assert torch.equal(eager[0][1].cpu(), i)
    want, wdz, bl, bd = R.distill(z, v, i, eager[0][2].cpu(), labels.cpu(), None, 0.8, T, 1 / rows)
    near(eager[0][3], want, bl, "loss")
    near(eager[0][4], wdz, bd + 2.0 ** -8 * (wdz.abs() + bd) + 1e-38, "dz")
    t, z = (x.clone() for x in sets[0])
    out, own = outputs(), spaces()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        graph.capture_begin()
        call(t, z, out, own, s)
        graph.capture_end()
    for n in (1, 0, 2, 1):
        t.copy_(sets[n][0])
        z.copy_(sets[n][1])
        torch.cuda.synchronize()
        graph.replay()
        other = call(*sets[(n + 1) % 3], outputs(), spaces())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[n])), n
        assert all(torch.equal(a, b) for a, b in zip(other, eager[(n + 1) % 3])), n


def test_past_two_to_31_elements():
    rows, C, k = 65600, 33000, 4
    assert rows * C > 2 ** 31
    z = torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda")
    at = (torch.arange(rows, device="cuda").unsqueeze(1) * 7919 + torch.tensor([11, 20011, 503, 32999], device="cuda")) % C
    z.scatter_(1, at, torch.tensor([8.0, 7.0, 6.0, 5.0], device="cuda", dtype=torch.bfloat16).expand(rows, k))
    values, index = torch.empty(rows, k, device="cuda"), torch.empty(rows, k, dtype=torch.int32, device="cuda")
    rest = torch.empty(rows, device="cuda")
    n = lpp.top_logits_ws(rows, C, k)
    lpp.kernel_top_logits(z, values, index, rest, 1.0, torch.empty(max(1, n), device="cuda"))
    assert torch.equal(index.long(), at)
    assert (values == torch.tensor([8.0, 7.0, 6.0, 5.0], device="cuda")).all()
    assert (rest - math.log(C - k)).abs().max() < 1e-4
    loss = torch.empty(rows, device="cuda")
    n = lpp.distill_ws(rows, C)
    lpp.kernel_distill(z, values, index, loss, z, rest, ws=torch.empty(max(1, n), device="cuda"))
    # the student is the teacher: nothing to learn
    assert loss.abs().max() < 1e-6 and z[-1].float().abs().max() < 1e-5 and z[0].float().abs().max() < 1e-5


@pytest.mark.parametrize("C", [6, 100, 700, 3000, 20000, 70000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_student_far_favourites(dtype, C):
    """A listed class of the student so far above all others that their exponentials relative to it are 0
    in float32: the rest's loss and the unlisted classes' gradients are those of the logits all the same.
    Rows of one workgroup and rows in pieces; the label the favourite, another class or none.  (An
    exponential relative to the favourite that is under 2^-126 may count as 0, with the gradient's
    factors: of the hard term, and of the soft one where the list stands for all.)"""
    rows, k, scale = 12, 3, 0.5
    gap = torch.tensor([60.0, 86.0, 88.0, 89.5, 100.0, 103.0, 104.5, 110.0, 150.0, 300.0, 500.0, 650.0])
    for n, (T, alpha, labelled) in enumerate([(1.0, 1.0, 0), (2.0, 0.6, 1), (4.0, 0.5, 1), (3.0, 0.7, 1), (1.0, 0.3, 1),
                                              (10.0, 1.0, 0), (3.0, 0.0, 1)]):
        for rest in (True, False):
            say("far favourites", dtype, C, T, alpha, rest)
            z, values, index, r, best = teacher(40 + n, rows, C, k, T, rest)
            labels = best.clone()
            labels[::4] = (index[::4, -1] + 1) % C
            labels[1::4] = index[1::4, 0]
            labels = labels if labelled else None
            z = z.scatter(1, index[:, :1].long(), (z.amax(1) + gap * max(1.0, T)).unsqueeze(1)).to(DT[dtype])
            loss, dz = run_distill(z, values, index, r, labels, alpha=alpha, temperature=T, scale=scale)
            want, wdz, bl, bd = R.distill(z, values, index, r, labels, None, alpha, T, scale)
            near(loss, want, bl + 1e-38, ("loss", T, alpha, rest))
            flushed = 2.0 ** -126 * (2 + scale * (1 - alpha + alpha * T))
            near(dz, wdz, bd + R.HALF[z.dtype] * (wdz.abs() + bd) + flushed, ("dz", T, alpha, rest))


def test_student_far_favourite_by_hand():
    """10 classes, one listed at 100 and the others at 0; the teacher gives the rest 31 of 100."""
    z = torch.zeros(1, 10)
    z[0, 4] = 100.0
    values, index = torch.full((1, 1), math.log(0.69)), torch.full((1, 1), 4, dtype=torch.int32)
    loss, dz = run_distill(z, values, index, torch.full((1,), math.log(0.31)))
    # p log(p / q): q = 1 and 9 e^-100
    want = 0.69 * math.log(0.69) + 0.31 * (math.log(0.31) - math.log(9) + 100)
    assert abs(loss.item() - want) < 40 * R.U * want
    assert abs(dz[0, 4].item() - 0.31) < 8 * R.U and (dz[0, :4] + 0.31 / 9).abs().max() < 8 * R.U / 9


@pytest.mark.parametrize("T", [2.0 ** -60, 1e-6, 0.05, 2.0 ** 60])
def test_distill_temperatures_of_the_range(T):
    """Down to where a softmax is its largest class, and up to the border, where the answers stay finite.

    The bounds of tests/distillref.py take the teacher's exponents to be off as their differences are, which
    holds for T of about 1 and more.  values * (1 / T) has two roundings, 2 U |values| / T each way; p is
    softmax of these (and rest, which is exact), so that it is off by at most twice that of itself:
    dz by scale * alpha * T * 4 U max |values| / T * p, for the classes that are not listed their share of
    the rest's."""
    for n, (rows, C, k) in enumerate([(9, 10, 5), (4, 1000, 40), (2, 20000, 16), (2, 70000, 9)]):
        say("distill", T, rows, C, k)
        z, values, index, r, best = teacher(80 + n, rows, C, k, T, True)
        p = torch.softmax(torch.cat([values.double() / T, r.double().unsqueeze(1)], 1), 1)
        others = torch.softmax((z.double() / T).scatter(1, index.long(), -INF), 1) * p[:, k:]
        target = others.scatter(1, index.long(), p[:, :k])
        for alpha in (1.0, 0.6):
            loss, dz = run_distill(z, values, index, r, best, alpha=alpha, temperature=T, scale=1 / rows)
            assert torch.isfinite(loss).all() and torch.isfinite(dz).all()
            if T < 1:
                want, wdz, bl, bd = R.distill(z, values, index, r, best, None, alpha, T, 1 / rows)
                near(loss, want, bl, "loss")
                more = alpha / rows * 4 * R.U * values.abs().amax(1, keepdim=True) * target
                near(dz, wdz, bd + more + R.U * (wdz.abs() + bd) + 1e-38, "dz")


@pytest.mark.parametrize("T", [10.0, 20.0, 100.0, 1000.0])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_high_temperatures(T, rest):
    """T^2 times a loss of about (spread / T)^2 / 2, which keeps its digits: also with a list of all
    classes and no rest."""
    for n, (rows, C, k) in enumerate([(9, 10, 10), (9, 10, 5), (5, 100, 100), (4, 1000, 40), (2, 20000, 128), (2, 70000, 9)]):
        say("distill", T, rest, rows, C, k)
        z, values, index, r, best = teacher(60 + n, rows, C, k, T, rest)
        for alpha in (1.0, 0.6):
            check_distill(z, values, index, r, best, None, alpha, T, 1 / rows)
        if k == C:
            # a term p (d + e^-d - 1), d = log(p / q), moves by p - q of what d is off (and its square).
            # That is: quotients of numbers under 16 (two roundings each) and their differences (under 24), 200 / T
            # in all; the two logs (of at most C and at least 1) and what they are added to, 8 log C; the
            # sums in them, 16 additions or exponentials each, and expm1's last digits: 40.  p itself is off by
            # about as much of the term.
            loss, _ = run_distill(z, values, index, r, temperature=T)
            want = R.distill(z, values, index, r, None, None, 1.0, T)[0]
            e = (200 / T + 8 * math.log(C) + 40) * R.U
            p = torch.softmax(values.double() / T, 1)
            q = torch.softmax(z.double() / T, 1).gather(1, index.long())
            near(loss, want, T * T * (2 * e * (p - q).abs().sum(1) + e * e) + 2 * e * want, "loss")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_length_is_launched(dtype):
    """Lengths on both sides of each number of a thread's chunks, in one row and in many: all outputs are
    written, whatever the temperature makes of the exponentials."""
    V = 4 if dtype == "fp32" else 8
    lanes = [16 * n for n in (1, 2)] + [64 * n for n in (1, 2, 4)] + [256 * n for n in (1, 2, 4, 6, 8, 10, 12, 16)] \
        + [512 * n for n in (4, 5, 6, 8, 12, 16)] + [40000]
    sizes = sorted({C for n in lanes for C in (n * V, n * V + 1) if C <= 41000})
    most = torch.randn(2048 * 41000, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(DT[dtype])
    for C in sizes:
        for rows in (1, 2048):
            z = most[:rows * C].view(rows, C)
            for k in (5, 33):
                k = min(k, C)
                v, i = torch.full((rows, k), math.nan, device="cuda"), torch.full((rows, k), -1, dtype=torch.int32, device="cuda")
                r = torch.full((rows,), math.nan, device="cuda")
                n = lpp.top_logits_ws(rows, C, k)
                lpp.kernel_top_logits(z, v, i, r, 1.0, torch.empty(n, device="cuda") if n else None)
                assert not v.isnan().any() and (i >= 0).all() and (i < C).all() and not r.isnan().any(), (C, rows, k)
            labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
            n = lpp.distill_ws(rows, C)
            ws = torch.empty(n, device="cuda") if n else None
            dz = torch.empty_like(z)
            for T in (1.0, 2.0, 3.0, 4.0):
                loss = torch.full((rows,), math.nan, device="cuda")
                dz.fill_(math.nan)
                lpp.kernel_distill(z, v, i, loss, dz, r, labels, alpha=0.5, temperature=T, ws=ws)
                assert torch.isfinite(loss).all() and torch.isfinite(dz).all(), (C, rows, T)
