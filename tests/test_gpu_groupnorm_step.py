"""Group norm layers and distillation inside lpp_step, against the same layer lists in float64
PyTorch with autograd (CPU), at the bars of the other networks."""
import math
import sys

import numpy as np
import pytest

import synth
from paper_2203_06638_amd import lpp
from paper_2203_06638_amd import models as PM
from tests import distillref as D
from tests import parity as PR

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    torch.cuda.init()


def inputs(model, batch, seed, bf16=False):
    c, h, w = model.in_shape
    img = synth.images(seed, batch, c, h, w)
    if bf16:
        img = synth.round_to_bf16(img)
    lab = synth.labels(seed, batch, model.n_classes)
    x = synth.init_params(model.specs, seed)
    rng, pos, tensors = np.random.default_rng(seed), 0, []
    for kind, n, _ in model.specs:
        if kind not in ("conv_w", "linear_w"):      # gammas about 1, shifts about 0
            x[pos:pos + n] += (0.1 * rng.standard_normal(n)).astype(np.float32)
        tensors.append((kind, pos, n))
        pos += n
    return img, lab, x, tensors


def reference(model, img, lab, x, teacher=None, eps=1e-5):
    """(loss, logits, gradient) in float64; teacher: (values, index, rest, alpha, T)."""
    F = torch.nn.functional
    p = torch.from_numpy(x.astype(np.float64)).requires_grad_()
    pos, outs = 0, []

    def take(*shape):
        nonlocal pos
        n = math.prod(shape)
        pos += n
        return p[pos - n:pos].view(*shape)
    for op, a, b, cin, cout, k, stride, pad, bias, _ in model.layers:
        t = outs[a] if a >= 0 else torch.from_numpy(img.astype(np.float64))
        if op == lpp.CONV:
            w = take(cout, cin, k, k)
            t = F.conv2d(t, w, take(cout) if bias else None, stride, pad)
        elif op == lpp.GROUPNORM:
            s = t.reshape(t.shape[0], k, -1)
            m, v = s.mean(2, keepdim=True), s.var(2, unbiased=False, keepdim=True)
            t = ((s - m) / torch.sqrt(v + eps)).view(t.shape) * take(cout).view(1, -1, 1, 1) + take(cout).view(1, -1, 1, 1)
        elif op == lpp.BN:
            m, v = t.mean((0, 2, 3), keepdim=True), t.var((0, 2, 3), unbiased=False, keepdim=True)
            t = (t - m) / torch.sqrt(v + eps) * take(cout).view(1, -1, 1, 1) + take(cout).view(1, -1, 1, 1)
        elif op == lpp.RMSNORM:
            t = t / torch.sqrt((t * t).mean(1, keepdim=True) + eps) * take(cout).view(1, -1, 1, 1)
        elif op == lpp.RELU:
            t = t.relu()
        elif op == lpp.ADD:
            t = t + outs[b]
        elif op == lpp.CONCAT:
            t = torch.cat([t, outs[b]], 1)
        elif op == lpp.MAXPOOL:
            t = F.max_pool2d(t, k, stride, pad)
        elif op == lpp.GAP:
            t = t.mean((2, 3), keepdim=True)
        elif op == lpp.LINEAR:
            w = take(cout, cin)
            t = (t.flatten(1) @ w.t() + take(cout)).view(-1, cout, 1, 1)
        else:
            raise AssertionError(op)
        outs.append(t)
    z = outs[-1].flatten(1)
    if teacher is None:
        loss = F.cross_entropy(z, torch.from_numpy(lab.astype(np.int64)))
    else:
        values, index, rest, alpha, T = teacher
        loss = D.distill(z, values, index, rest, torch.from_numpy(lab.astype(np.int32)), None, alpha, T)[0].mean()
    loss.backward()
    return loss.item(), z.detach().numpy(), p.grad.numpy()


def step(model, img, lab, x, part=0, dtype=lpp.FP32, steps=1, teacher=None, plain_first=False, **kw):
    """(loss, logits, gradient) of a step at parameters x, which is repeated there with
    steps > 1 (replays); plain_first: a step without the teacher goes before each."""
    im, lb = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    with lpp.Context(model, K=1, batch=len(lab), dtype=dtype, **kw) as ctx:
        for _ in range(steps):
            if plain_first:
                ctx.set_params(x)
                ctx.step(0, im, lb, part, 0.1)
            ctx.set_params(x)
            if teacher is None:
                ctx.step(0, im, lb, part, 0.1)
            else:
                v, i, r, alpha, T = teacher
                ctx.step_distill(0, im, lb, v.cuda(), i.cuda(), part, 0.1, None if r is None else r.cuda(), alpha, T)
            ctx.sync()
        return ctx.get_loss(0), ctx.get_logits(0), ctx.get_grad(0)


def resnet(act=True, groups=4, blocks=None):
    return PM.resnet_cifar(8, (16, 32, 32), 10, 12, blocks or [1, 2, 2, 3, 3], act, groups)


def wired():
    """Group norms of a conv, of a sum, of a norm, of a ReLU, of a pool and of a concat; one tensor read
    by two norms; one group, and a group for each channel."""
    m = PM.Model("wired", (3, 12, 12), 10)
    a = m.conv(-1, 16, 3, bias=True)
    b = m.conv(m.groupnorm(a, 16), 16, 3)
    m.new_unit()
    s = m.add(b, a)
    n1, n2 = m.groupnorm(s, 1), m.groupnorm(m.relu(m.groupnorm(s, 4)), 2)
    c = m.concat(m.conv(n1, 16, 1, 1, 0, bias=True), m.groupnorm(n2, 8))
    m.new_unit()
    d = m.maxpool(m.groupnorm(c, 4), 2, 2, 0)
    e = m.conv(m.groupnorm(d, 8), 24, 3)
    f = m.add(m.groupnorm(e, 3), m.groupnorm(e, 6))
    m.new_unit()
    m.linear(m.gap(m.relu(m.groupnorm(f, 2))), 10)
    return m.assign_blocks([1, 2, 3, 3])


def check(model, got, want, tensors, lo, hi, what):
    loss, z, g = want
    assert abs(got[0] - loss) <= 1e-5 * abs(loss), what
    assert PR.relerr(got[1], z, PR.TAU_LOGITS) <= PR.TOL_LOGITS, what
    for kind, at, n in tensors:
        if at >= lo and at + n <= hi:
            assert PR.relerr(got[2][at:at + n], g[at:at + n], PR.TAU) <= PR.TOL_GRAD, (what, kind, at)
    assert not got[2][:lo].any() and not got[2][hi:].any()


@pytest.mark.parametrize("unfused", [False, True])
def test_resnet_against_float64(unfused):
    m = resnet(act=False)
    img, lab, x, tensors = inputs(m, 6, 3)
    check(m, step(m, img, lab, x, unfused=unfused), reference(m, img, lab, x), tensors, 0, len(x), unfused)


@pytest.mark.parametrize("act8", [False, True])
def test_resnet_with_relu(act8):
    """A ReLU decision may differ where its input is within float32 rounding of 0: gradients in
    the 2-norm; with 8-bit checkpoints they are those of the rounded activations."""
    m = resnet()
    img, lab, x, _ = inputs(m, 6, 4)
    loss, z, g = reference(m, img, lab, x)
    got = step(m, img, lab, x, act8=act8, steps=3)
    assert PR.relerr(got[1], z, PR.TAU_LOGITS) <= PR.TOL_LOGITS
    assert np.linalg.norm(got[2] - g) <= (0.05 if act8 else 1e-3) * np.linalg.norm(g)
    if act8:
        full = step(m, img, lab, x)
        assert got[0] == full[0] and np.array_equal(got[1], full[1])


def test_fused_and_unfused_decide_alike():
    m = resnet()
    img, lab, x, _ = inputs(m, 6, 14)
    a, b = step(m, img, lab, x), step(m, img, lab, x, unfused=True)
    assert np.linalg.norm(a[2] - b[2]) <= 1e-5 * np.linalg.norm(b[2])


def test_resnet_bf16():
    m = resnet(act=False)
    img, lab, x, tensors = inputs(m, 8, 5, True)
    loss, z, g = reference(m, img, lab, x)
    got = step(m, img, lab, x, dtype=lpp.BF16)
    assert PR.relerr(got[1], z, PR.TAU_BF16) <= PR.TOL_BF16
    for kind, lo, n in tensors:
        assert PR.relerr(got[2][lo:lo + n], g[lo:lo + n], PR.TAU_BF16) <= PR.TOL_BF16, (kind, lo)


@pytest.mark.parametrize("unfused", [False, True])
@pytest.mark.parametrize("part", [0, 1, 2, 3])
def test_wired_every_way(part, unfused):
    m = wired()
    img, lab, x, tensors = inputs(m, 5, 13)
    info = lpp.describe(m, 5)
    want = reference(m, img, lab, x)
    got = step(m, img, lab, x, part, unfused=unfused, steps=2)
    check(m, got, want, tensors, info.block_lo[part], info.block_hi[part], part)
    low = step(m, img, lab, x, part, unfused=unfused, act8=True, steps=2)
    assert np.array_equal(got[1], low[1])
    assert np.linalg.norm(low[2] - got[2]) <= 0.06 * np.linalg.norm(got[2])


@pytest.mark.parametrize("dtype", [lpp.FP32, lpp.BF16])
def test_partial_is_restricted_full(dtype):
    m = resnet()
    img, lab, x, _ = inputs(m, 6, 6, True)
    full = step(m, img, lab, x, 0, dtype)
    info = lpp.describe(m, 6, dtype=dtype)
    for part in range(1, m.P + 1):
        got = step(m, img, lab, x, part, dtype)
        lo, hi = info.block_lo[part], info.block_hi[part]
        assert np.array_equal(got[2][lo:hi], full[2][lo:hi]), part
        assert not got[2][:lo].any() and not got[2][hi:].any()
        assert got[0] == full[0]


def test_answers_depend_on_their_image_alone():
    m = resnet()
    img, lab, x, _ = inputs(m, 6, 7)
    z = step(m, img, lab, x)[1]
    other = img.copy()
    other[1:] = synth.images(99, 5, 3, 12, 12)
    assert np.array_equal(step(m, other, lab, x)[1][0], z[0])


def test_refusals():
    def model(groups, first=True, dtype=lpp.FP32):
        m = PM.Model("bad", (3, 8, 8), 8)
        t = m.conv(-1, 16, 3)
        if not first:
            t = m.gap(t)
        m.layers.append([lpp.GROUPNORM, t, -1, 16, 16, groups, 1, 0, 0, 1])
        m.unit_of.append(0)
        m.shapes.append(m.shapes[t])
        m.specs += [("gn_gamma", 16, 0), ("gn_beta", 16, 0)]
        t = len(m.layers) - 1
        m.linear(m.gap(t) if first else t, 8)
        m.assign_blocks([1])
        return lpp.describe(m, 2, dtype=dtype)
    assert model(4).d == 16 * 27 + 32 + 16 * 8 + 8
    assert model(4, False).P == 1
    for g in (0, -1, 3, 32):
        with pytest.raises(lpp.LppError) as e:
            model(g)
        assert e.value.code == lpp.EINVAL
    with pytest.raises(lpp.LppError) as e:
        model(4, False, lpp.BF16)
    assert e.value.code == lpp.EUNSUPPORTED


# -- distillation ----------------------------------------------------------------

def lists(batch, classes, k, T, seed, rest=True):
    g = torch.Generator().manual_seed(seed)
    z = 3 * torch.randn(batch, classes, generator=g)
    values, index = torch.topk(z, k, 1)
    r = torch.logsumexp(z.scatter(1, index, -math.inf) / T, 1) if rest else None
    return values.contiguous(), index.int(), r


@pytest.mark.parametrize("how", ["narrow", "wide", "pool"])
@pytest.mark.parametrize("alpha,T,rest", [(0.7, 2.0, True), (1.0, 3.0, False), (0.0, 2.0, True), (0.5, 1.0, True)])
def test_step_distill(how, alpha, T, rest):
    """Heads that form logits and loss in one kernel, a wide one, and logits that are a pool's."""
    if how == "narrow":
        m = resnet(act=False)
    elif how == "wide":
        m = PM.Model("wide", (3, 8, 8), 1200)
        m.linear(m.gap(m.conv(m.groupnorm(m.conv(-1, 16, 3), 4), 128, 3)), 1200)
        m.assign_blocks([1])
    else:
        m = PM.Model("pool", (3, 8, 8), 12)
        m.gap(m.conv(m.groupnorm(m.conv(-1, 16, 3), 4), 12, 1, 1, 0, bias=True))
        m.assign_blocks([1])
    img, lab, x, tensors = inputs(m, 6, 21)
    t = (*lists(6, m.n_classes, 4, T, 5, rest), alpha, T)
    want = reference(m, img, lab, x, t)
    got = step(m, img, lab, x, teacher=t, steps=3, plain_first=True)
    check(m, got, want, tensors, 0, len(x), how)
    again = step(m, img, lab, x, teacher=t, graphs=False)
    assert got[0] == again[0] and np.array_equal(got[2], again[2])
    if alpha == 0.0:
        plain = step(m, img, lab, x)
        assert abs(plain[0] - got[0]) <= 1e-5 * abs(plain[0])


def test_teacher_and_student_together():
    """A teacher's step with lr = 0, its top logits, and the student's step on them; the truncated
    step's gradient is the whole one's."""
    big, small = PM.resnet_cifar(8, (32, 32, 64), 10, 12, [1, 1, 1, 1, 1], True, 8), resnet()
    img, lab, xt, _ = inputs(big, 6, 31)
    _, _, xs, tensors = inputs(small, 6, 32)
    im, lb = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    k, T = 3, 2.0
    values, index = torch.empty(6, k, device="cuda"), torch.empty(6, k, dtype=torch.int32, device="cuda")
    rest = torch.empty(6, device="cuda")
    with lpp.Context(big, K=1, batch=6) as teacher:
        with pytest.raises(lpp.LppError) as e:
            teacher.top_logits(0, values, index, rest, T)
        assert e.value.code == lpp.ESTATE
        teacher.set_params(xt)
        teacher.step(0, im, lb, 1, 0.0)
        assert np.array_equal(teacher.get_params(0), xt)
        teacher.top_logits(0, values, index, rest, T)
        z = torch.from_numpy(teacher.get_logits(0))
        for kw in (dict(temperature=0.0), dict(temperature=math.nan)):
            with pytest.raises(lpp.LppError):
                teacher.top_logits(0, values, index, rest, **kw)
        with pytest.raises(lpp.LppError) as e:
            teacher.top_logits(0, torch.empty(6, 11, device="cuda"), torch.empty(6, 11, dtype=torch.int32, device="cuda"))
        assert e.value.code == lpp.EINVAL
    v, i = D.top(z, k)
    assert torch.equal(index.cpu(), i) and torch.equal(values.cpu(), v)
    assert ((rest.cpu().double() - D.rest(z, i, T)).abs() <= D.rest_bound(z, i, T)).all()
    with lpp.Context(small, K=1, batch=6) as student:
        student.set_params(xs)
        student.step_distill(0, im, lb, values, index, 0, 0.1, rest, 0.8, T)
        loss, g = student.get_loss(0), student.get_grad(0)
        after = student.get_params(0)
        lo, hi = student.block_range(3)
        student.set_params(xs)
        student.trace_enable(4)
        student.step_distill(0, im, lb, values, index, 3, 0.1, rest, 0.8, T)
        part = student.get_grad(0)
        assert np.array_equal(part[lo:hi], g[lo:hi]) and student.get_loss(0) == loss
        for kw, code in ((dict(alpha=1.5), lpp.EINVAL), (dict(alpha=math.nan), lpp.EINVAL),
                         (dict(temperature=-1.0), lpp.EINVAL)):
            with pytest.raises(lpp.LppError) as e:
                student.step_distill(0, im, lb, values, index, 0, 0.1, rest, **kw)
            assert e.value.code == code
        assert student.counter(0) == 2
    want = reference(small, img, lab, xs, (v, i, rest.cpu(), 0.8, T))
    assert abs(loss - want[0]) <= 1e-5 * abs(want[0])
    assert np.linalg.norm(g - want[2]) <= 1e-3 * np.linalg.norm(want[2])
    assert np.allclose(after, xs - np.float32(0.1) * g, rtol=1e-6, atol=1e-7)


def test_student_learns_the_teacher_asynchronously():
    """Four workers step on a teacher's list at once (updates are lock-free): it runs, and stays finite."""
    m = PM.resnet20(groups=8)
    img, lab, x, _ = inputs(m, 16, 41)
    im, lb = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    v, i, r = (t.cuda() for t in lists(16, 10, 4, 2.0, 9))
    with lpp.Context(m, K=1, batch=16, mode=lpp.ASYNC, momentum=0.9) as ctx:
        ctx.set_params(x)
        for n in range(5):
            for w in range(4):
                ctx.step_distill(w, im, lb, v, i, 0 if n % 2 else w + 1, 0.01, r, 0.9, 2.0)
        ctx.sync()
        assert all(math.isfinite(ctx.get_loss(w)) for w in range(4))
        assert np.isfinite(ctx.get_params(0)).all() and ctx.counter(0) == 20


def heads(how):
    """Models whose logits one kernel forms with the loss, a matrix product, a linear layer of its own or
    a pool."""
    if how in ("narrow", "unfused"):
        return resnet(act=False)
    m = PM.Model(how, (3, 8, 8), 1200 if how == "wide" else 12)
    t = m.groupnorm(m.conv(-1, 16, 3), 4)
    if how == "wide":
        m.linear(m.gap(m.conv(t, 128, 3)), 1200)
    else:
        m.gap(m.conv(t, 12, 1, 1, 0, bias=True))
    return m.assign_blocks([1])


@pytest.mark.parametrize("how", ["narrow", "wide", "pool", "unfused"])
def test_step_distill_images_without_a_label(how):
    """Labels that are no class: those images have the teacher's part alone."""
    m = heads(how)
    img, lab, x, tensors = inputs(m, 8, 23)
    lab = lab.astype(np.int32)
    lab[[0, 2, 3, 5, 6]] = [-1, m.n_classes, -100, 2 ** 31 - 1, -2 ** 31]
    for alpha in (0.6, 1.0, 0.0):
        say("no label", how, alpha)
        t = (*lists(8, m.n_classes, 4, 2.0, 5), alpha, 2.0)
        got = step(m, img, lab, x, teacher=t, steps=2, unfused=how == "unfused")
        check(m, got, reference(m, img, lab, x, t), tensors, 0, len(x), how)


@pytest.mark.parametrize("how", ["narrow", "wide", "pool"])
def test_step_distill_without_labels(how):
    """A batch without labels steps as one whose labels are no classes; replayed in turn with labelled
    ones.  A step without a teacher needs them."""
    m = heads(how)
    img, lab, x, _ = inputs(m, 6, 24)
    im, lb = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    none = torch.full_like(lb, -1)
    v, i, r = (t.cuda() for t in lists(6, m.n_classes, 4, 2.0, 6))
    with lpp.Context(m, K=1, batch=6) as ctx:
        got = {}
        for labels in (lb, None, none, lb, None):
            ctx.set_params(x)
            ctx.step_distill(0, im, labels, v, i, 0, 0.1, r, 0.6, 2.0)
            now = ctx.get_loss(0), ctx.get_grad(0)
            key = "with" if labels is lb else "without"
            before = got.setdefault(key, now)
            assert now[0] == before[0] and np.array_equal(now[1], before[1])
        assert got["with"][0] != got["without"][0]
        for bad in (lb.long(), lb[:5], lb.cpu()):
            with pytest.raises(lpp.LppError) as e:
                ctx.step_distill(0, im, bad, v, i, 0, 0.1, r, 0.6, 2.0)
            assert e.value.code == lpp.EINVAL
        with pytest.raises(lpp.LppError) as e:
            lpp._check(lpp.lib().lpp_step(ctx._ctx, 0, lpp.C.byref(lpp.Batch(im.data_ptr(), None, 6)), 0, 0.1))
        assert e.value.code == lpp.EINVAL
    want = reference(m, img, np.full(6, -1, np.int32), x, (v.cpu(), i.cpu(), r.cpu(), 0.6, 2.0))
    assert abs(got["without"][0] - want[0]) <= 1e-5 * abs(want[0])


@pytest.mark.parametrize("how", ["bf16", "act8"])
def test_step_distill_in_fewer_bits(how):
    """bf16 activations, and 8-bit checkpoints, whose forward pass and loss are the full step's."""
    m = resnet(act=how == "act8")
    img, lab, x, tensors = inputs(m, 8, 25, how == "bf16")
    t = (*lists(8, 10, 4, 2.0, 7), 0.7, 2.0)
    loss, z, g = reference(m, img, lab, x, t)
    if how == "bf16":
        got = step(m, img, lab, x, dtype=lpp.BF16, teacher=t, steps=2, plain_first=True)
        assert PR.relerr(got[1], z, PR.TAU_BF16) <= PR.TOL_BF16
        for kind, lo, n in tensors:
            assert PR.relerr(got[2][lo:lo + n], g[lo:lo + n], PR.TAU_BF16) <= PR.TOL_BF16, (kind, lo)
        # the loss and its gradient at the logits that the step had
        want = D.distill(torch.from_numpy(got[1]), t[0], t[1], t[2], torch.from_numpy(lab.astype(np.int32)), None, 0.7, 2.0)
        bound = want[2].mean().item() + 16 * D.U * want[0].abs().mean().item()
        assert abs(got[0] - want[0].mean().item()) <= bound
    else:
        got, full = step(m, img, lab, x, act8=True, teacher=t, steps=2), step(m, img, lab, x, teacher=t)
        assert got[0] == full[0] and np.array_equal(got[1], full[1])
        assert np.linalg.norm(got[2] - g) <= 0.05 * np.linalg.norm(g)
