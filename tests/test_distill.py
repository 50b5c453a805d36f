"""Top logits and distillation without a GPU: workspaces, every call that is refused before
anything is launched, and the reference forms' gradient against autograd and differences."""
import ctypes as C

import pytest
import torch

from paper_2203_06638_amd import lpp
from tests import distillref as R

OKP = 4096      # an aligned address that no refused call touches
LONG = 300000   # classes of rows that are taken in pieces


def refused(rc, code=lpp.EINVAL):
    assert rc == code
    assert lpp.lib().lpp_last_error()


def test_workspaces():
    assert lpp.top_logits_ws(0, 10, 3) == 0 and lpp.distill_ws(0, 10) == 0
    assert lpp.top_logits_ws(100, 10, 10) == 0 and lpp.distill_ws(100, 1000) == 0
    assert lpp.top_logits_ws(3, LONG, 128) > 0 and lpp.distill_ws(3, LONG) > 0
    for f in (lambda: lpp.top_logits_ws(-1, 10, 3), lambda: lpp.top_logits_ws(4, 0, 1), lambda: lpp.top_logits_ws(4, 10, 0),
              lambda: lpp.top_logits_ws(4, 10, 11), lambda: lpp.top_logits_ws(4, 1000, 129),
              lambda: lpp.top_logits_ws(1 << 39, 10, 1), lambda: lpp.top_logits_ws(1, 1 << 40, 1),
              lambda: lpp.distill_ws(-1, 10), lambda: lpp.distill_ws(3, 0), lambda: lpp.distill_ws(3, (1 << 24) + 1),
              lambda: lpp.distill_ws(1 << 39, 10)):
        with pytest.raises(lpp.LppError) as e:
            f()
        assert e.value.code == lpp.EINVAL


def test_top_refusals():
    L = lpp.lib()
    need = lpp.top_logits_ws(4, LONG, 5)

    def f(**kw):
        a = lpp.TopLogitsArgs()
        v = dict(z=OKP, ldz=LONG, rows=4, classes=LONG, k=5, dtype=lpp.FP32, temperature=1.0, values=OKP, index=OKP, rest=OKP,
                 ws=OKP, ws_floats=need)
        v.update(kw)
        for k, x in v.items():
            setattr(a, k, x)
        return L.lpp_kernel_top_logits(C.byref(a), None)
    refused(L.lpp_kernel_top_logits(None, None))
    for kw in (dict(z=None), dict(values=None), dict(index=None), dict(z=OKP + 2), dict(values=OKP + 2), dict(index=OKP + 1),
               dict(rest=OKP + 2), dict(ldz=LONG - 1), dict(rows=-1), dict(classes=0), dict(k=0), dict(k=-1),
               dict(classes=4), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
               dict(temperature=float("inf")), dict(dtype=2), dict(ws=None), dict(ws=OKP + 8), dict(ws_floats=need - 1),
               dict(classes=(1 << 24) + 1, ldz=1 << 25), dict(rows=1 << 39)):
        refused(f(**kw))
    refused(f(k=129), lpp.EUNSUPPORTED)
    # more threads than a launch has: 256, and 1024 that merge pieces, to a row
    refused(f(rows=1 << 24, classes=500, ldz=500, k=100, ws=None, ws_floats=0), lpp.EUNSUPPORTED)
    rows = 1 << 22
    refused(f(rows=rows, classes=70000, ldz=70000, ws_floats=lpp.top_logits_ws(rows, 70000, 5)), lpp.EUNSUPPORTED)


def test_distill_refusals():
    L = lpp.lib()
    need = lpp.distill_ws(4, LONG)

    def f(**kw):
        a = lpp.DistillArgs()
        v = dict(z=OKP, dz=OKP, ldz=LONG, lddz=LONG, rows=4, classes=LONG, k=5, dtype=lpp.FP32, values=OKP, index=OKP,
                 rest=OKP, labels=OKP, weight=OKP, loss=OKP, alpha=0.5, temperature=2.0, scale=1.0, ws=OKP,
                 ws_floats=need)
        v.update(kw)
        for k, x in v.items():
            setattr(a, k, x)
        return L.lpp_kernel_distill(C.byref(a), None)
    nan, inf = float("nan"), float("inf")
    refused(L.lpp_kernel_distill(None, None))
    for kw in (dict(z=None), dict(values=None), dict(index=None), dict(loss=None), dict(z=OKP + 1), dict(dz=OKP + 2),
               dict(values=OKP + 2), dict(index=OKP + 2), dict(rest=OKP + 1), dict(labels=OKP + 2), dict(weight=OKP + 3),
               dict(loss=OKP + 2), dict(ldz=LONG - 1), dict(lddz=5), dict(rows=-1), dict(classes=0), dict(k=0),
               dict(alpha=-0.1), dict(alpha=1.1), dict(alpha=nan), dict(temperature=0.0), dict(temperature=nan),
               dict(temperature=inf), dict(scale=nan), dict(scale=inf), dict(dtype=5), dict(ws=None), dict(ws=OKP + 4),
               dict(ws_floats=need - 1), dict(rows=1 << 39), dict(classes=(1 << 24) + 1, ldz=1 << 25, lddz=1 << 25)):
        refused(f(**kw))
    refused(f(k=129), lpp.EUNSUPPORTED)
    refused(f(rows=1 << 24, classes=5000, ldz=5000, lddz=5000, ws=None, ws_floats=0), lpp.EUNSUPPORTED)


def test_binding_refuses():
    z, v, i = torch.zeros(4, 9), torch.zeros(4, 3), torch.zeros(4, 3, dtype=torch.int32)
    for f in (lambda: lpp.kernel_top_logits(z, v, i), lambda: lpp.kernel_distill(z, v, i, z[:, 0], z),
              lambda: lpp.kernel_top_logits([1.0], v, i)):
        with pytest.raises(lpp.LppError) as e:
            f()
        assert e.value.code == lpp.EINVAL
    for vals, idx, rows in ((v, i, 5), (v, i[:, :2], 4), (v[0], i[0], 4)):
        with pytest.raises(lpp.LppError):
            lpp._list(vals, idx, rows, 0)


# -- the reference forms -------------------------------------------------------

def test_reference_top():
    z = torch.tensor([[1.0, 3.0, 3.0, -0.0, 0.0, float("nan"), 3.0]])
    v, i = R.top(z, 6)
    assert i[0].tolist() == [5, 1, 2, 6, 0, 3]
    assert R.rest(z, i, 1.0).item() == 0.0


@pytest.mark.parametrize("rest", [False, True])
def test_reference_gradient(rest):
    g = torch.Generator().manual_seed(1)
    rows, n, k = 5, 12, 4
    z = torch.randn(rows, n, generator=g, dtype=torch.float64)
    values, index = torch.topk(3 * torch.randn(rows, n, generator=g, dtype=torch.float64), k, 1)
    index = index.int()
    index[1, 2] = -1
    index[2, 3] = index[2, 0]
    r = torch.randn(rows, generator=g, dtype=torch.float64) if rest else None
    labels = torch.randint(n, (rows,), generator=g).int()
    labels[3] = -1
    w = torch.rand(rows, generator=g, dtype=torch.float64)
    args = (values, index, r, labels, w, 0.6, 2.5, 0.5)
    dz = R.distill(z, *args)[1]
    leaf = z.clone().requires_grad_()
    auto, = torch.autograd.grad(0.5 * R.distill(leaf, *args)[0].sum(), leaf)
    assert torch.allclose(dz, auto, rtol=1e-10, atol=1e-12)
    e = 1e-6
    for _ in range(3):
        d = torch.randn(z.shape, generator=g, dtype=torch.float64)
        num = 0.5 * (R.distill(z + e * d, *args)[0] - R.distill(z - e * d, *args)[0]).sum() / (2 * e)
        # (central differences: e^2 of the third derivative, and rounding 2^-53 / e)
        assert abs(num - (dz * d).sum()) < 1e-7 * dz.abs().sum()


def test_step_refusals():
    """A teacher is looked at before the context is."""
    L = lpp.lib()

    def f(**kw):
        t = lpp.Teacher(OKP, OKP, OKP, 4, 0.5, 2.0)
        for k, x in kw.items():
            setattr(t, k, x)
        return L.lpp_step_distill(None, 0, None, C.byref(t), 0, 0.1)
    refused(L.lpp_step_distill(None, 0, None, None, 0, 0.1))
    nan, inf = float("nan"), float("inf")
    for kw in ({}, dict(values=None), dict(index=None), dict(values=OKP + 2), dict(index=OKP + 1), dict(rest=OKP + 2),
               dict(k=0), dict(k=-3), dict(alpha=-0.5), dict(alpha=2.0), dict(alpha=nan), dict(temperature=0.0),
               dict(temperature=nan), dict(temperature=inf)):
        refused(f(**kw))
    refused(f(k=129), lpp.EUNSUPPORTED)
    refused(L.lpp_top_logits(None, 0, 3, 1.0, OKP, OKP, OKP))


def test_temperatures():
    """Distillation takes temperatures whose squares and reciprocals float32 holds with room for what they
    are multiplied by, [2^-60, 2^60]; the top logits every one with a reciprocal in float32."""
    L = lpp.lib()
    z, k, t = 100, 5, 0

    def top(T):
        return L.lpp_kernel_top_logits(C.byref(lpp.TopLogitsArgs(OKP, z, 4, z, k, lpp.FP32, T, OKP, OKP, OKP, None, 0)), None)

    def distill(T):
        return L.lpp_kernel_distill(C.byref(lpp.DistillArgs(OKP, OKP, z, z, 4, z, k, lpp.FP32, OKP, OKP, OKP, OKP, OKP, OKP,
                                                            0.5, T, 1.0, None, 0)), None)

    def step(T):
        return L.lpp_step_distill(None, 0, None, C.byref(lpp.Teacher(OKP, OKP, OKP, 4, 0.5, T)), 0, 0.1)
    for T in (1e-45, 1e-39, 2.0 ** -127):
        refused(top(T))
    for T in (1e-45, 1e-38, 2.0 ** -60 * (1 - 2.0 ** -24), 2.0 ** 60 * (1 + 2.0 ** -23), 1e20, 3e38):
        for f in (distill, step):
            refused(f(T))
            assert b"temperature" in L.lpp_last_error()
