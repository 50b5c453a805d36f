"""Group norm without a GPU: workspaces, every call that is refused before anything is
launched, and the reference form's gradient against differences and autograd."""
import ctypes as C

import pytest
import torch

from paper_2203_06638_amd import lpp
from tests import gnref as R

OKP = 4096      # an aligned address that no refused call touches


def refused(rc, code=lpp.EINVAL):
    assert rc == code
    assert lpp.lib().lpp_last_error()


BAD_SIZES = [dict(images=-1), dict(pixels=0), dict(channels=0), dict(groups=0), dict(groups=-4), dict(groups=3),
             dict(groups=80), dict(images=1 << 36), dict(pixels=1 << 38), dict(channels=(1 << 24) + 4)]


def test_workspaces():
    for f in (lpp.groupnorm_ws, lpp.groupnorm_bwd_ws):
        assert f(2, 100, 40, 4) >= 0 and f(0, 1, 40, 4) >= 0
        for kw in BAD_SIZES + [dict(channels=1 << 40)]:
            with pytest.raises(lpp.LppError) as e:
                f(**{**dict(images=4, pixels=9, channels=40, groups=4), **kw})
            assert e.value.code == lpp.EINVAL


def test_forward_refusals():
    L = lpp.lib()
    need = lpp.groupnorm_ws(4, 900, 40, 4)

    def f(**kw):
        a = lpp.GroupNormArgs()
        v = dict(x=OKP, y=OKP, ldx=40, ldy=40, gamma=OKP, beta=OKP, mean=OKP, rstd=OKP, ws=OKP, ws_floats=need, images=4,
                 pixels=900, channels=40, groups=4, dtype=lpp.FP32, act=lpp.ACT_RELU, eps=1e-5)
        v.update(kw)
        for k, x in v.items():
            setattr(a, k, x)
        return L.lpp_kernel_groupnorm(C.byref(a), None)
    refused(L.lpp_kernel_groupnorm(None, None))
    for kw in BAD_SIZES + [dict(x=None), dict(y=None), dict(gamma=None), dict(beta=None), dict(gamma=OKP + 2),
                           dict(beta=OKP + 1), dict(mean=OKP + 2), dict(rstd=OKP + 3), dict(ldx=39), dict(ldy=39),
                           dict(x=OKP + 2), dict(y=OKP + 1, dtype=lpp.BF16), dict(dtype=2), dict(act=3), dict(act=-1),
                           dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(ldx=1 << 50),
                           dict(ws=None), dict(ws=OKP + 8), dict(ws_floats=need - 1)]:
        refused(f(**kw))
    # more threads than a launch has: 256 to an image
    refused(f(images=1 << 24, pixels=1, ws_floats=lpp.groupnorm_ws(1 << 24, 1, 40, 4)), lpp.EUNSUPPORTED)


def test_backward_refusals():
    L = lpp.lib()
    need = lpp.groupnorm_bwd_ws(4, 900, 40, 4)

    def f(**kw):
        a = lpp.GroupNormBwdArgs()
        v = dict(dy=OKP, x=OKP, dx=OKP, lddy=40, ldx=40, lddres=40, lddx=40, gamma=OKP, beta=OKP, mean=OKP, rstd=OKP,
                 dgamma=OKP, dbeta=OKP, ws=OKP, ws_floats=need, images=4, pixels=900, channels=40, groups=4,
                 dtype=lpp.FP32, act=lpp.ACT_RELU)
        v.update(kw)
        for k, x in v.items():
            setattr(a, k, x)
        return L.lpp_kernel_groupnorm_bwd(C.byref(a), None)
    refused(L.lpp_kernel_groupnorm_bwd(None, None))
    for kw in BAD_SIZES + [dict(dy=None), dict(x=None), dict(dx=None, dgamma=None, dbeta=None), dict(gamma=None),
                           dict(beta=None), dict(mean=None), dict(rstd=None), dict(mean=OKP + 1), dict(dgamma=OKP + 2),
                           dict(dbeta=OKP + 2), dict(lddy=39), dict(ldx=3), dict(lddx=39), dict(dres=OKP, lddres=39),
                           dict(dres=OKP + 2), dict(dx=OKP + 2), dict(dtype=-1), dict(act=7), dict(ws=None),
                           dict(ws=OKP + 4), dict(ws_floats=need - 1)]:
        refused(f(**kw))
    refused(f(images=1 << 24, pixels=1, ws_floats=lpp.groupnorm_bwd_ws(1 << 24, 1, 40, 4)), lpp.EUNSUPPORTED)


def test_binding_refuses():
    x, v, s = torch.zeros(6, 8), torch.zeros(8), torch.zeros(2, 2)
    for f in (lambda: lpp.kernel_groupnorm(x, 2, 2, v, v, x), lambda: lpp.kernel_groupnorm([1.0], 2, 2, v, v, x),
              lambda: lpp.kernel_groupnorm_bwd(x, x, 2, 2, v, v, s, s, x)):
        with pytest.raises(lpp.LppError) as e:
            f()
        assert e.value.code == lpp.EINVAL
    for rows, images, ch, groups in [(7, 2, 8, 2), (6, 0, 8, 2), (0, 2, 8, 2), (6, -2, 8, 2), (6, 2, 8, 3), (6, 2, 8, 0),
                                     (6, 2, 8, 2 ** 32 + 1)]:
        with pytest.raises(lpp.LppError):
            lpp._pixels(rows, images, ch, groups)
    assert lpp._pixels(6, 2, 8, 2) == 3 and lpp._pixels(0, 0, 8, 8) == 1


@pytest.mark.parametrize("name", ["none", "relu", "silu"])
def test_reference_gradient(name):
    g = torch.Generator().manual_seed(3)
    n, p, ch, G = 2, 6, 12, 3
    x, dy = (torch.randn(n * p, ch, generator=g, dtype=torch.float64) for _ in range(2))
    gamma, beta = (torch.randn(ch, generator=g, dtype=torch.float64) for _ in range(2))

    def loss(x, gamma, beta):
        return (R.forward(x, n, G, gamma, beta, 1e-5, name)[0] * dy).sum()
    _, mean, rstd = R.forward(x, n, G, gamma, beta, 1e-5, name)
    got = R.backward(dy, x, n, G, gamma, beta, mean, rstd, name)
    leaves = [t.clone().requires_grad_() for t in (x, gamma, beta)]
    for a, b in zip(got, torch.autograd.grad(loss(*leaves), leaves)):
        assert torch.allclose(a, b, rtol=1e-9, atol=1e-11)
    e = 1e-6
    for _ in range(5):
        v = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (x, gamma, beta)]
        up, down = (loss(*(t + s * e * d for t, d in zip((x, gamma, beta), v))) for s in (1, -1))
        # (central differences: e^2 of the third derivative, and rounding 2^-53 / e)
        assert abs((up - down) / (2 * e) - sum((a * d).sum() for a, d in zip(got, v))) < 1e-6 * sum(a.abs().sum() for a in got)


def test_layer():
    """A layer's parameters and what lpp_describe refuses."""
    from paper_2203_06638_amd import models as PM

    def model(groups, c=16):
        m = PM.Model("m", (3, 8, 8), 8)
        t = m.conv(-1, 16, 3)
        m.layers.append([lpp.GROUPNORM, t, -1, c, c, groups, 1, 0, 0, 0])
        m.unit_of.append(0)
        m.shapes.append(m.shapes[t])
        m.linear(m.gap(1), 8)
        return lpp.describe(m.assign_blocks([1]), 2)
    assert model(4).d == 16 * 27 + 2 * 16 + 16 * 8 + 8
    for kw in (dict(groups=0), dict(groups=-2), dict(groups=3), dict(groups=32), dict(groups=4, c=8)):
        with pytest.raises(lpp.LppError) as e:
            model(**kw)
        assert e.value.code == lpp.EINVAL
    m = PM.resnet20(groups=8)
    assert lpp.describe(m, 4).d == PM.resnet20().d
