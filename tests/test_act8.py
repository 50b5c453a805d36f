"""8-bit checkpoints and RMS norm without a GPU: buffer sizes, every call that is
refused before anything is launched, and the reference forms themselves."""
import ctypes as C

import pytest
import torch

from paper_2203_06638_amd import lpp
from tests import act8ref as R

OKP = 4096      # an aligned address that no refused call touches


def test_bytes():
    for rows, cols in [(0, 1), (1, 1), (7, 16), (5, 33), (3, 96), (1000003, 250)]:
        assert lpp.act8_bytes(rows, cols) == rows * (R.pitch(cols) + R.groups(cols))
    for rows, cols in [(-1, 4), (4, 0), (4, -3), (1 << 40, 2), (1, 1 << 25), (1, 1 << 40)]:
        with pytest.raises(lpp.LppError) as e:
            lpp.act8_bytes(rows, cols)
        assert e.value.code == lpp.EINVAL


def test_workspaces():
    assert lpp.act8_wgrad_ws(1, 8, 8) == 0            # one split writes dw itself
    assert lpp.act8_wgrad_ws(0, 8, 8) == 0
    n = lpp.act8_wgrad_ws(100000, 36, 100)
    assert n > 0 and n % 3600 == 0
    assert lpp.rmsnorm_bwd_ws(0, 10) >= 12 and lpp.rmsnorm_bwd_ws(100000, 10) % 12 == 0
    for f in (lambda: lpp.act8_wgrad_ws(-1, 8, 8), lambda: lpp.act8_wgrad_ws(8, 0, 8),
              lambda: lpp.act8_wgrad_ws(8, 1 << 20, 1 << 20), lambda: lpp.rmsnorm_bwd_ws(4, 0)):
        with pytest.raises(lpp.LppError):
            f()


def refused(rc, code=lpp.EINVAL):
    assert rc == code
    assert lpp.lib().lpp_last_error()


@pytest.mark.parametrize("call", ["pack", "unpack"])
def test_pack_refusals(call):
    L = lpp.lib()

    def f(x=OKP, dtype=lpp.FP32, rows=4, cols=40, ld=40, q=OKP):
        if call == "pack":
            return L.lpp_kernel_act8_pack(x, dtype, rows, cols, ld, 0, q, None)
        return L.lpp_kernel_act8_unpack(q, rows, cols, x, dtype, ld, None)
    for kw in (dict(x=None), dict(q=None), dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(cols=0), dict(ld=39),
               dict(x=OKP + 2), dict(q=OKP + 8), dict(ld=1 << 60), dict(rows=1 << 40), dict(x=OKP + 1, dtype=lpp.BF16)):
        refused(f(**kw))


def test_wgrad_refusals():
    L = lpp.lib()
    need = lpp.act8_wgrad_ws(5000, 64, 64)
    assert need > 0

    def f(dy=OKP, dtype=lpp.FP32, rows=5000, cout=64, ld=64, q=OKP, cin=64, dw=OKP, ws=OKP, ws_floats=need):
        return L.lpp_kernel_act8_wgrad(dy, dtype, rows, cout, ld, q, cin, dw, ws, ws_floats, None)
    for kw in (dict(dy=None), dict(q=None), dict(dw=None), dict(ws=None), dict(ws_floats=need - 1), dict(ws=OKP + 8),
               dict(dw=OKP + 2), dict(dtype=7), dict(rows=-5), dict(cout=0), dict(cin=0), dict(ld=63), dict(q=OKP + 4),
               dict(cout=1 << 20, ld=1 << 20, cin=1 << 20)):
        refused(f(**kw))


def test_rmsnorm_refusals():
    L = lpp.lib()

    def f(**kw):
        a = lpp.RmsNormArgs()
        v = dict(x=OKP, y=OKP, gamma=OKP, rstd=OKP, ldx=40, ldy=40, ldres=40, ldh=40, rows=4, cols=40, dtype=lpp.FP32,
                 eps=1e-5)
        v.update(kw)
        for k, x in v.items():
            setattr(a, k, x)
        return L.lpp_kernel_rmsnorm(C.byref(a), None)
    refused(L.lpp_kernel_rmsnorm(None, None))
    for kw in (dict(x=None), dict(y=None), dict(gamma=None), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(h=OKP), dict(ldx=39), dict(ldy=8), dict(res=OKP, ldres=8),
               dict(res=OKP, h=OKP, ldh=2), dict(q=OKP + 8), dict(gamma=OKP + 2), dict(rstd=OKP + 2), dict(dtype=3),
               dict(rows=-1), dict(cols=0), dict(y=OKP + 2), dict(res=OKP + 2)):
        refused(f(**kw))
    refused(f(cols=16385, ldx=16385, ldy=16385), lpp.EUNSUPPORTED)


def test_rmsnorm_bwd_refusals():
    L = lpp.lib()
    need = lpp.rmsnorm_bwd_ws(100, 40)

    def f(**kw):
        a = lpp.RmsNormBwdArgs()
        v = dict(dy=OKP, h=OKP, dx=OKP, gamma=OKP, rstd=OKP, dgamma=OKP, ws=OKP, ws_floats=need, lddy=40, ldh=40,
                 lddres=40, lddx=40, rows=100, cols=40, dtype=lpp.FP32)
        v.update(kw)
        for k, x in v.items():
            setattr(a, k, x)
        return L.lpp_kernel_rmsnorm_bwd(C.byref(a), None)
    refused(L.lpp_kernel_rmsnorm_bwd(None, None))
    for kw in (dict(dy=None), dict(h=None), dict(q=OKP), dict(dx=None, dgamma=None), dict(gamma=None), dict(rstd=None),
               dict(ws=None), dict(ws_floats=need - 1), dict(ws=OKP + 4), dict(dgamma=OKP + 1), dict(lddy=4),
               dict(ldh=4), dict(lddx=4), dict(dres=OKP, lddres=4), dict(h=None, q=OKP + 8), dict(dtype=9),
               dict(rows=-1), dict(cols=0), dict(dx=OKP + 2)):
        refused(f(**kw))
    refused(f(cols=16385, lddy=16385, ldh=16385, lddx=16385), lpp.EUNSUPPORTED)


def test_binding_refuses_cpu_tensors():
    x, q = torch.zeros(4, 40), torch.zeros(lpp.act8_bytes(4, 40), dtype=torch.uint8)
    v = torch.zeros(40)
    for f in (lambda: lpp.kernel_act8_pack(x, q), lambda: lpp.kernel_act8_unpack(q, x),
              lambda: lpp.kernel_act8_wgrad(x, q, torch.zeros(40, 40)), lambda: lpp.kernel_rmsnorm(x, v, v[:4], y=x),
              lambda: lpp.kernel_rmsnorm_bwd(x, v, v[:4], dx=x, h=x), lambda: lpp.kernel_act8_pack([1.0], q)):
        with pytest.raises(lpp.LppError) as e:
            f()
        assert e.value.code == lpp.EINVAL


# -- the reference forms -------------------------------------------------------

def test_reference_format():
    x = torch.tensor([[1.0, -0.5, 0.0, 127.4, 1e-3]], dtype=torch.float64)
    codes, s = R.pack(x)
    assert s.item() == 133 and codes[0, :5].tolist() == [1, 0, 0, 127, 0]     # (-0.5 ties to even)
    assert R.pack(x, True)[0][0, :5].tolist() == [1, -1, 0, 127, 1]
    assert R.pack(torch.tensor([[127.5]], dtype=torch.float64))[1].item() == 134
    assert R.pack(torch.tensor([[0.0]], dtype=torch.float64))[1].item() == 7
    v = R.values(*R.pack(torch.tensor([[float("inf"), 1.0]], dtype=torch.float64)), 2)
    assert torch.isnan(v).all()
    # every value is exact in bf16 and float32, down to the smallest step
    for e in (7, 8, 133, 254):
        c = torch.arange(-127, 128, dtype=torch.float64)
        v = c * 2.0 ** (e - 133)
        assert torch.equal(v.to(torch.bfloat16).double(), v) and torch.equal(v.float().double(), v)


def test_reference_gradient_against_differences():
    g = torch.Generator().manual_seed(3)
    x, gamma, dy = (torch.randn(*n, generator=g, dtype=torch.float64) for n in ((6, 21), (21,), (6, 21)))
    _, rstd, _ = R.norm(x, gamma, 1e-5)
    dx, dg, _, _ = R.norm_bwd(dy, x, rstd, gamma)

    def loss(x, gamma):
        return (R.norm(x, gamma, 1e-5)[2] * dy).sum()
    e = 1e-6
    for _ in range(5):
        vx, vg = torch.randn(6, 21, generator=g, dtype=torch.float64), torch.randn(21, generator=g, dtype=torch.float64)
        num = (loss(x + e * vx, gamma + e * vg) - loss(x - e * vx, gamma - e * vg)) / (2 * e)
        # (central differences: e^2 of the third derivative, and rounding 2^-53 / e)
        assert abs(num - (dx * vx).sum() - (dg * vg).sum()) < 1e-7 * (dx.abs().sum() + dg.abs().sum())


# -- RMS norm layers in a model description --------------------------------------

def test_describe_rmsnorm():
    from paper_2203_06638_amd import models as PM
    m = PM.pre_norm_net((16, 32), 1, 10, 12)
    info = lpp.describe(m)
    assert info.d == m.d
    assert sum(n for kind, n, _ in m.specs if kind == "rms_gamma") == 16 * 3 + 32 * 3
    bad = PM.Model("bad", (3, 8, 8), 4)
    t = bad.rmsnorm(bad.conv(-1, 8, 3))
    bad.layers[t][4] = 12
    bad.linear(bad.gap(t), 4)
    with pytest.raises(lpp.LppError) as e:
        lpp.describe(bad.assign_blocks([1]))
    assert e.value.code == lpp.EINVAL
    wide = PM.Model("wide", (3, 2, 2), 4)
    wide.linear(wide.gap(wide.rmsnorm(wide.conv(-1, 16388, 1, 1, 0))), 4)
    with pytest.raises(lpp.LppError) as e:
        lpp.describe(wide.assign_blocks([1]))
    assert e.value.code == lpp.EUNSUPPORTED
    pooled = PM.Model("pooled", (8, 4, 4), 4)
    pooled.linear(pooled.gap(pooled.rmsnorm(pooled.gap(pooled.conv(-1, 8, 1, 1, 0)))), 4)
    lpp.describe(pooled.assign_blocks([1]))
    with pytest.raises(lpp.LppError) as e:
        lpp.describe(pooled, dtype=lpp.BF16)
    assert e.value.code == lpp.EUNSUPPORTED
