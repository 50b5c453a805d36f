"""The stand-alone norm and weight-gradient calls at values their other tests leave out.
Tolerances as in test_gpu_act8.py."""
import pytest

from paper_2203_06638_amd import lpp
from tests import act8ref as R
from tests.test_gpu_act8 import DT, HALF, NORM_SHAPES, U, checkpoint, rand, wgrad

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_norm_gradient_of_far_rows(dtype, packed):
    """eps = 0 and rows about 1e-20, 1e-19, 1 and 1e17: 1 / rms and the gradient are
    float32 numbers, the square of 1 / rms is not.  u = h * rstd takes one
    rounding, g another, their sum over C terms C + 1, the rest of dx four."""
    for k, cols in enumerate((70, 250, 2000, 3000, 9000)):
        scale = torch.tensor([1e-20, 1e-19, 1.0, 1e17, 3e-20]).repeat(3)[:, None]
        h = (rand(k, 15, cols, spread=0.1) * scale).to(DT[dtype])
        dy = (rand(k + 20, 15, cols) * 1e-3).to(DT[dtype])
        gamma = rand(k + 40, 1, cols)[0]
        q, hv = checkpoint(h) if packed else (None, h.double())
        rstd = (1 / torch.sqrt((h.double() ** 2).mean(1))).float()
        assert torch.isfinite(rstd).all()
        dx, dg = torch.empty_like(dy, device="cuda"), torch.empty(cols, device="cuda")
        lpp.kernel_rmsnorm_bwd(dy.cuda(), gamma.cuda(), rstd.cuda(), dx, dg,
                               torch.empty(lpp.rmsnorm_bwd_ws(15, cols), device="cuda"),
                               h=None if packed else h.cuda(), q=q)
        wx, wg, sx, sg = R.norm_bwd(dy.double(), hv, rstd.double(), gamma.double())
        tol = (cols + 12) * U * sx
        assert ((dx.cpu().double() - wx).abs() <= tol + HALF[dtype] * (wx.abs() + tol)).all(), cols
        assert ((dg.cpu().double() - wg).abs() <= 30 * U * sg).all(), cols


def test_wgrad_of_a_nan_with_a_low_payload():
    """A float32 NaN stays one where its upper 16 bits alone would be an
    infinity: in a row of the steps and in the last row, which ends a ragged
    matrix."""
    rows, cin, cout = 100, 70, 66
    x, dy = rand(1, rows, cin).abs() + 0.1, rand(2, rows, cout)
    bits = dy.view(torch.int32)
    bits[17, 5], bits[40, 9], bits[rows - 1, 65] = 0x7f800001, -0x7fff00, 0x7f80ffff
    assert torch.isnan(dy).sum() == 3
    q, xv = checkpoint(x)
    got = wgrad(dy.cuda(), q, rows, cin)
    bad = torch.zeros(cout, dtype=torch.bool)
    bad[[5, 9, 65]] = True
    assert torch.isnan(got[bad]).all() and torch.isfinite(got[~bad]).all()
    want, size = dy.double().t() @ xv, dy.double().abs().t() @ xv.abs()
    assert ((got - want).abs() <= (rows + 64) * 2.0 ** -23 * size)[~bad].all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rmsnorm_keep_sign(dtype):
    """The norm's checkpoint with keep_sign: codes of y's sign, 0 where y is 0 and in
    the padding, half a step off where |y| is half a step at least and under a
    step below."""
    for k, (rows, cols) in enumerate(NORM_SHAPES):
        x, res = rand(k, rows, cols, dtype, 2.0), rand(60 + k, rows, cols, dtype, 2.0)
        x[:, ::3], res[:, ::3] = 0, 0
        x[::5] *= 1e-3
        if cols == 1:
            x[:] = 1.5
        gamma = rand(90 + k, 1, cols)[0]
        gamma = torch.where(gamma.abs() < 1e-3, torch.ones(()), gamma)
        for r in (None, res):
            q = torch.full((lpp.act8_bytes(rows, cols),), 99, dtype=torch.uint8, device="cuda")
            lpp.kernel_rmsnorm(x.cuda(), gamma.cuda(), None, 1e-5, res=None if r is None else r.cuda(), q=q,
                               keep_sign=True)
            _, _, y = R.norm(x.double(), gamma.double(), 1e-5, None if r is None else r.double(), DT[dtype])
            codes, s = R.split(q.cpu(), rows, cols)
            assert (codes[:, cols:] == 0).all()
            assert torch.equal(torch.sign(codes[:, :cols].double()), torch.sign(y)), (rows, cols)
            tol = (cols / 2 + 6) * U
            lo, hi = R.exponents(y * (1 - 2 * tol)), R.exponents(y * (1 + 2 * tol))
            assert ((s.long() >= lo) & (s.long() <= hi)).all()
            step = torch.exp2(s.double() - 133).repeat_interleave(32, 1)[:, :cols]
            err = (R.values(codes, s, cols) - y).abs()
            far = y.abs() * (1 - 2 * tol) > step / 2
            assert (err <= step * 0.5 + 3 * tol * y.abs())[far].all()
            assert (err < step)[~far & (y != 0)].all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rmsnorm_beyond_float32_squares(dtype):
    """A row whose squares add up to more than float32 holds: rstd 0 and y 0; with
    eps = 0 one whose squares vanish: rstd infinite.  Other rows are as ever."""
    for cols in (40, 3000):
        x = rand(3, 4, cols, dtype, 0.1)
        x[1] = torch.finfo(DT[dtype]).min
        x[2] = 1e-30
        xd = x.cuda()
        y, rstd = torch.empty_like(xd), torch.empty(4, device="cuda")
        lpp.kernel_rmsnorm(xd, torch.ones(cols, device="cuda"), rstd, 0.0, y=y)
        assert rstd[1] == 0 and rstd[2] == float("inf") and (y[1] == 0).all()
        _, rr, yr = R.norm(x.double(), torch.ones(cols, dtype=torch.float64), 0.0)
        tol = (cols / 2 + 9) * U + HALF[dtype]
        for r in (0, 3):
            assert ((y[r].cpu().double() - yr[r]).abs() <= tol * yr[r].abs()).all()
