"""Gradients of tensors with several readers where one of the readers is fused into a
later layer, and so runs its backward before its place in the layer list."""
import numpy as np
import pytest

from paper_2203_06638_amd import lpp
from paper_2203_06638_amd import models as PM
from tests import parity as PR
from tests.test_gpu_act8_step import inputs, reference, step

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def net(name):
    m = PM.Model(name, (8, 8, 8), 8)
    x = m.conv(-1, 16, 3, bias=name != "two_bns")    # (a bias that only batch norms read has no gradient)
    if name == "conv_of_the_residual":
        t = m.add(m.conv(x, 16, 3, bias=True), x)
    elif name == "two_convs_of_a_norm":
        n = m.rmsnorm(x)
        t = m.add(m.conv(n, 16, 3, bias=True), m.conv(n, 16, 1, 1, 0))
    elif name == "conv_added_after_a_normed_sum":
        y = m.conv(x, 16, 3)
        late = m.conv(x, 16, 1, 1, 0)
        n = m.rmsnorm(m.add(x, y))
        t = m.add(late, n)
    elif name == "bn_and_conv":
        t = m.add(m.bn(x), m.conv(x, 16, 3))
    elif name == "bn_of_the_residual":
        t = m.add(m.bn(x), x)
    elif name == "two_bns":
        t = m.add(m.bn(x), m.bn(x))
    m.new_unit()
    m.linear(m.gap(m.conv(t, 16, 3, 2)), 8)
    return m.assign_blocks([1, 2])


NETS = ["conv_of_the_residual", "two_convs_of_a_norm", "conv_added_after_a_normed_sum", "bn_and_conv",
        "bn_of_the_residual", "two_bns"]


@pytest.mark.parametrize("act8", [False, True])
@pytest.mark.parametrize("unfused", [False, True])
@pytest.mark.parametrize("dtype", [lpp.FP32, lpp.BF16])
@pytest.mark.parametrize("name", NETS)
def test_gradient_against_float64(name, dtype, unfused, act8):
    """A contribution that is lost or added onto another buffer's leftovers changes a
    gradient by half of its norm and more.  Roundings in float32: sums of up to
    656 terms (9 x 16 channels, 512 rows) in five passes, 656 x 5 x 2^-24 = 2e-4
    of the terms' magnitudes, which the batch norms' cancellations raise by up to
    50: 1% of the norm.  bf16: ten stored tensors of up to 2^-8 each, and 8-bit
    checkpoints of 2.3% each, four on a path: 10% and 20%."""
    m = net(name)
    img, lab, x, tensors = inputs(m, 8, 17, True)
    loss, z, g = reference(m, img, lab, x)
    bf = dtype == lpp.BF16
    got = step(m, img, lab, x, 0, dtype, steps=2, unfused=unfused, act8=act8)
    assert PR.relerr(got[1], z, PR.TAU_BF16 if bf else PR.TAU_LOGITS) <= (PR.TOL_BF16 if bf else PR.TOL_LOGITS)
    bar = 0.2 if act8 else 0.1 if bf else 0.01
    for kind, lo, n in tensors:
        a, b = got[2][lo:lo + n], g[lo:lo + n]
        assert np.linalg.norm(a - b) <= bar * (np.linalg.norm(b) + 0.01 * np.linalg.norm(g)), (kind, lo)


@pytest.mark.parametrize("unfused", [False, True])
@pytest.mark.parametrize("dtype", [lpp.FP32, lpp.BF16])
def test_concat_of_a_tensor_with_itself(dtype, unfused):
    """A 1x1 conv over concat(x, x) is one over x with the sum of its halves: the
    reference net; the gradients of the halves are that of their sum."""
    def make(twice):
        m = PM.Model("twice", (8, 8, 8), 8)
        x = m.conv(-1, 16, 3, bias=True)
        t = m.conv(m.concat(x, x) if twice else x, 16, 1, 1, 0)
        m.linear(m.gap(m.conv(t, 16, 3, 2)), 8)
        return m.assign_blocks([1])
    m, one = make(True), make(False)
    img, lab, x, tensors = inputs(m, 8, 23, True)
    lo, n = tensors[2][1:]
    assert tensors[2][0] == "conv_w" and n == 16 * 32
    w = x[lo:lo + n].reshape(16, 2, 16)
    loss, z, g = reference(one, img, lab, np.concatenate([x[:lo], w.sum(1).ravel(), x[lo + n:]]))
    half = g[lo:lo + n // 2].reshape(16, 1, 16)
    g = np.concatenate([g[:lo], np.broadcast_to(half, (16, 2, 16)).ravel(), g[lo + n // 2:]])
    got = step(m, img, lab, x, 0, dtype, steps=2, unfused=unfused)
    bar = 0.1 if dtype == lpp.BF16 else 0.01     # (as above)
    for kind, at, k in tensors:
        a, b = got[2][at:at + k], g[at:at + k]
        assert np.linalg.norm(a - b) <= bar * (np.linalg.norm(b) + 0.01 * np.linalg.norm(g)), (kind, at)
