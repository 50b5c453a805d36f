"""ReLU decisions read off 8-bit checkpoints whose groups hold an infinity: a step
with LPP_ACT8 lets the gradient through where a step without it does."""
import numpy as np
import pytest

from paper_2203_06638_amd import lpp
from paper_2203_06638_amd import models as PM
from tests.test_gpu_act8_step import inputs, step

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def chain(channels, bias):
    m = PM.Model("chain", (3, 6, 6), 8)
    t = m.relu(m.conv(-1, channels, 3, bias=bias))
    m.linear(m.gap(m.conv(t, 16, 1, 1, 0)), 8)
    return m.assign_blocks([1])


def fire(channels, bias):
    m = PM.Model("fire", (3, 6, 6), 8)
    t = m.conv(-1, 8, 1, 1, 0)
    a = m.relu(m.conv(t, channels, 1, 1, 0, bias=bias))
    b = m.relu(m.conv(t, 16, 3, bias=bias))
    m.linear(m.gap(m.conv(m.concat(a, b), 16, 1, 1, 0)), 8)
    return m.assign_blocks([1])


@pytest.mark.parametrize("unfused", [False, True])
@pytest.mark.parametrize("dtype,net,channels,bias", [
    (lpp.FP32, chain, 32, True), (lpp.FP32, chain, 32, False), (lpp.FP32, chain, 20, True), (lpp.FP32, chain, 20, False),
    (lpp.BF16, chain, 32, True), (lpp.BF16, chain, 24, True), (lpp.FP32, fire, 24, True), (lpp.BF16, fire, 24, True)])
def test_relu_decisions_beside_an_infinity(dtype, net, channels, bias, unfused):
    """Channel 3 of the first ReLU is infinite in every pixel, channel 5 negative
    in every pixel, the others finite.  The loss is NaN, so the gradient is NaN
    wherever a ReLU passes it on: at the same entries with 8-bit checkpoints."""
    m = net(channels, bias)
    img, lab, x, tensors = inputs(m, 2, 21, True)
    img = np.abs(img) + np.float32(0.25)
    at = 0 if net is chain else 1
    convs = [t for t in tensors if t[0] == "conv_w"]
    if net is fire:     # a first conv that keeps its input positive
        x[convs[0][1]:convs[0][1] + convs[0][2]] = 0.5
    kind, lo, n = convs[at]
    w = x[lo:lo + n].reshape(channels, -1)
    w[3], w[5] = 3e38, -np.abs(w[5]) - np.float32(0.01)
    if bias:
        x[lo + n + 5] = -1
    a = step(m, img, lab, x, 0, dtype, unfused=unfused)[2]
    b = step(m, img, lab, x, 0, dtype, unfused=unfused, act8=True)[2]
    own = np.isfinite(a[lo:lo + n]).reshape(channels, -1)
    assert own[5].all() and not own[3].any() and (~own).all(1).sum() > 1 + channels // 8
    assert np.array_equal(np.isfinite(a), np.isfinite(b))
