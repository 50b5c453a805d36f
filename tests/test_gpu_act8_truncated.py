"""LPP_ACT8 in truncated steps: what is packed and unpacked is what the partition's
backward pass reads, and a checkpoint that a step does not write is not read."""
import numpy as np
import pytest

from paper_2203_06638_amd import lpp
from paper_2203_06638_amd import models as PM
from tests.test_gpu_act8_step import inputs, step

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def relu_chain():
    """Five units, a block each: four convs with ReLU, and the head."""
    m = PM.Model("relu_chain", (3, 8, 8), 8)
    t = m.relu(m.conv(-1, 16, 3, bias=True))
    for k in (1, 3, 1):
        m.new_unit()
        t = m.relu(m.conv(t, 16, k, bias=True))
    m.new_unit()
    m.linear(m.gap(t), 8)
    return m.assign_blocks([1, 2, 3, 4, 5])


def norm_chain():
    """Three units, a block each: a conv, a norm and a 1x1 conv, a norm and the head."""
    m = PM.Model("norm_chain", (3, 8, 8), 8)
    t = m.conv(-1, 32, 3, bias=True)
    m.new_unit()
    t = m.conv(m.rmsnorm(t), 32, 1, 1, 0)
    m.new_unit()
    m.linear(m.gap(m.rmsnorm(t)), 8)
    return m.assign_blocks([1, 2, 3])


def fire_chain():
    """A block that ends in one branch of a concat of two fused conv + ReLU."""
    m = PM.Model("fire_chain", (3, 8, 8), 8)
    t = m.relu(m.conv(-1, 16, 3, bias=True))
    a = m.relu(m.conv(t, 16, 1, 1, 0, bias=True))
    m.new_unit()
    b = m.relu(m.conv(t, 16, 3, bias=True))
    m.linear(m.gap(m.concat(a, b)), 8)
    return m.assign_blocks([1, 2])


def counted(m, family, part, batch=4):
    """(launches, work) of a kernel family in one step of a partition."""
    img, lab, x, _ = inputs(m, batch, 5)
    with lpp.Context(m, K=1, batch=batch, act8=True) as ctx:
        ctx.set_params(x)
        ctx.timer_enable(family)
        ctx.step(0, torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda(), part, 0.1)
        _, n, work = ctx.timer_read()
        return n, work


def test_steps_pack_what_their_backward_reads():
    # a conv reads its input for the weight gradient and its output for the ReLU;
    # the 3x3 conv's input is unpacked
    m = relu_chain()
    assert [counted(m, "act8_pack", p)[0] for p in range(6)] == [4, 4, 4, 3, 2, 0]
    assert [counted(m, "act8_unpack", p)[0] for p in range(6)] == [1, 0, 0, 1, 0, 0]
    # the convs' outputs are packed for the norms' gradients, the norms' by the norms: 4 bytes read, 4 written and
    # one more of checkpoint a value; the second norm's output is read by no backward
    m = norm_chain()
    assert [counted(m, "act8_pack", p)[0] for p in range(4)] == [2, 2, 2, 1]
    values = 4 * 8 * 8 * 32
    assert [counted(m, "rmsnorm", p)[1] for p in range(4)] == [17 * values, 16 * values, 17 * values, 16 * values]
    # block 2 wants the second branch alone
    m = fire_chain()
    assert [counted(m, "act8_pack", p)[0] for p in range(3)] == [3, 3, 2]
    assert [counted(m, "act8_unpack", p)[0] for p in range(3)] == [3, 2, 2]


@pytest.mark.parametrize("dtype", [lpp.FP32, lpp.BF16])
@pytest.mark.parametrize("net", [relu_chain, norm_chain, fire_chain])
def test_partitions_in_turn(net, dtype):
    """Steps of one worker over all partitions in turn, new images each, give the
    bits of a context that runs the one step."""
    m = net()
    with lpp.Context(m, K=1, batch=4, dtype=dtype, act8=True) as ctx:
        for k, part in enumerate([m.P, 1, 0, m.P, 2, 0, 1, m.P]):
            img, lab, x, _ = inputs(m, 4, 30 + k, True)
            ctx.set_params(x)
            ctx.step(0, torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda(), part, 0.1)
            ctx.sync()
            got = ctx.get_loss(0), ctx.get_grad(0)
            want = step(m, img, lab, x, part, dtype, act8=True)
            assert got[0] == want[0] and np.array_equal(got[1], want[2]), (k, part)
