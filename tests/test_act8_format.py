"""The bounds that the 8-bit format promises, on its definition (float64, no GPU)."""
import torch

from tests import act8ref as R


def test_step_and_error_bounds():
    """A step is more than amax / 127.5, where rint reaches 128 (a tie, to even), and
    at most amax / 63.75, where half of it would do, but 2^-126 at least; a value
    is off by half a step, a saturated one by less than one."""
    g = torch.Generator().manual_seed(2)
    f = torch.finfo(torch.float32)
    edge = torch.tensor([127.5, 63.75, 127.0, 127.49, 127.51, 64.0, 1.0, 1.9921875, 1.99])
    x = torch.cat([torch.exp(torch.randn(4000, generator=g, dtype=torch.float64) * 20), edge.double(),
                   edge.double() * 2.0 ** -126, edge.double() * 2.0 ** 120,
                   torch.tensor([f.tiny, f.tiny / 8, f.max, f.max / 2, 1e-37, 0.0], dtype=torch.float64)])
    x = x[x <= f.max][:, None] * torch.tensor([1.0, -0.73, 0.011, 0.0], dtype=torch.float64)
    codes, s = R.pack(x)
    step, amax = torch.exp2(s[:, 0].double() - 133), x.abs().amax(1)
    top, low = amax >= 127.5 * 2.0 ** 121, amax < 63.75 * 2.0 ** -126
    assert top.any() and low.any()
    assert (step > amax / 127.5)[~top].all() and (step <= amax / 63.75)[~low].all()
    assert (step == 2.0 ** -126)[low].all() and (step == 2.0 ** 121)[top].all()
    err = (R.values(codes, s, 4) - x).abs()
    assert (err <= step[:, None] / 2)[~top].all() and (err < step[:, None])[top].all()
