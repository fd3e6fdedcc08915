"""A reference whose softmax is NaN: the divergence, and with it the loss and the
gradient, wherever in the row the reason lies."""
import math

import pytest

from paper_2304_13724_amd import ranking

import torch

from test_gpu_policy import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("cols", [50, 3000, 20_001, 80_001])
@pytest.mark.parametrize("at", ["first", "last"])
def test_beside_a_probability_of_zero(dtype, value, cols, at):
    """Rows: an item of probability 0 with such a reference; the same excluded; none."""
    dtype, i = TYPES[dtype], 0 if at == "first" else cols - 1
    g = torch.Generator().manual_seed(cols)
    x = torch.randn(3, cols, generator=g).to(dtype)
    y = (x.float() + 0.1 * torch.randn(3, cols, generator=g)).to(dtype)
    x[:, i] = -300.0  # e^-300: 0 in 32 bits
    y[:2, i] = value
    ex = torch.zeros(3, cols, dtype=torch.bool)
    ex[1, i] = True
    x, y, ex = x.cuda(), y.cuda(), ex.cuda()
    given = torch.full((3,), cols // 2, dtype=torch.int32).cuda()
    old, adv = torch.full((3,), -math.log(cols)).cuda(), torch.ones(3).cuda()
    for weight in (0.0, 0.1):
        o = dict(reference=y, kl_weight=weight, excluded=ex)
        r, grad = ranking.policy_loss_and_grad(x, given, adv, old, **o)
        leaf = x.clone().requires_grad_()
        r2 = ranking.policy_loss(leaf, given, adv, old, **o)
        r2.loss.sum().backward()
        for r, grad in ((r, grad), (r2, leaf.grad)):
            assert r.kl.isnan().tolist() == [True, False, False]
            assert r.loss.isnan().tolist() == [weight != 0, False, False]
            assert torch.isfinite(r.log_prob).all()
            assert grad[0].isnan().all() if weight else torch.isfinite(grad[0]).all()
            assert torch.isfinite(grad[1:]).all() and grad[1, i] == 0
