"""The 4-bit catalogue, dropout, the policy loss and clipping together, as
examples/rank_items.py uses them: gradients of the whole step against 64 bits,
and the loop runs."""
import math
import os
import sys

import numpy as np
import pytest

from paper_2304_13724_amd import ranking

import torch

from philox import words

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def plain_step(u, v, u0, v0, shown, old, advantage, kl_weight, t, p, seed, offset):
    """The same in 64 bits on the CPU, by automatic differentiation."""
    u, v = u.double().requires_grad_(), v.double().requires_grad_()
    kept = torch.from_numpy((words(seed, offset, u.numel()) >= int(p * 2.0 ** 32)).reshape(u.shape))
    lp = torch.log_softmax((u * kept * float(np.float32(1 / (1 - p)))) @ v.t() / t, 1)
    lq = torch.log_softmax(u0.double() @ v0.double().t() / t, 1)
    at = lp.gather(1, shown.long()[:, None])[:, 0]
    rho, a = (at - old.double()).exp(), advantage.double()
    # 0.2 as 32 bits hold it
    lo, hi = 1 - float(np.float32(0.2)), 1 + float(np.float32(0.2))
    kl = (lp.exp() * (lp - lq)).sum(1)
    loss = -torch.minimum(rho * a, rho.clamp(lo, hi) * a) + kl_weight * kl
    loss.mean().backward()
    return loss.detach(), rho.detach(), u.grad, v.grad


@pytest.mark.parametrize("rows,items,k,p", [(64, 500, 64, 0.1), (33, 1001, 50, 0.5), (5, 70, 7, 0.0)])
def test_gradients_of_a_step(rows, items, k, p):
    import rank_items
    g = torch.Generator().manual_seed(rows)
    u, v = torch.randn(rows, k, generator=g) * 0.5, torch.randn(items, k, generator=g) * 0.5
    u0, v0 = (x + 0.05 * torch.randn(x.shape, generator=g) for x in (u, v))
    draws = torch.Generator(device="cuda").manual_seed(1)
    catalogue = ranking.Catalogue(v.cuda(), bits=4)
    shown, old = rank_items.show(catalogue, u.cuda(), 1.0, draws)
    advantage = torch.randn(rows, generator=g)
    r, gu, gv = rank_items.feedback_step(u.cuda(), v.cuda(), (u0.cuda(), v0.cuda()), shown, old,
                                         advantage.cuda(), 0.05, 1.0, p, 3, 40)
    loss, rho, wu, wv = plain_step(u, v, u0, v0, shown.cpu(), old.cpu(), advantage, 0.05, 1.0, p, 3,
                                   40)
    # no ratio where the slope jumps, within the error of the ratio below
    assert ((rho - 0.8).abs() > 1e-4 * rho).all() and ((rho - 1.2).abs() > 1e-4 * rho).all()
    # A score is a sum of k products of at most m = max|u| max|v| / (1 - p): off by at
    # most (k + 2) k m 2^-24, both policies' alike; ln p by twice that and (4 D + 58) 2^-24,
    # D the range of the scores; the ratio by as much of itself, and the divergence's
    # terms (below the range) by three times it.
    m = u.abs().max() * v.abs().max() / (1 - p)
    score = ((k + 2) * k * m * 2.0 ** -24).item()
    spread = 2 * k * m.item()
    e = 2 * score + (4 * spread + 58) * 2.0 ** -24
    assert ((r.loss.cpu() - loss).abs() <= e * (rho * advantage.abs().double() * 1.01 + 3 * 0.05 * (
        1 + spread)) + 1e-6).all()
    # a row's gradient dx has sum |dx| <= (2 |slope| + 0.05 * 2 spread) / rows, off by as
    # much of it as ln p is, and 3 e for each probability; u's gradient sums it with |v|
    dx = (2 * rho * advantage.abs() + 0.1 * spread) / rows
    near = 5 * e + (items + 10) * 2.0 ** -24
    assert ((gu.cpu() - wu).abs().amax(1) <= near * dx * v.abs().max() / (1 - p) + 1e-9).all()
    near += rows * 2.0 ** -24
    assert ((gv.cpu() - wv).abs().max() <= near * dx.sum() * u.abs().max() / (1 - p) + 1e-9)


def test_ratios_of_what_a_4_bit_catalogue_showed():
    """Before any step the policy differs from what served by the 4 bits alone: with the
    served scores in place of its own the ratio is exactly 1."""
    import rank_items
    u, v = torch.randn(50, 64).cuda() * 0.3, torch.randn(2000, 64).cuda() * 0.3
    c = ranking.Catalogue(v, bits=4)
    shown, old = rank_items.show(c, u, 0.7, torch.Generator(device="cuda").manual_seed(2))
    assert shown.min() >= 0 and shown.max() < 2000
    a = torch.randn(50).cuda()
    r = ranking.policy_loss(c.scores(u), shown, a, old, temperature=0.7)
    # both log probabilities are off by at most 2e-6 (the sums of 2,000 terms)
    assert ((r.loss + a).abs() <= 8e-6 * a.abs()).all()


def test_the_loop_runs():
    import rank_items
    got = rank_items.main(["--epochs", "1", "--steps", "5", "--batch", "256", "--feedback", "4",
                           "--dropout", "0.2", "--bits", "4"])
    assert len(got["rewards"]) == 4 and all(math.isfinite(x) for x in got["rewards"])
    assert torch.isfinite(got["U"]).all() and torch.isfinite(got["V"]).all()
    assert got["answer"].top_item.min() >= 0
    again = rank_items.main(["--epochs", "1", "--steps", "5", "--batch", "256", "--feedback", "4",
                             "--dropout", "0.2", "--bits", "4"])
    assert again["rewards"][0] == got["rewards"][0]
