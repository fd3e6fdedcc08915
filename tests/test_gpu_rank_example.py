"""The ranking operators together, as examples/rank_items.py uses them."""
import importlib.util
import os

import numpy as np
import pytest

from paper_2304_13724_amd import ranking

import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "rank_items", os.path.join(ROOT, "examples", "rank_items.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_learns_and_answers():
    r = _example().main(["--epochs", "2", "--steps", "60", "--batch", "256", "--top", "5"])
    losses, answer, w = r["losses"], r["answer"], r["workload"]
    assert np.isfinite(losses).all() and np.mean(losses[-10:]) < np.mean(losses[:10])
    item, lp = answer.top_item.cpu().numpy(), answer.top_log_prob.cpu().numpy()
    assert ((item >= 0) & (item < w.m)).all() and (np.diff(lp, axis=1) <= 0).all()
    for i, u in enumerate(r["who"]):  # nothing already rated is recommended
        assert not set(item[i]) & set(w.cols[w.rows == u].tolist())
    # the 8-bit scores of the recommended items are within the two sides' rounding
    # (half a step of each factor, k of them) of the fp32 ones
    U, V = r["U"][:len(item)].double(), r["V"].double()
    exact = U @ V.t()
    q = ranking.Catalogue(r["V"]).scores(r["U"][:len(item)]).double()
    step_u, step_v = U.abs().amax(1) / 254, V.abs().amax(1) / 254
    bound = (U.abs().sum(1)[:, None] * step_v[None] + V.abs().sum(1)[None] * step_u[:, None]
             + U.shape[1] * step_u[:, None] * step_v[None]) * 1.001
    assert ((q - exact).abs() <= bound).all()


def test_clipped_training_matches_plain_pytorch():
    """One training step through the operators against PyTorch's own functions."""
    g = torch.Generator(device="cuda").manual_seed(1)
    U = torch.randn(64, 32, generator=g, device="cuda")
    V = torch.randn(777, 32, generator=g, device="cuda")
    given = torch.randint(0, 777, (64,), generator=g, device="cuda")
    ours = [U.clone().requires_grad_(), V.clone().requires_grad_()]
    r = ranking.log_probs(ours[0] @ ours[1].t(), given.int(), temperature=0.5)
    (-(r.log_prob + 0.1 * r.entropy).mean()).backward()
    norm = ranking.clip_grad_norm([x.grad for x in ours], 0.01)
    theirs = [U.double().requires_grad_(), V.double().requires_grad_()]
    lp = torch.log_softmax(theirs[0] @ theirs[1].t() / 0.5, 1)
    entropy = -(lp.exp() * lp).sum(1)
    (-(lp[torch.arange(64), given] + 0.1 * entropy).mean()).backward()
    want = torch.nn.utils.clip_grad_norm_(theirs, 0.01)
    assert abs(norm.item() - want.item()) < 1e-4 * want.item()
    for a, b in zip(ours, theirs):
        assert (a.grad.double() - b.grad).norm() < 1e-4 * b.grad.norm()
