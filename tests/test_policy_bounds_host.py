"""The 64-bit policy loss that the GPU tests compare with: against automatic
differentiation, difference quotients and a direct evaluation."""
import pytest
import torch

import policy_bounds as pb


def direct(x, c, kind):
    z = x / c["t"]
    if c["ex"] is not None:
        z = z.masked_fill(c["ex"], -torch.inf)
    lp = torch.log_softmax(z, 1)
    at = lp.gather(1, c["given"][:, None])[:, 0]
    rho = (at - c["old"].double()).exp()
    a = c["adv"].double()
    loss = -torch.minimum(rho * a, rho.clamp(1 - pb.LO, 1 + pb.HI) * a)
    if kind == "full":
        zy = c["y"].double() / c["t"]
        if c["ex"] is not None:
            zy = zy.masked_fill(c["ex"], -torch.inf)
        lq = torch.log_softmax(zy, 1)
        keep = lp > -torch.inf
        kl = (lp.exp() * torch.where(keep, lp - lq.masked_fill(~keep, 0.0), 0.0)).nan_to_num(0.0)
        loss = loss + pb.KL * kl.sum(1)
    if kind == "shown":
        u = c["ref_lp"].double() - at
        loss = loss + pb.KL * (u.exp() - 1 - u)
    return loss


def formula(c, kind, x=None):
    return pb.reference(
        c["x"].double() if x is None else x, c["given"], c["adv"].double(), c["old"].double(),
        c["t"], pb.LO, pb.HI, pb.KL if kind != "none" else 0.0,
        y=c["y"].double() if kind == "full" else None,
        ref_lp=c["ref_lp"].double() if kind == "shown" else None, excluded=c["ex"],
        g=c["weight"].double())


@pytest.mark.parametrize("kind", ["none", "shown", "full"])
@pytest.mark.parametrize("excluded", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 7), (9, 40)])
def test_gradient_by_autograd_and_by_differences(kind, excluded, rows, cols):
    c = pb.case(rows, cols, torch.float32, rows, excluded)
    got = formula(c, kind)
    x = c["x"].double().requires_grad_()
    loss = direct(x, c, kind)
    assert torch.allclose(got["loss"][0], loss.detach(), rtol=1e-12, atol=1e-12)
    (want,) = torch.autograd.grad(loss, x, c["weight"].double())
    if c["ex"] is not None:
        want = want.masked_fill(c["ex"], 0.0)
    assert torch.allclose(got["grad"][0], want.nan_to_num(0.0), rtol=1e-10, atol=1e-12)
    h = 1e-6
    for i, j in ((0, 0), (rows - 1, cols - 1), (rows // 2, int(c["given"][rows // 2]))):
        up, down = c["x"].double(), c["x"].double()
        up[i, j] += h
        down[i, j] -= h
        quotient = ((direct(up, c, kind) - direct(down, c, kind)) @ c["weight"].double()) / (2 * h)
        assert abs(quotient - got["grad"][0][i, j]) < 1e-7
