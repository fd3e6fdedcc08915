"""Rows of scores that go in parts give what the same scores give in a row that a
workgroup holds: infinities, NaN, masks of the lowest value and stretches of them."""
import math

import pytest

from paper_2304_13724_amd import ranking

import torch

import policy_bounds as pb
from test_gpu_policy import TYPES, args, options, special

pytestmark = pytest.mark.gpu

# scores past which rows go in parts, without a gradient and with one, twice that in 16 bits
VALUE, STEP = 18_432, 36_864


def longer(dtype, step):
    return (STEP if step else VALUE) * 4 // dtype.itemsize + 1_703


def spread(c, cols):
    """The same rows with other items between theirs, all of them excluded, whose scores
    are NaN and infinities."""
    rows, k = c["x"].shape
    at = torch.arange(k) * (cols // k) + 5  # items in every part
    new = {**c, "x": torch.full((rows, cols), math.nan, dtype=c["x"].dtype),
           "y": torch.full((rows, cols), math.inf, dtype=c["x"].dtype),
           "ex": torch.ones(rows, cols, dtype=torch.bool)}
    new["x"][:, at], new["y"][:, at] = c["x"], c["y"]
    new["ex"][:, at] = c["ex"]
    inside = (c["given"] >= 0) & (c["given"] < k)
    new["given"] = torch.where(inside, at[c["given"].clamp(0, k - 1)], c["given"])
    new["given"][c["given"] == k] = cols
    return new, at


def results(c, kind, step, weighted=True):
    """(loss, log_prob, kl, gradient) on the CPU, by policy_loss_and_grad or through autograd."""
    a, o, w = args(c), options(c, kind), c["weight"].cuda()
    if not weighted:
        o["kl_weight"] = 0.0
    if step:
        r, grad = ranking.policy_loss_and_grad(*a, w, **o)
    else:
        a[0].requires_grad_()
        r = ranking.policy_loss(*a, **o)
        (grad,) = torch.autograd.grad(r.loss, a[0], w)
    return [t.detach().cpu() for t in (*r, grad)]


def alike(got, want, dtype, c):
    """The same NaN and infinities; otherwise within twice the bounds that
    test_special_rows derives for the same rows."""
    def agree(x, y, tol):
        x, y = x.double(), y.double()
        assert torch.equal(x.isnan(), y.isnan()) and torch.equal(x.isinf(), y.isinf())
        off = torch.where(torch.isfinite(y), (x - y).abs() - tol, -1.0)
        assert (off <= 0).all(), (off.max(), (off > 0).nonzero()[:5])

    def size(t):
        return t.double().abs().nan_to_num(0.0, 0.0, 0.0)

    (loss, lp, kl, grad), (loss0, lp0, kl0, grad0) = got, want
    agree(lp, lp0, 2 * 6e-6 + 2.0 ** -23 * size(lp0))
    agree(kl, kl0, 2 * 5.7e-4 + 2.0 ** -23 * size(kl0))
    agree(loss, loss0, 2 * 6.2e-6 * (size(loss0) + 1) + 2 * 0.06 * 5.7e-4)
    row = c["weight"].double().abs()[:, None] / c["t"] * (
        (size(loss0) + 0.06 * 30)[:, None] * 320 * pb.U + 0.06 * 2e-3)
    agree(grad, grad0, 2 * row + torch.finfo(dtype).eps * size(grad0) + 2 * pb.TINY[dtype])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["none", "shown", "full"])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("step", [False, True])
def test_special_rows(dtype, kind, weighted, step):
    held = special(TYPES[dtype])
    parts, at = spread(held, longer(TYPES[dtype], step))
    want = results(held, kind, step, weighted)
    got = results(parts, kind, step, weighted)
    between = torch.ones(parts["x"].shape[1], dtype=torch.bool)
    between[at] = False
    assert (got[3][:, between] == 0).all()
    alike(got[:3] + [got[3][:, at]], want, TYPES[dtype], held)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("value", ["lowest", -300.0, -math.inf])
@pytest.mark.parametrize("first", [True, False])
def test_a_masked_stretch_without_a_reference(dtype, step, value, first):
    """Items whose probability is 0 (in 32 bits) add nothing to the divergence, though
    the reference's is 0 too: in whole parts of them as well."""
    dtype = TYPES[dtype]
    cols = longer(dtype, step)
    c = pb.case(5, cols, dtype, 3, excluded=False)  # t = 1
    part = 16 // dtype.itemsize * 1280
    low = torch.finfo(dtype).min if value == "lowest" else value
    mask = torch.zeros(5, cols, dtype=torch.bool)
    for i, parts in enumerate((1, 2, 1.7, 3)):  # of the longest parts
        n = min(int(parts * part), cols - 1)
        mask[i, :n] = first
        mask[i, cols - n:] |= not first
    c["given"] = (~mask).int().argmax(1)  # the first one left
    c["x"][mask], c["y"][mask] = low, -math.inf
    D, _, lnS, _ = pb.softmax_of(c["x"].double(), c["t"], mask)
    c["old"] = (-D.gather(1, c["given"][:, None]) - lnS)[:, 0].sub(0.1).float()  # a ratio of 1.1
    expected = pb.reference(
        c["x"].double(), c["given"], c["adv"].double(), c["old"].double(), c["t"], pb.LO, pb.HI,
        pb.KL, y=c["y"].double(), excluded=mask, g=c["weight"].double())
    loss, lp, kl, grad = results(c, "full", step)
    for name, got in (("loss", loss), ("log_prob", lp), ("kl", kl)):
        v, tol = expected[name]
        assert ((got.double() - v).abs() <= tol).all(), (name, got)
    v, err = expected["grad"]
    assert ((grad.double() - v).abs() <= pb.allowed(v, err, dtype)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("step", [False, True])
def test_probabilities_that_vanish_beside_another_part(dtype, step):
    """An item with a reference of 0 counts where its probability is not 0 beside the
    whole row, whatever it is beside its own part: in the first part, whose other items
    are 60 below the row's largest in the last row, and the item 45 below them."""
    dtype = TYPES[dtype]
    cols = longer(dtype, step)
    x = torch.zeros(4, cols, dtype=dtype)
    x[3, :cols // 2] = -60.0  # more than the longest part
    y = x.clone()
    at = 64
    for i, below in enumerate((0.0, 30.0, 50.0, 105.0)):
        x[i, at], y[i, at] = -below, -math.inf
    c = dict(x=x, y=y, given=torch.full((4,), cols - 1), ex=None, adv=torch.full((4,), -1.0),
             old=torch.full((4,), -math.log(cols)), weight=torch.ones(4), t=1.0)
    loss, lp, kl, grad = results(c, "full", step)
    assert (kl[:3] == math.inf).all() and torch.isfinite(lp).all()
    assert abs(kl[3]) < 1e-6 and torch.isfinite(loss[3])
    assert torch.isfinite(grad[3]).all() and grad[3, at] == 0 and grad[3, cols - 1] > 0.5


@pytest.mark.parametrize("rows,cols,drift", [(200, 5_000, 0.3), (200, 5_000, 0.002),
                                             (100, 18_433, 0.3), (100, 18_433, 0.03),
                                             (40, 100_003, 0.03), (20, 625_001, 0.03)])
def test_the_divergence_is_as_exact_as_its_terms(rows, cols, drift):
    """Held rows and parts.  With u = 2^-24: exp(-D) and exp(-E) of an item are off by at
    most 2 u of themselves each, whichever way, and the divergence by their difference's
    share, on the root mean square 2 sqrt(2) u sqrt(sum p^2); the roundings of D and E
    change it at second order, those of the sums by steps of the terms' differences
    (drift), below 1.2 u sqrt(sum p^2); log2 e in 32 bits by u, the result by u of
    itself."""
    c = {k: v.cuda() if isinstance(v, torch.Tensor) else v
         for k, v in pb.case(rows, cols, torch.float32, 3, drift=drift).items()}  # t = 1
    lp, lq = torch.log_softmax(c["x"].double(), 1), torch.log_softmax(c["y"].double(), 1)
    want = (lp.exp() * (lp - lq)).sum(1)
    spread = lp.mul(2).exp().sum(1).mean().sqrt()
    bound = 4 * pb.U * spread + 2 * pb.U * want.mean()
    assert bound < 0.05 * want.mean()
    at = (c["x"], c["given"].int(), c["adv"], c["old"])
    for call in (ranking.policy_loss, lambda *a, **o: ranking.policy_loss_and_grad(*a, **o)[0]):
        kl = call(*at, reference=c["y"], kl_weight=pb.KL, temperature=c["t"]).kl
        assert (kl.double() - want).square().mean().sqrt() <= bound


@pytest.mark.parametrize("cols", [18_433, 100_003, 1_500_001])
def test_the_policy_is_its_own_reference(cols):
    c = pb.case(6, cols, torch.float32, cols)
    c["y"] = c["x"]
    loss, lp, kl, grad = results(c, "full", False)
    assert (kl == 0).all()
    c["adv"].zero_()
    assert (results(c, "full", False)[3] == 0).all()


@pytest.mark.parametrize("step", [False, True])
def test_more_parts_than_threads_of_the_join(step):
    """293 parts: items without a reference, and the row's largest, in the last ones."""
    cols = 1_500_001
    c = pb.case(4, cols, torch.float32, 3)  # t = 1
    last = slice(cols - 20_000, cols)
    mask = torch.zeros(4, cols, dtype=torch.bool)
    mask[0, last] = True  # masked in whole parts
    c["x"][0, last], c["y"][0, last] = torch.finfo(torch.float32).min, -math.inf
    c["x"][1, last] += 200.0  # all of the probability
    c["y"][1, last] += 200.0
    c["given"] = torch.tensor([7, cols - 9, cols - 1, 3])
    D, _, lnS, _ = pb.softmax_of(c["x"].double(), c["t"], mask)
    c["old"] = (-D.gather(1, c["given"][:, None]) - lnS)[:, 0].sub(0.1).float()  # a ratio of 1.1
    expected = pb.reference(
        c["x"].double(), c["given"], c["adv"].double(), c["old"].double(), c["t"], pb.LO, pb.HI,
        pb.KL, y=c["y"].double(), excluded=mask, g=c["weight"].double())
    c["y"][3, cols - 5] = -math.inf
    loss, lp, kl, grad = results(c, "full", step)
    for name, got in (("loss", loss), ("log_prob", lp), ("kl", kl)):
        v, tol = expected[name]
        assert ((got.double() - v).abs() <= tol)[:3].all(), (name, got)
    v, err = expected["grad"]
    assert ((grad.double() - v).abs() <= pb.allowed(v, err, torch.float32))[:3].all()
    assert kl[3] == math.inf and torch.isfinite(lp[3])
