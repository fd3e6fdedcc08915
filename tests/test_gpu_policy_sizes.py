"""The policy loss at sizes on both sides of what a thread, a workgroup and a part
hold, within the bounds of policy_bounds.py, computed on the GPU in 64 bits."""
import pytest

from paper_2304_13724_amd import ranking

import torch

import policy_bounds as pb

pytestmark = pytest.mark.gpu

# vectors of 16 bytes that 64, 256, 512 and 1,024 threads hold (of four and nine each),
# and one more or less; rows from which the threads hold more
VECS = [256, 257, 1280, 1281, 2304, 2305, 2560, 2561, 4608, 4609, 5120, 5121, 9216, 9217]


def on_gpu(c):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vecs", VECS)
@pytest.mark.parametrize("rows", [3, 515])
def test_held_vectors(dtype, vecs, rows):
    n = 16 // dtype.itemsize
    cols = vecs * n + (1 if vecs % 2 else n - 1)
    if rows > 3 and vecs > 5200:
        rows = 40
    c = on_gpu(pb.case(rows, cols, dtype, vecs, excluded=vecs % 3 == 0))
    full = vecs % 5 != 0
    o = dict(reference=c["y"] if full else None, kl_weight=pb.KL, clip_low=pb.LO, clip_high=pb.HI,
             reference_log_prob=None if full else c["ref_lp"], temperature=c["t"], excluded=c["ex"])
    at = (c["x"], c["given"].int(), c["adv"], c["old"])
    want = pb.reference(
        c["x"].double(), c["given"], c["adv"].double(), c["old"].double(), c["t"], pb.LO, pb.HI,
        pb.KL, y=c["y"].double() if full else None, ref_lp=None if full else c["ref_lp"].double(),
        excluded=c["ex"], g=c["weight"].double())
    r, grad = ranking.policy_loss_and_grad(*at, c["weight"], **o)
    leaf = c["x"].clone().requires_grad_()
    r2 = ranking.policy_loss(leaf, *at[1:], **o)
    r2.loss.backward(c["weight"])
    for got, g in ((r, grad), (r2, leaf.grad)):
        for name in ("loss", "log_prob", "kl"):
            v, tol = want[name]
            assert ((getattr(got, name).detach().double() - v).abs() <= tol).all(), name
        v, err = want["grad"]
        assert ((g.double() - v).abs() <= pb.allowed(v, err, dtype)).all()


@pytest.mark.parametrize("vecs", [3, 257, 1281, 2305, 2561, 4609, 9217])
@pytest.mark.parametrize("flat", ["policy", "reference"])
def test_policies_far_apart(vecs, flat):
    """One of the two flat, the other with one item almost alone: sums that say
    nothing of each other."""
    cols = 4 * vecs + 1
    c = on_gpu(pb.case(4, cols, torch.float32, vecs))
    peak = 0.01 * c["x"]
    peak[torch.arange(4), torch.arange(4) * (cols // 5)] = 25.0
    c["x"], c["y"] = (torch.zeros_like(peak), peak) if flat == "policy" else (peak, 0.0 * peak)
    D, _, lnS, _ = pb.softmax_of(c["x"].double(), c["t"], None)
    c["old"] = (-D.gather(1, c["given"][:, None]) - lnS)[:, 0].sub(0.1).float()  # a ratio of 1.1
    o = dict(reference=c["y"], kl_weight=pb.KL, clip_low=pb.LO, clip_high=pb.HI,
             temperature=c["t"])
    at = (c["x"], c["given"].int(), c["adv"], c["old"])
    want = pb.reference(
        c["x"].double(), c["given"], c["adv"].double(), c["old"].double(), c["t"], pb.LO, pb.HI,
        pb.KL, y=c["y"].double(), g=c["weight"].double())
    r, grad = ranking.policy_loss_and_grad(*at, c["weight"], **o)
    for got in (r, ranking.policy_loss(*at, **o)):
        for name in ("loss", "log_prob", "kl"):
            v, tol = want[name]
            assert ((getattr(got, name).double() - v).abs() <= tol).all(), name
    v, err = want["grad"]
    assert ((grad.double() - v).abs() <= pb.allowed(v, err, torch.float32)).all()


def test_the_divergence_is_as_exact_as_its_terms():
    """Few items, scores near the reference's: the sums' own rounding is not in the
    divergence.  Of the terms, exp(-D) and exp(-E) are off by some (D + E + 2) / 2 steps
    of 2^-24 each, at random: on the root mean square over rows of 16 items, below 4
    steps of the divergence's own scale, the mean difference of 0.3."""
    c = on_gpu(pb.case(4096, 16, torch.float32, 2))
    want = pb.reference(
        c["x"].double(), c["given"], c["adv"].double(), c["old"].double(), c["t"], pb.LO, pb.HI,
        pb.KL, y=c["y"].double())["kl"][0]
    at = (c["x"], c["given"].int(), c["adv"], c["old"])
    for call in (ranking.policy_loss, lambda *a, **o: ranking.policy_loss_and_grad(*a, **o)[0]):
        kl = call(*at, reference=c["y"], kl_weight=pb.KL, temperature=c["t"]).kl
        assert (kl.double() - want).square().mean().sqrt() <= 4 * 2.0 ** -24 * 0.3


@pytest.mark.parametrize("cols", [18_432, 18_433, 20_480, 20_481, 25_600, 36_865, 512_063])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_parts(dtype, cols):
    """Rows in parts: whole ones, a last one of one score, one that is left whole by its
    exclusions alone, rows that fill the batch up."""
    cols *= 4 // dtype.itemsize
    c = on_gpu(pb.case(7, cols, dtype, 3, excluded=True))
    c["ex"][2, :cols // 2] = True
    c["ex"][torch.arange(7), c["given"]] = False
    D, _, lnS, _ = pb.softmax_of(c["x"].double(), c["t"], c["ex"])
    c["old"] = (-D.gather(1, c["given"][:, None]) - lnS)[:, 0].sub(0.1).float()
    o = dict(reference=c["y"], kl_weight=pb.KL, clip_low=pb.LO, clip_high=pb.HI,
             temperature=c["t"], excluded=c["ex"])
    want = pb.reference(
        c["x"].double(), c["given"], c["adv"].double(), c["old"].double(), c["t"], pb.LO, pb.HI,
        pb.KL, y=c["y"].double(), excluded=c["ex"], g=c["weight"].double())
    given = c["given"].int()
    given[5] = -1
    leaf = c["x"].clone().requires_grad_()
    r = ranking.policy_loss(leaf, given, c["adv"], c["old"], **o)
    r.loss.backward(c["weight"])
    rows = torch.tensor([0, 1, 2, 3, 4, 6]).cuda()
    for name in ("loss", "log_prob", "kl"):
        got = getattr(r, name).detach().double()
        v, tol = want[name]
        assert ((got - v).abs() <= tol)[rows].all(), name
        assert got[5] == 0
    v, err = want["grad"]
    assert ((leaf.grad.double() - v).abs() <= pb.allowed(v, err, dtype))[rows].all()
    assert (leaf.grad[5] == 0).all()
