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
