"""The policy loss and its gradient, against 64 bits within bounds by arithmetic
(policy_bounds.py), and the rows that its description names."""
import math

import pytest

from paper_2304_13724_amd import bgmf, ranking

import torch
from torch.autograd import forward_ad

import policy_bounds as pb

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SHAPES = [(1, 1), (3, 2), (5, 17), (2, 255), (4, 1024), (3, 2049), (3, 4099), (2, 18000),
          (5, 9001), (1, 100003), (700, 33), (2, 33000), (40, 12345)]


def options(c, kind):
    return dict(reference=c["y"].cuda() if kind == "full" else None,
                reference_log_prob=c["ref_lp"].cuda() if kind == "shown" else None,
                kl_weight=pb.KL if kind != "none" else 0.0, clip_low=pb.LO, clip_high=pb.HI,
                temperature=c["t"], excluded=None if c["ex"] is None else c["ex"].cuda())


def args(c):
    return [c[n].cuda() for n in ("x",)] + [c["given"].int().cuda(), c["adv"].cuda(), c["old"].cuda()]


def want(c, kind):
    return pb.reference(
        c["x"].double(), c["given"], c["adv"].double(), c["old"].double(), c["t"], pb.LO, pb.HI,
        pb.KL if kind != "none" else 0.0, y=c["y"].double() if kind == "full" else None,
        ref_lp=c["ref_lp"].double() if kind == "shown" else None, excluded=c["ex"],
        g=c["weight"].double())


def check(r, expected, grad=None):
    for n in ("loss", "log_prob", "kl"):
        v, tol = expected[n]
        off = (getattr(r, n).detach().cpu().double() - v).abs() - tol
        assert off.max() <= 0, (n, off.max())
    if grad is not None:
        v, err = expected["grad"]
        off = (grad.cpu().double() - v).abs() - pb.allowed(v, err, grad.dtype)
        assert off.max() <= 0, ("grad", off.max())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["none", "shown", "full"])
@pytest.mark.parametrize("excluded", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_values_and_gradient(dtype, kind, excluded, rows, cols):
    c = pb.case(rows, cols, TYPES[dtype], rows + cols, excluded)
    expected, a, o = want(c, kind), args(c), options(c, kind)
    check(ranking.policy_loss(*a, **o), expected)
    r, grad = ranking.policy_loss_and_grad(*a, c["weight"].cuda(), **o)
    check(r, expected, grad)
    leaf = a[0].clone().requires_grad_()
    r = ranking.policy_loss(leaf, *a[1:], **o)
    r.loss.backward(c["weight"].cuda())
    check(r, expected, leaf.grad)


def test_scores_near_the_reference_and_an_offset_between_them():
    """The bounds do not grow with an offset of 1000 between all of the scores."""
    c = pb.case(6, 5000, torch.float32, 3, drift=0.001)
    expected, a, o = want(c, "full"), args(c), options(c, "full")
    check(ranking.policy_loss(*a, **o), expected)
    c["y"] = (c["y"].double() + 1000.0).float()
    c2 = dict(c)
    check(ranking.policy_loss(*a, **options(c2, "full")), want(c2, "full"))


def test_the_policy_is_its_own_reference():
    c = pb.case(6, 5000, torch.float32, 3)
    c["y"] = c["x"]
    r = ranking.policy_loss(*args(c), **options(c, "full"))
    assert (r.kl == 0).all()


def special(dtype):
    cols = 3000
    c = pb.case(24, cols, dtype, 1, True)
    x, y, ex, given = c["x"], c["y"], c["ex"], c["given"]
    given[0] = -1
    x[0, 5] = math.nan
    ex[1] = True  # nothing left
    x[2] = -math.inf  # nothing left
    given[3] = cols
    given[4] = -2
    given[5] = -(2 ** 31)
    x[6, int(given[6]) - 1] = math.nan
    ex[6, int(given[6]) - 1] = False
    x[7, (int(given[7]) + 1) % cols] = math.inf
    ex[7, (int(given[7]) + 1) % cols] = False
    x[8, 3], ex[8, 3] = math.nan, True  # does not matter
    y[8, 4], ex[8, 4] = math.inf, True
    given[8] = 9
    ex[8, 9] = False
    ex[9, given[9]] = True  # an excluded shown item
    x[10, given[10]] = -math.inf  # one of probability 0
    y[11, (int(given[11]) + 2) % cols] = -math.inf  # q = 0 < p
    ex[11, (int(given[11]) + 2) % cols] = False
    j = (int(given[12]) + 2) % cols  # q = p = 0
    x[12, j] = y[12, j] = -math.inf
    ex[12, j] = False
    y[13, (int(given[13]) + 2) % cols] = math.nan
    ex[13, (int(given[13]) + 2) % cols] = False
    y[14] = -math.inf  # the reference has nothing left
    x[15] = torch.finfo(dtype).min  # the lowest value everywhere: uniform
    ex[15] = False
    y[15] = torch.finfo(dtype).min
    x[16, ::2] = torch.finfo(dtype).min  # and as a mask
    x[16, given[16]] = 0.5
    return c


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["none", "shown", "full"])
@pytest.mark.parametrize("weighted", [False, True])
def test_special_rows(dtype, kind, weighted):
    c = special(TYPES[dtype])
    a, o = args(c), options(c, kind)
    if not weighted:
        o["kl_weight"] = 0.0
    r, grad = ranking.policy_loss_and_grad(*a, c["weight"].cuda(), **o)
    loss, lp, kl, grad = (t.cpu() for t in (*r, grad))
    full, some = kind == "full", kind == "full" and weighted
    assert loss[0] == lp[0] == kl[0] == 0 and (grad[0] == 0).all()
    for i in (1, 2):
        assert loss[i] == kl[i] == 0 and lp[i] == -math.inf and (grad[i] == 0).all()
    for i in (3, 4, 5):
        assert loss[i].isnan() and lp[i].isnan()
        assert grad[i].masked_select(~c["ex"][i]).isnan().all() and (grad[i][c["ex"][i]] == 0).all()
    for i in (6, 7):
        assert loss[i].isnan() and lp[i].isnan()
        assert grad[i].masked_select(~c["ex"][i]).isnan().all() and (grad[i][c["ex"][i]] == 0).all()
    assert torch.isfinite(loss[8]) and torch.isfinite(grad[8]).all()
    for i in (9, 10):  # rho = 0
        bound = (1 - pb.LO) * abs(c["adv"][i].item()) if c["adv"][i] < 0 else 0.0
        assert lp[i] == -math.inf
        if kind != "shown":
            assert abs(loss[i] - bound - o["kl_weight"] * kl[i]) < 1e-6
            if not full:
                assert (grad[i] == 0).all()
        else:
            assert kl[i] == math.inf and (loss[i] == math.inf) == weighted
    for i, nan in ((11, False), (13, True), (14, False)):
        if full:
            assert kl[i].isnan() if nan else kl[i] == math.inf
        assert torch.isfinite(loss[i]) != some
        left = grad[i].masked_select(~c["ex"][i])
        assert not torch.isfinite(left).all() if some else torch.isfinite(left).all()
        assert (grad[i][c["ex"][i]] == 0).all()
    for i in (12, 15, 16):
        assert torch.isfinite(loss[i]) and torch.isfinite(kl[i]) and torch.isfinite(grad[i]).all()
    if full:
        assert abs(kl[15]) < 1e-6  # uniform both
    assert abs(lp[15] + math.log(3000)) < 1e-5
    # The two ways to the gradient agree on all of it: each is within the bounds of
    # policy_bounds.py, with D and E below 30, D1 and E1 below 10, |d - dy| below 30
    # but in rows 14 and 16 (where they are lost in infinities or p = 0): ln p_g to
    # 98 u = 6e-6 (the ratio and the loss, of themselves), kl to (300 + 30 (120 + 78)
    # + 30 * 99 + 2 * 98) u = 5.7e-4, an element of the gradient to
    # |w| / t (|slope| (222 + 98) u + 0.06 (60 (222 + 8) + 2 * 5.7e-4 / u) u).
    leaf = a[0].clone().requires_grad_()
    again = ranking.policy_loss(leaf, *a[1:], **o)
    again.loss.backward(c["weight"].cuda())

    def agree(x, y, tol):
        x, y = x.detach().cpu().double(), y.double()
        assert torch.equal(x.isnan(), y.isnan()) and torch.equal(x.isinf(), y.isinf())
        off = torch.where(torch.isfinite(y), (x - y).abs() - tol, -1.0)
        assert (off <= 0).all(), off.max()

    size = loss.double().abs().nan_to_num(0.0, 0.0, 0.0)
    agree(again.log_prob, lp, 2 * 6e-6 + 2.0 ** -23 * lp.double().abs().nan_to_num(0, 0, 0))
    agree(again.kl, kl, 2 * 5.7e-4 + 2.0 ** -23 * kl.double().abs().nan_to_num(0, 0, 0))
    agree(again.loss, loss, 2 * 6.2e-6 * (size + 1) + 2 * 0.06 * 5.7e-4)
    slope = (size + 0.06 * 30)[:, None]  # of rows whose slope is finite
    row = c["weight"].double().abs()[:, None] / c["t"] * (slope * 320 * pb.U + 0.06 * 2e-3)
    agree(leaf.grad, grad, 2 * row + torch.finfo(grad.dtype).eps * grad.double().abs().nan_to_num(0, 0, 0)
          + 2 * pb.TINY[grad.dtype])


def test_the_rows_that_are_there_do_not_depend_on_the_others():
    c = special(torch.float32)
    a, o = args(c), options(c, "full")
    w = c["weight"].cuda()
    r, grad = ranking.policy_loss_and_grad(*a, w, **o)
    for i in (8, 12, 17, 23):
        oi = {**o, "reference": o["reference"][i:i + 1], "excluded": o["excluded"][i:i + 1]}
        ri, gi = ranking.policy_loss_and_grad(*(t[i:i + 1] for t in a), w[i:i + 1], **oi)
        assert torch.equal(ri.loss, r.loss[i:i + 1]) and torch.equal(gi, grad[i:i + 1])


def test_ratio_at_the_bounds():
    """At the bound itself the gradient passes; past it, it stops on the side that the
    advantage names; without an upper bound it never stops above."""
    x = torch.zeros(6, 4).cuda()
    given = torch.zeros(6, dtype=torch.int32).cuda()
    lp = -math.log(4.0)
    old = torch.tensor([lp, lp - 1.0, lp - 1.0, lp + 1.0, lp + 1.0, lp - 80.0]).cuda()
    adv = torch.tensor([1.0, 1.0, -1.0, 1.0, -1.0, 1.0]).cuda()
    r, g = ranking.policy_loss_and_grad(x, given, adv, old, clip_low=0.0, clip_high=0.0)
    e = math.e
    assert torch.allclose(r.loss.cpu(), torch.tensor([-1.0, -1.0, e, -1 / e, 1.0, -1.0]), rtol=1e-6)
    passes = torch.tensor([g[i].abs().sum() > 0 for i in range(6)])
    assert passes.tolist()[1:] == [False, True, True, False, False]
    r, g = ranking.policy_loss_and_grad(x, given, adv, old, clip_low=1.0, clip_high=math.inf)
    assert torch.allclose(r.loss[:5].cpu(), torch.tensor([-1.0, -e, e, -1 / e, 1 / e]), rtol=1e-6)
    assert (g.abs().sum(1) > 0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_strides_in_place_and_outputs(dtype):
    c = pb.case(9, 777, TYPES[dtype], 2, True)
    a, o = args(c), options(c, "full")
    w = c["weight"].cuda()
    r0, g0 = ranking.policy_loss_and_grad(*a, w, **o)

    def apart(t, before, after):
        wide = torch.full((9, 777 + before + after), 1, dtype=t.dtype, device="cuda")
        wide[:, before:before + 777] = t
        return wide[:, before:before + 777]

    x = apart(a[0], 3, 5)
    o2 = {**o, "reference": apart(o["reference"], 1, 0), "excluded": apart(o["excluded"], 2, 7)}
    r, g = ranking.policy_loss_and_grad(x, *a[1:], w, **o2)
    assert torch.equal(g, g0) and torch.equal(r.loss, r0.loss)
    for target in (x, o2["reference"]):  # in place of the scores, then of the reference
        keep = target.clone()
        r, g = ranking.policy_loss_and_grad(x, *a[1:], w, out=target, **o2)
        assert g.data_ptr() == target.data_ptr() and torch.equal(target, g0)
        assert torch.equal(r.loss, r0.loss)
        target.copy_(keep)
    out = apart(torch.zeros(9, 777, dtype=TYPES[dtype], device="cuda"), 4, 4)
    ranking.policy_loss_and_grad(x, *a[1:], w, out=out, **o2)
    assert torch.equal(out, g0)
    base = out._base
    assert (base[:, :4] == 1).all() and (base[:, 781:] == 1).all()
    # the same row many times over
    one = {**o, "reference": o["reference"][:1].expand(9, 777),
           "excluded": o["excluded"][:1].expand(9, 777)}
    r, g = ranking.policy_loss_and_grad(a[0][:1].expand(9, 777), *a[1:], w, **one)
    same = {**one, "reference": one["reference"].contiguous(), "excluded": one["excluded"].contiguous()}
    r1, g1 = ranking.policy_loss_and_grad(a[0][:1].expand(9, 777).contiguous(), *a[1:], w, **same)
    assert torch.equal(g, g1) and torch.equal(r.loss, r1.loss)


def test_empty_calls():
    for rows, cols in ((0, 5), (0, 0)):
        z = torch.zeros(rows, device="cuda")
        r, g = ranking.policy_loss_and_grad(torch.zeros(rows, cols, device="cuda"), z.int(), z, z)
        assert r.loss.shape == (rows,) and g.shape == (rows, cols)
    z = torch.zeros(3, device="cuda")
    given = torch.tensor([-1, 0, -1]).int().cuda()
    r, g = ranking.policy_loss_and_grad(torch.zeros(3, 0, device="cuda"), given, z, z)
    assert r.loss[0] == r.loss[2] == 0 and g.shape == (3, 0)


def test_more_rows_than_workgroups():
    rows, cols = (1 << 20) + 50_007, 5
    g = torch.Generator(device="cuda").manual_seed(1)
    line = 2 * torch.randn(rows + cols, generator=g, device="cuda")
    x = line.as_strided((rows, cols), (1, 1))
    given = torch.arange(rows, device="cuda", dtype=torch.int32) % cols
    adv = torch.randn(rows, generator=g, device="cuda")
    lp = torch.log_softmax(x.double(), 1).gather(1, given.long()[:, None])[:, 0]
    old = (lp - 0.1).float()  # rho = 1.105: within the bounds
    r, got = ranking.policy_loss_and_grad(x, given, adv, old)
    rho = (lp - old.double()).exp()
    assert ((r.loss + rho * adv).abs() <= 2e-5 * adv.abs() + 1e-30).all()
    p = torch.softmax(x.double(), 1)
    own = torch.nn.functional.one_hot(given.long(), cols)
    expected = -(rho * adv)[:, None] * (own - p)
    # e_lp + r_j with D below 20: (80 + 58 + 80 + 80 + 62 + 10) 2^-24 = 2.3e-5
    assert ((got - expected).abs() <= 2.3e-5 * (rho * adv).abs()[:, None] * (own + p) + 1e-30).all()


def test_rows_past_32_bits_of_elements():
    rows, cols = 3, (1 << 30) + 5
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[2, cols - 1] = 20.0
    given = torch.tensor([0, cols - 1, cols - 1]).int().cuda()
    z, one = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    r, g = ranking.policy_loss_and_grad(x, given, one, z - 20.0, reference=x, kl_weight=0.5)
    lp = torch.tensor([-math.log(cols)] * 2 + [20.0 - math.log(cols - 1 + math.exp(20.0))])
    assert torch.allclose(r.log_prob.cpu(), lp, atol=1e-4)
    assert g[1, cols - 1] != 0 and (g[0, 1:5] == g[1, 1:5]).all() and (r.kl.abs() < 1e-6).all()


# --- graphs, streams, autograd ---------------------------------------------------

def test_captured_forward_and_backward():
    c = pb.case(20, 4000, torch.float32, 1, True)
    a, o, w = args(c), options(c, "full"), c["weight"].cuda()
    ranking.policy_loss_and_grad(*a, w, **o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, g = ranking.policy_loss_and_grad(*a, w, **o)
    for seed in range(4):
        a[0].copy_(pb.case(20, 4000, torch.float32, 5 + seed)["x"])
        graph.replay()
        r1, g1 = ranking.policy_loss_and_grad(*a, w, **o)
        assert torch.equal(r.loss, r1.loss) and torch.equal(g, g1)
        torch.cuda.synchronize()


def test_captured_autograd():
    c = pb.case(6, 70_000, torch.float32, 1)
    a, o, w = args(c), options(c, "full"), c["weight"].cuda()
    leaf = a[0].clone().requires_grad_()

    def step():
        r = ranking.policy_loss(leaf, *a[1:], **o)
        return r.loss, torch.autograd.grad(r.loss, leaf, w)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, g = step()
    for seed in range(4):
        with torch.no_grad():
            leaf.copy_(pb.case(6, 70_000, torch.float32, 5 + seed)["x"])
        graph.replay()
        loss1, g1 = ranking.policy_loss_and_grad(leaf.detach(), *a[1:], w, **o)
        assert torch.allclose(loss, loss1.loss, rtol=1e-5, atol=1e-6)
        torch.cuda.synchronize()
        l2, g2 = step()
        assert torch.equal(loss, l2) and torch.equal(g, g2)


def test_on_two_streams_at_once():
    c = pb.case(40, 30_000, torch.bfloat16, 1, True)
    a, o, w = args(c), options(c, "full"), c["weight"].cuda()
    r0, g0 = ranking.policy_loss_and_grad(*a, w, **o)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(ranking.policy_loss_and_grad(*a, w, **o))
    for s in streams:
        s.synchronize()
    assert all(torch.equal(r.loss, r0.loss) and torch.equal(g, g0) for r, g in got)


def test_only_the_scores_and_the_loss_have_a_derivative():
    c = pb.case(4, 50, torch.float32, 1)
    a, o = args(c), options(c, "full")
    x = a[0].requires_grad_()
    r = ranking.policy_loss(x, *a[1:], **o)
    assert r.loss.requires_grad and not r.kl.requires_grad and not r.log_prob.requires_grad
    for name in ("reference",):
        with pytest.raises(ValueError, match="requires grad"):
            ranking.policy_loss(x, *a[1:], **{**o, name: o[name].clone().requires_grad_()})
    with pytest.raises(ValueError, match="requires grad"):
        ranking.policy_loss(x, a[1], a[2].clone().requires_grad_(), a[3], **o)
    (g,) = torch.autograd.grad(r.loss.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="no derivative"):
        g.sum().backward()


def test_backward_after_the_scores_were_overwritten_raises():
    c = pb.case(4, 50, torch.float32, 1)
    a, o = args(c), options(c, "full")
    x = a[0].requires_grad_() * 1
    r = ranking.policy_loss(x, *a[1:], **o)
    with torch.no_grad():
        ranking.policy_loss_and_grad(x, *a[1:], out=x, **o)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        r.loss.sum().backward()


def test_gradients_as_autograd_may_pass_them():
    c = pb.case(4, 50, torch.float32, 1)
    a, o = args(c), options(c, "full")
    x = a[0].requires_grad_()
    r = ranking.policy_loss(x, *a[1:], **o)
    want = torch.autograd.grad(r.loss, x, torch.ones(4, device="cuda"), retain_graph=True)[0]
    for g in (torch.ones(1, device="cuda").expand(4), torch._neg_view(-torch.ones(4).cuda()),
              torch.ones(8, device="cuda")[::2]):
        assert torch.equal(torch.autograd.grad(r.loss, x, g, retain_graph=True)[0], want)


def test_gradients_without_memory_or_with_a_tangent():
    c = pb.case(4, 50, torch.float32, 1)
    a, o = args(c), options(c, "full")
    x = a[0].requires_grad_()
    r = ranking.policy_loss(x, *a[1:], **o)
    zeros = torch._efficientzerotensor((4,), device="cuda")
    (got,) = torch.autograd.grad(r.loss, x, zeros, retain_graph=True)
    assert torch.equal(got, torch.zeros(4, 50, device="cuda"))
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(torch.ones(4, device="cuda"), torch.ones(4, device="cuda"))
        with pytest.raises(RuntimeError, match="tangent"):
            torch.autograd.grad(r.loss, x, dual, retain_graph=True)
    with pytest.raises(RuntimeError, match="memory"):
        torch.autograd.grad(r.loss, x, torch.eye(4, device="cuda"), is_grads_batched=True)


@pytest.mark.parametrize("change", [torch.Tensor.half, torch.Tensor.cpu, lambda t: t[:1]])
def test_saved_tensors_that_a_hook_changes_are_refused(change):
    c = pb.case(4, 50, torch.float32, 1)
    a, o = args(c), options(c, "full")
    x = a[0].requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(change, lambda t: t):
        r = ranking.policy_loss(x, *a[1:], **o)
    with pytest.raises(RuntimeError, match="came back changed"):
        r.loss.sum().backward()
    with torch.autograd.graph.save_on_cpu():
        r = ranking.policy_loss(x, *a[1:], **o)
    (got,) = torch.autograd.grad(r.loss.sum(), x)
    assert torch.equal(got, torch.autograd.grad(ranking.policy_loss(x, *a[1:], **o).loss.sum(), x)[0])


def test_refusals_on_the_gpu():
    c = pb.case(4, 50, torch.float32, 1)
    a, o = args(c), options(c, "full")
    x, given, adv, old = a
    call = ranking.policy_loss
    for f in (lambda: call(x.t(), given, adv, old), lambda: call(x, given.long(), adv, old),
              lambda: call(x, None, adv, old), lambda: call(x, given, adv[:3], old),
              lambda: call(x, given, adv, old.double()), lambda: call(x, given, adv.cpu(), old),
              lambda: call(x, given, adv, old, reference=x.bfloat16()),
              lambda: call(x, given, adv, old, reference=x[:, :40]),
              lambda: call(x, given, adv, old, reference=x, reference_log_prob=old),
              lambda: call(x, given, adv, old, excluded=x),
              lambda: call(x, given, adv, old, kl_weight="much"),
              lambda: ranking.policy_loss_and_grad(x, given, adv, old, adv[:2]),
              lambda: ranking.policy_loss_and_grad(x, given, adv, old, out=x[:3])):
        with pytest.raises(ValueError):
            f()
    for change in (dict(temperature=0.0), dict(temperature=math.nan), dict(clip_low=-0.1),
                   dict(clip_low=1.1), dict(clip_high=-0.1), dict(clip_high=math.nan),
                   dict(kl_weight=math.inf)):
        with pytest.raises(bgmf.BgmfError):
            call(x, given, adv, old, **change)
    flat = torch.zeros(500, device="cuda")
    with pytest.raises(bgmf.BgmfError, match="shares memory"):
        ranking.policy_loss_and_grad(flat[:200].view(4, 50), given, adv, old,
                                     out=flat[100:300].view(4, 50))
    with pytest.raises(bgmf.BgmfError, match="shares memory"):
        ranking.policy_loss_and_grad(x, given, flat[:4], old, out=flat[:200].view(4, 50))
