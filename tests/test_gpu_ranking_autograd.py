"""The ranking calls behave beside autograd as PyTorch's own functions do: writes
into tensors of the caller's are seen by earlier graphs, and no derivative is
dropped silently."""
import pytest

from paper_2304_13724_amd import ranking

import torch
import torch.autograd.forward_ad as forward_ad

pytestmark = pytest.mark.gpu


def scores(rows=4, cols=50):
    g = torch.Generator().manual_seed(rows + cols)
    return torch.randn(rows, cols, generator=g).cuda()


GIVEN = [1, 2, 3, -1]


# --- writes into the caller's tensors -------------------------------------------

def test_backward_after_the_scores_were_overwritten_raises():
    leaf = scores().requires_grad_()
    x = leaf * 1  # not a leaf: what a model computes
    given = torch.tensor(GIVEN).int().cuda()
    r = ranking.log_probs(x, given)
    with torch.no_grad():
        ranking.log_probs_backward(x, given, r.row_max, r.row_sum, None, torch.ones(4).cuda(), out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        r.log_prob.sum().backward()


def test_written_tensors_have_a_new_version():
    x = scores()
    given = torch.tensor(GIVEN).int().cuda()
    r = ranking.log_probs(x, given)
    gl = torch.ones(4).cuda()
    before = [t._version for t in (x, given, r.row_max, r.row_sum, gl)]
    out = torch.empty_like(x)
    ranking.log_probs_backward(x, given, r.row_max, r.row_sum, None, gl, out=out)
    assert out._version == 1
    assert [t._version for t in (x, given, r.row_max, r.row_sum, gl)] == before

    c = ranking.Catalogue(torch.ones(5, 50).cuda())
    to = torch.empty(4, 5).cuda()
    ranking.quantized_scores(x, c.items, c.scale, out=to)
    assert (to._version, x._version, c.items._version) == (1, before[0], 0)

    bucket = torch.ones(12).cuda()
    grads = list(bucket.split([5, 7]))
    ranking.clip_grad_norm(grads, 1.0)
    assert bucket._version == 2  # one write for each view
    clipped = [torch.empty_like(t) for t in grads]
    ranking.clip_grad_norm(grads, 1.0, out=clipped)
    assert bucket._version == 2 and [t._version for t in clipped] == [1, 1]


def test_tensors_of_inference_mode_can_be_written():
    """They have no version, and no graph can hold them."""
    with torch.inference_mode():
        g = torch.full((9,), 2.0, device="cuda")
    ranking.clip_grad_norm([g], 1.0)
    assert torch.allclose(g, torch.full((9,), 1 / 3, device="cuda"))
    with torch.inference_mode():
        ranking.clip_grad_norm([g], 0.5)
        assert torch.allclose(g, torch.full((9,), 1 / 6, device="cuda"))


# --- forward mode ----------------------------------------------------------------

@pytest.mark.parametrize("needs_grad", [False, True])
def test_a_tangent_is_refused(needs_grad):
    x = scores().requires_grad_(needs_grad)
    given = torch.tensor(GIVEN).int().cuda()
    with forward_ad.dual_level():
        with pytest.raises((ValueError, RuntimeError), match="tangent|jvp"):
            ranking.log_probs(forward_ad.make_dual(x, torch.ones_like(x)), given)
        assert torch.isfinite(ranking.log_probs(x, given).log_prob).all()


# --- gradients as autograd may pass them -----------------------------------------

def test_gradients_that_negate_their_memory_or_are_broadcast():
    given = torch.tensor(GIVEN).int().cuda()
    got = []
    for g in (torch._neg_view(torch.ones(4).cuda()), torch.full((1,), -1.0).cuda().expand(4),
              -torch.ones(4).cuda()):
        leaf = scores().requires_grad_()
        r = ranking.log_probs(leaf, given)
        torch.autograd.backward([r.log_prob, r.entropy], [g, g])
        got.append(leaf.grad)
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[2])


# --- results without a derivative -----------------------------------------------

def test_scores_in_8_bit_integers_have_no_derivative_and_say_so():
    users, items = scores(3, 64).requires_grad_(), scores(7, 64)
    c = ranking.Catalogue(items)
    s = c.scores(users)
    want = c.scores(users.detach())
    assert s.requires_grad and not want.requires_grad and torch.equal(s.detach(), want)
    with pytest.raises(RuntimeError, match="derivative"):
        s.sum().backward()
    r = c.rank(users, torch.tensor([1, 2, 3]).int().cuda(), top=2)
    with pytest.raises(RuntimeError, match="derivative"):
        r.log_prob.sum().backward()
    # the scales: of the items, and of users' rows
    q, a = ranking.quantize_rows(users)
    assert a.requires_grad and not q.requires_grad
    with pytest.raises(RuntimeError, match="derivative"):
        a.sum().backward()
    with pytest.raises(RuntimeError, match="derivative"):
        ranking.quantized_scores(q, c.items, c.scale, a).sum().backward()
    learned = ranking.Catalogue(items.clone().requires_grad_())
    with pytest.raises(RuntimeError, match="derivative"):
        learned.scores(users.detach()).sum().backward()
    with torch.no_grad():
        assert not c.scores(users).requires_grad and not c.rank(users).log_prob.requires_grad
        assert not ranking.quantize_rows(users)[1].requires_grad


def test_given_outputs_take_no_part_in_a_graph():
    users, items = scores(3, 64).requires_grad_(), scores(7, 64)
    c = ranking.Catalogue(items)
    to = torch.empty(3, 7, device="cuda")
    with pytest.raises(ValueError, match="out"):
        ranking.quantized_scores(users, c.items, c.scale, out=to)
    with torch.no_grad():
        ranking.quantized_scores(users, c.items, c.scale, out=to)
    assert torch.equal(to, c.scores(users.detach()))


def test_the_backward_call_has_no_derivative_and_says_so():
    x = scores().requires_grad_()
    given = torch.tensor(GIVEN).int().cuda()
    r = ranking.log_probs(x.detach(), given)
    gl = torch.ones(4).cuda()
    d = ranking.log_probs_backward(x, given, r.row_max, r.row_sum, None, gl)
    want = ranking.log_probs_backward(x.detach(), given, r.row_max, r.row_sum, None, gl)
    assert torch.equal(d.detach(), want) and not want.requires_grad
    with pytest.raises(RuntimeError, match="derivative"):
        d.sum().backward()
    with pytest.raises(RuntimeError, match="derivative"):
        ranking.log_probs_backward(x.detach(), given, r.row_max, r.row_sum, None,
                                   gl.clone().requires_grad_()).sum().backward()
    with pytest.raises(ValueError, match="out"):
        ranking.log_probs_backward(x, given, r.row_max, r.row_sum, None, gl,
                                   out=torch.empty_like(want))


# --- memory ----------------------------------------------------------------------

def test_out_of_memory_is_pytorchs_error():
    """4 TiB of scores, and half a TiB of alternatives: refused by the allocator."""
    one = torch.ones(1, 1, device="cuda")
    rows = one.expand(1 << 20, 1)
    with pytest.raises(torch.OutOfMemoryError):
        ranking.quantized_scores(rows, one.to(torch.int8).expand(1 << 20, 1),
                                 torch.ones(1 << 20, device="cuda"))
    with pytest.raises(torch.OutOfMemoryError):
        ranking.log_probs(one.expand(1 << 30, 1), top=128)
    r = ranking.log_probs(torch.zeros(2, 3, device="cuda"), top=1)  # and calls go on
    assert r.top_item.tolist() == [[0], [0]]
