"""An output of the caller's that is part of a graph: the call would leave its history
behind, and a backward pass through it would give gradients of what it no longer holds."""
import pytest

from paper_2304_13724_amd import ranking

import torch

pytestmark = pytest.mark.gpu


def calls():
    """name -> (shape of out, call)"""
    x = torch.randn(4, 64, generator=torch.Generator().manual_seed(1)).cuda()
    q, s = ranking.quantize_rows_mx4(x)
    b, scale = ranking.quantize_rows(x)
    z, given = torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    r = ranking.log_probs(x, given)
    return {
        "dropout": ((4, 64), lambda out: ranking.dropout(x, 0.5, 1, out=out)),
        "dequantize_rows_mx4": ((4, 64), lambda out: ranking.dequantize_rows_mx4(q, s, out=out)),
        "mx4_scores": ((4, 4), lambda out: ranking.mx4_scores(x, q, s, out=out)),
        "quantized_scores": ((4, 4), lambda out: ranking.quantized_scores(x, b, scale, out=out)),
        "log_probs_backward": ((4, 64), lambda out: ranking.log_probs_backward(
            x, given, r.row_max, r.row_sum, r.entropy, z + 1, out=out)),
        "policy_loss_and_grad": ((4, 64), lambda out: ranking.policy_loss_and_grad(
            x, given, z + 1, z, out=out)[1])}


@pytest.mark.parametrize("name", ["dropout", "dequantize_rows_mx4", "mx4_scores",
                                  "quantized_scores", "log_probs_backward",
                                  "policy_loss_and_grad"])
def test_outputs_in_a_graph_are_refused(name):
    shape, call = calls()[name]
    want = call(torch.empty(shape, device="cuda")).clone()
    leaf = torch.ones(shape, device="cuda", requires_grad=True)
    node = leaf * 2
    for out in (leaf, node):
        with pytest.raises(ValueError, match="out takes no part in a graph"):
            call(out)
    assert (leaf == 1).all() and (node == 2).all()
    with torch.no_grad():
        assert torch.equal(call(leaf), want) and leaf._version == 1


def test_the_policys_gradient_in_place_of_its_scores():
    """The one output that may be in a graph: the scores, whose history the gradient
    then goes through."""
    u = torch.randn(4, 8, generator=torch.Generator().manual_seed(1)).cuda().requires_grad_()
    v = torch.randn(50, 8, generator=torch.Generator().manual_seed(2)).cuda()
    z, given = torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    scores = u @ v.t()
    want = ranking.policy_loss_and_grad(scores, given, z + 1, z - 4)[1]
    _, grad = ranking.policy_loss_and_grad(scores, given, z + 1, z - 4, out=scores)
    assert grad.data_ptr() == scores.data_ptr() and torch.equal(grad, want)
    scores.backward(grad.detach())
    assert torch.equal(u.grad, want @ v)
