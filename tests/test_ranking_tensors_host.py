"""Tensors that the ranking calls refuse before anything else is looked at, so
on the CPU too."""
import pytest

from paper_2304_13724_amd import ranking

import torch
import torch.autograd.forward_ad as forward_ad

F = torch.zeros(3, 5)
B = torch.zeros(4, 5, dtype=torch.int8)
G = torch.zeros(3, dtype=torch.int32)
Z, Z4 = torch.zeros(3), torch.zeros(4)


def calls(change):
    """Every call with one of its float tensors changed."""
    yield lambda: ranking.log_probs(change(F), G)
    yield lambda: ranking.log_probs_backward(change(F), G, Z, Z, Z, Z, Z)
    yield lambda: ranking.quantize_rows(change(F))
    yield lambda: ranking.quantized_scores(change(F), B, Z4)
    yield lambda: ranking.clip_grad_norm([change(F)], 1.0)


def test_a_tangent_is_refused():
    """Forward-mode derivatives are not computed, and not dropped."""
    with forward_ad.dual_level():
        for call in calls(lambda t: forward_ad.make_dual(t, torch.ones_like(t))):
            with pytest.raises(ValueError, match="tangent"):
                call()


def test_tensors_whose_memory_is_not_their_values_are_refused():
    """A view that negates its memory (the imaginary part of a conjugated
    tensor), and a tensor of zeros without memory."""
    for change in (torch._neg_view, lambda t: torch._efficientzerotensor(t.shape),
                   lambda t: torch.zeros(*t.shape, dtype=torch.complex64).conj().imag):
        for call in calls(change):
            with pytest.raises(ValueError, match="memory"):
                call()
