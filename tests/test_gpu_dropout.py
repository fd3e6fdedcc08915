"""Dropout: bits equal to the generator's, the gradient by the same words."""
import numpy as np
import pytest

from paper_2304_13724_amd import bgmf, ranking

import torch
from torch.autograd import forward_ad

from philox import words

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def want(x, p, seed, offset):
    """The definition: the factor and the product in fp32, then the type."""
    w = torch.from_numpy(words(seed, offset, x.numel()).astype(np.int64)).view(x.shape)
    kept = (w >= int(p * 2.0 ** 32)) if p < 1 else torch.zeros_like(w, dtype=torch.bool)
    factor = np.float32(1.0 / (1.0 - p)) if p < 1 else np.float32(0)
    y = (x.float() * float(factor)).to(x.dtype)
    return torch.where(kept, y, torch.zeros_like(y))


def draw(shape, dtype, seed=1):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(1,), (2,), (3,), (5,), (7,), (8,), (9,), (1, 64), (13, 17),
                                   (3, 5, 7), (257, 129), (1000, 1001), ()])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(dtype, shape, p):
    x = draw(shape, TYPES[dtype])
    for seed, offset in ((0, 0), (2 ** 64 - 1, 12345), (7, 2 ** 64 - 2), (1 << 40, 2 ** 32 - 3)):
        got = ranking.dropout(x.cuda(), p, seed, offset)
        assert torch.equal(got.cpu(), want(x, p, seed, offset)) and got.shape == x.shape


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,pitch", [(5, 3, 7), (9, 64, 80), (17, 33, 100), (300, 129, 131),
                                             (4, 1, 5)])
def test_rows_apart_have_the_same_mask(dtype, rows, cols, pitch):
    wide = draw((rows, pitch), TYPES[dtype])
    x, on = wide[:, 2:2 + cols], wide.cuda()[:, 2:2 + cols]
    expected = want(x.contiguous(), 0.3, 5, 9)
    assert torch.equal(ranking.dropout(on, 0.3, 5, 9).cpu(), expected)
    # into rows apart, and in place
    out = torch.full_like(wide, 3.0).cuda()
    ranking.dropout(x.contiguous().cuda(), 0.3, 5, 9, out=out[:, 1:1 + cols])
    assert torch.equal(out[:, 1:1 + cols].cpu(), expected)
    assert (out[:, 0] == 3).all() and (out[:, 1 + cols:] == 3).all()
    assert ranking.dropout(on, 0.3, 5, 9, out=on) is not None
    assert torch.equal(on.cpu(), expected)


def test_broadcast_rows_and_empty_tensors():
    x = draw((1, 45), torch.float32)
    got = ranking.dropout(x.cuda().expand(6, 45), 0.5, 3)
    assert torch.equal(got.cpu(), want(x.expand(6, 45).contiguous(), 0.5, 3, 0))
    assert ranking.dropout(x[:0].cuda(), 0.5, 3).shape == (0, 45)
    assert ranking.dropout(torch.empty(3, 0, device="cuda"), 0.5, 3).shape == (3, 0)


def test_what_is_dropped_is_zero_whatever_it_was():
    x = torch.full((4096,), float("nan"), device="cuda")
    y = ranking.dropout(x, 0.5, 1)
    kept = torch.from_numpy(words(1, 0, 4096) >= 2 ** 31).cuda()
    assert (y[~kept] == 0).all() and y[kept].isnan().all()


def test_share_of_kept_elements():
    """Of n = 2^24 elements a share 1 - p is kept: within 6 of its standard deviations."""
    n = 1 << 24
    x = torch.ones(n, device="cuda")
    for p in (0.1, 0.5, 0.9):
        kept = (ranking.dropout(x, p, 11, 1 << 50) > 0).double().mean().item()
        assert abs(kept - (1 - p)) < 6 * (p * (1 - p) / n) ** 0.5


def test_calls_that_are_apart_continue_one_stream():
    x = torch.ones(4000, device="cuda")
    whole = ranking.dropout(x, 0.5, 9, 100)
    parts = [ranking.dropout(x[i:i + 1000], 0.5, 9, 100 + i // 4) for i in range(0, 4000, 1000)]
    assert torch.equal(torch.cat(parts), whole)


def test_past_two_to_the_32_elements():
    n = (1 << 32) + 5000
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = ranking.dropout(x, 0.5, 3, 7, out=x)
    at = (1 << 32) - 8
    assert torch.equal(y[at:].cpu(), want(torch.ones(n - at, dtype=torch.bfloat16), 0.5, 3,
                                          7 + at // 4))


# --- the gradient ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradient(dtype):
    x = draw((33, 50), TYPES[dtype]).cuda().requires_grad_()
    y = ranking.dropout(x, 0.25, 4, 8)
    g = draw((33, 50), TYPES[dtype], 2)
    (got,) = torch.autograd.grad(y, x, g.cuda())
    assert torch.equal(y.detach().cpu(), want(x.detach().cpu(), 0.25, 4, 8))
    assert torch.equal(got.cpu(), want(g, 0.25, 4, 8))


def test_gradient_by_differences_and_twice():
    """The call is linear: differences are exact but for roundings of values near 1."""
    x = draw((8, 9), torch.float32).cuda().requires_grad_()
    a = draw((8, 9), torch.float32, 2).cuda().requires_grad_()
    y = ranking.dropout(x, 0.5, 4)
    (g,) = torch.autograd.grad(y, x, a, create_graph=True)
    step = torch.zeros_like(x)
    step[3, 4] = 2.0 ** -8
    more = ranking.dropout(x.detach() + step, 0.5, 4) - ranking.dropout(x.detach() - step, 0.5, 4)
    quotient = (more / 2.0 ** -7 * a.detach()).sum()
    assert abs(quotient - g[3, 4]) <= 2.0 ** -14  # values below 8: steps of 2^-21 over 2^-7
    (gg,) = torch.autograd.grad(g.sum(), a)  # the gradient's own gradient
    assert torch.equal(gg, ranking.dropout(torch.ones_like(a), 0.5, 4))


def test_gradients_as_autograd_may_pass_them():
    x = draw((6, 7), torch.float32).cuda().requires_grad_()
    y = ranking.dropout(x, 0.5, 4)
    for g in (torch.ones(1, 1, device="cuda").expand(6, 7), torch._neg_view(-torch.ones(6, 7).cuda()),
              torch.ones(7, 6, device="cuda").t()):
        (got,) = torch.autograd.grad(y, x, g, retain_graph=True)
        assert torch.equal(got, ranking.dropout(torch.ones(6, 7, device="cuda"), 0.5, 4))


def test_gradients_without_memory_or_with_a_tangent():
    x = draw((6, 7), torch.float32).cuda().requires_grad_()
    y = ranking.dropout(x, 0.5, 4)
    zeros = torch._efficientzerotensor((6, 7), device="cuda")
    assert torch.autograd.grad(y, x, zeros, retain_graph=True)[0].eq(0).all()
    ones = torch.ones(6, 7, device="cuda")
    with forward_ad.dual_level():
        with pytest.raises(RuntimeError, match="tangent"):
            torch.autograd.grad(y, x, forward_ad.make_dual(ones, ones), retain_graph=True)
    with pytest.raises(RuntimeError, match="memory"):
        torch.autograd.grad(y, x, torch.ones(2, 6, 7, device="cuda"), is_grads_batched=True)


def test_an_offset_that_a_hook_changes_is_refused():
    x = draw((6, 7), torch.float32).cuda().requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(torch.Tensor.int, lambda t: t):
        y = ranking.dropout(x, 0.5, 4, torch.tensor([3]).cuda())
    with pytest.raises(RuntimeError, match="came back changed"):
        y.sum().backward()


def test_no_graph_with_an_output():
    x = torch.ones(5, device="cuda", requires_grad=True)
    with pytest.raises(ValueError, match="out"):
        ranking.dropout(x, 0.5, 1, out=torch.empty(5, device="cuda"))
    with torch.no_grad():
        before = x._version
        ranking.dropout(x, 0.5, 1, out=x)
        assert x._version == before + 1


# --- an offset on the device -----------------------------------------------------

def test_offset_on_the_device_in_a_captured_graph():
    x = draw((100, 64), torch.float32).cuda()
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    ranking.dropout(x, 0.5, 3, offset)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ranking.dropout(x, 0.5, 3, offset)
        offset += 1600
    for i in range(4):
        graph.replay()
        assert torch.equal(y, ranking.dropout(x, 0.5, 3, 1600 * i))
        torch.cuda.synchronize()
    offset.fill_(-1)  # 2^64 - 1
    assert torch.equal(ranking.dropout(x, 0.5, 3, offset), ranking.dropout(x, 0.5, 3, 2 ** 64 - 1))


def test_an_offset_that_changed_before_the_backward_pass_raises():
    x = torch.ones(64, device="cuda", requires_grad=True)
    offset = torch.zeros((), dtype=torch.int64, device="cuda")
    y = ranking.dropout(x, 0.5, 3, offset)
    offset += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y = ranking.dropout(x, 0.5, 3, offset)
    y.sum().backward()
    assert torch.equal(x.grad, ranking.dropout(torch.ones(64, device="cuda"), 0.5, 3, 1))


def test_refusals_on_the_gpu():
    x = torch.ones(6, 8, device="cuda")
    at = torch.zeros(2, dtype=torch.int64, device="cuda")
    for call in (lambda: ranking.dropout(x.t(), 0.5, 1), lambda: ranking.dropout(x.double(), 0.5, 1),
                 lambda: ranking.dropout(x, 0.5, -1), lambda: ranking.dropout(x, 0.5, 1 << 64),
                 lambda: ranking.dropout(x, 0.5, 1.5), lambda: ranking.dropout(x, 0.5, 1, at),
                 lambda: ranking.dropout(x, 0.5, 1, at[:1].int()),
                 lambda: ranking.dropout(x, 0.5, 1, at[:1].cpu()),
                 lambda: ranking.dropout(x, None, 1), lambda: ranking.dropout(x, 0.5, 1, None),
                 lambda: ranking.dropout(x, 0.5, 1, out=x[:5]),
                 lambda: ranking.dropout(x.view(2, 3, 8).transpose(0, 1), 0.5, 1)):
        with pytest.raises(ValueError):
            call()
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(bgmf.BgmfError, match="p must be"):
            ranking.dropout(x, p, 1)
    flat = torch.ones(100, device="cuda")
    with pytest.raises(bgmf.BgmfError, match="shares memory"):
        ranking.dropout(flat[:50], 0.5, 1, out=flat[10:60])
