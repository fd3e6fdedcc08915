"""The gradient's formulas against differences, and what the bounds of the GPU
tests can tell apart: mistakes planted in the formulas' results."""
import pytest

import ranking_bounds as rb

import torch


@pytest.mark.parametrize("mode", range(4))
def test_gradient_against_differences(mode):
    x, given, t, excluded, gl, gh = rb.case(3, 23, torch.float64, mode)
    gl, gh = (None if g is None else g.double() for g in (gl, gh))

    def loss(v):
        z = (v if excluded is None else v.masked_fill(excluded, -float("inf"))) / t
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        total = torch.zeros((), dtype=torch.float64)
        if gl is not None:
            at = lp[torch.arange(3), given.clamp_min(0)]
            total += (gl * torch.where(given >= 0, at, 0.0)).sum()
        if gh is not None:
            total -= (gh * torch.where(p > 0, p * lp, 0.0).sum(1)).sum()
        return total.item()

    grad, _ = rb.terms(x, given, t, excluded, gl, gh)
    for i in range(3):
        for j in range(23):
            up, down = x.clone(), x.clone()
            up[i, j] += 1e-5
            down[i, j] -= 1e-5
            assert abs(grad[i, j].item() - (loss(up) - loss(down)) / 2e-5) < 1e-8


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", range(4))
@pytest.mark.parametrize("rows,cols", [s for s in rb.SHAPES if s[1] > 200])
def test_what_the_bounds_tell_apart(rows, cols, mode, dtype):
    x, given, t, excluded, gl, gh = rb.case(rows, cols, dtype, mode)
    given[given < 0] = 5  # (a row without a given item has nothing to lose in mode 0 and 3)
    if excluded is not None:
        excluded[:, 5] = False
    a = [None if g is None else g.double() for g in (gl, gh)]
    grad, tol = rb.bounds(x.double(), given, t, excluded, *a, dtype)
    kept = torch.ones_like(grad, dtype=torch.bool) if excluded is None else ~excluded
    # an element that was not written, or is a neighbour's
    assert (grad.abs() > tol)[kept].double().mean() > 0.999
    assert ((grad - grad.roll(1, 1)).abs() > tol)[kept].double().mean() > 0.95
    if excluded is not None:
        assert (tol[excluded] == 0).all()
    # a lost term
    if gh is not None and gl is not None:
        for lost in ([a[0], None], [None, a[1]]):
            other, _ = rb.terms(x.double(), given, t, excluded, *lost)
            assert ((grad - other).abs() > tol)[kept].double().mean() > 0.9
