"""Gradients of log_probs in 64 bits, and how far an element computed in 32 bits
may be from them, relative to the element's own terms.

With u = 2^-24 (one rounding), D_j = (max x - x_j) / t, p_j the probabilities,
D1 and D2 the means of D and D^2 under p:

  exp(-D_j)    the argument is rounded four times (difference, log2 e, division
               by t, product): 4 D_j u; the exponential is good to 2 u
  S            every term has that error, is rescaled to a larger maximum some
               20 times at most (2 u each, and the D's add up), and is summed with
               15 others in 32 bits before 64-bit sums: (4 D1 + 58) u of itself
  p_j          exp(-D_j) times the rounded 1 / S: r_j = (4 D_j + 4 D1 + 62) u
  H            ln S and the mean of D, whose terms have the errors of S and of D
               itself: (4 D2 + 4 D1^2 + 129 D1 + 58 + 3 ln S + H) u
  ln p_j + H   5 D_j u, the error of H, and roundings of ln S and of itself
"""
import math

import torch

U = 2.0 ** -24
HALF_STEP = {d: torch.finfo(d).eps / 2 for d in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def terms(x, given, t, excluded, gl, gh):
    """(gradient, its error before the last rounding), float64; x float64, gl
    and gh float64 or None."""
    v = x if excluded is None else x.masked_fill(excluded, -math.inf)
    top = v.amax(1, keepdim=True)
    some = top > -math.inf
    D = torch.where(v > -math.inf, (torch.where(some, top, 0.0) - v) / t, 0.0)
    e = torch.where(v > -math.inf, torch.exp(-D), 0.0)
    S = e.sum(1, keepdim=True)
    p = torch.where(some, e / S, 0.0)
    D1, D2 = (p * D).sum(1, keepdim=True), (p * D * D).sum(1, keepdim=True)
    lnS = torch.where(some, S.log(), 0.0)
    H = lnS + D1
    r = (4 * D + 4 * D1 + 62) * U
    grad, err = torch.zeros_like(p), torch.zeros_like(p)
    rows = torch.arange(x.shape[0])
    if gl is not None:
        g = torch.where(given >= 0, gl, 0.0)[:, None] / t
        grad -= g * p
        err += g.abs() * p * (r + 2 * U)
    if gh is not None:
        h = gh[:, None] / t
        inner = torch.where(p > 0, H - lnS - D, 0.0)  # ln p + H
        err_h = (4 * D2 + 4 * D1 ** 2 + 129 * D1 + 58 + 3 * lnS + H) * U
        err_inner = 5 * D * U + err_h + (2 * lnS + (H - lnS).abs() + inner.abs()) * U
        grad -= h * p * inner
        err += h.abs() * p * (inner.abs() * (r + 4 * U) + err_inner)
    err += 2 * U * grad.abs()
    if gl is not None:
        grad[rows, given.clamp_min(0)] += g[:, 0]
        err[rows, given.clamp_min(0)] += 3 * U * g[:, 0].abs()
    # below 2^-126 an exponential may be 0
    size = sum(a.abs() for a in (gl, gh) if a is not None)
    if not isinstance(size, int):
        err += 2.0 ** -118 * size[:, None] / t
    if excluded is not None:
        grad[excluded] = err[excluded] = 0.0
    return grad, err


def bounds(x, given, t, excluded, gl, gh, dtype):
    """(gradient, allowed error of one rounded to dtype)."""
    grad, err = terms(x, given, t, excluded, gl, gh)
    tol = err + HALF_STEP[dtype] * (grad.abs() + err) + TINY[dtype]
    if excluded is not None:
        tol[excluded] = 0.0
    return grad, tol


def case(rows, cols, dtype, mode):
    """Inputs of a parametrised case: temperature, exclusions and which of the
    two gradients differ by mode."""
    g = torch.Generator().manual_seed(7 * rows + cols + mode)
    x = (2.0 * torch.randn(rows, cols, generator=g)).to(dtype)
    given = torch.randint(-1, cols, (rows,), generator=g)
    gl, gh = (torch.randn(rows, generator=g) for _ in range(2))
    excluded = None
    if mode in (1, 3):
        excluded = torch.rand(rows, cols, generator=g) < 0.2
        excluded[torch.arange(rows), given.clamp_min(0)] = False
    t = float(torch.tensor((1.0, 0.7, 1.7, 1.0)[mode]))  # as 32 bits hold it
    return x, given, t, excluded, gl if mode != 2 else None, gh if mode in (1, 2) else None


SHAPES = [(1, 1), (3, 2), (5, 17), (2, 255), (4, 1024), (3, 2049), (3, 4099), (2, 18000),
          (1, 100003), (700, 33)]
