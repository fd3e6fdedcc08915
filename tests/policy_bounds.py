"""The policy loss in 64 bits, and how far results computed in 32 bits may be from it.

With u = 2^-24, D_j = (max x - x_j) / t and E_j = (max y - y_j) / t, p and q the
two softmaxes, D1 the mean of D under p and E1 that of E under q:

  exp(-D_j)    the argument is rounded four times (difference, log2 e, division by
               t, product): 4 D_j u; the exponential is good to 2 u
  S            terms with that error, rescaled to a larger maximum some 20 times
               at most (2 u each, and the D's add up), summed with 15 others in
               32 bits before 64-bit sums: (4 D1 + 58) u of itself; Sy likewise
  ln p_g       64 bits but for S: e_lp = (4 D1 + 58) u (and c, the rounded 1 / t,
               is in the terms alone)
  rho          e_lp of itself; the loss and its slope likewise
  mean         sum p_j (E_j - D_j): the terms' (5 D_j + 5 E_j) u, their weights'
               (4 D_j + 62 + 16) u of |E_j - D_j|, and S's error of the whole;
               it is stored in 32 bits
  kl           mean, ln S and ln Sy
  estimate     z in 64 bits: |e^z - 1| e_lp
  p_j          r_j = (4 D_j + 4 D1 + 62) u
"""
import math

import torch

U = 2.0 ** -24
HALF_STEP = {d: torch.finfo(d).eps / 2 for d in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def softmax_of(x, t, excluded):
    v = x if excluded is None else x.masked_fill(excluded, -math.inf)
    top = v.amax(1, keepdim=True)
    D = torch.where(v > -math.inf, (top - v) / t, 0.0)
    e = torch.where(v > -math.inf, torch.exp(-D), 0.0)
    S = e.sum(1, keepdim=True)
    p = e / S
    return D, p, S.log(), (p * D).sum(1, keepdim=True)


def reference(x, given, adv, old, t, lo, hi, weight, y=None, ref_lp=None, excluded=None, g=None):
    """{name: (value, allowed error)} of rows that take part and are not empty; float64."""
    D, p, lnS, D1 = softmax_of(x, t, excluded)
    at = given[:, None]
    lp = -D.gather(1, at) - lnS
    adv, old = adv[:, None], old[:, None]
    e_lp = (4 * D1 + 58) * U
    rho = (lp - old).exp()
    free, held = rho * adv, rho.clamp(1 - lo, 1 + hi) * adv
    passes = free <= held
    loss, e_loss = -torch.minimum(free, held), rho * adv.abs() * 1.01 * e_lp
    slope = torch.where(passes, -free, 0.0)
    e_slope = torch.where(passes, e_loss, 0.0)
    kl, e_kl = torch.zeros_like(lp), torch.zeros_like(lp)
    if ref_lp is not None:
        z = ref_lp[:, None] - lp
        kl, e_kl = z.expm1() - z, z.expm1().abs() * 1.01 * e_lp + e_lp ** 2
        slope = slope - weight * z.expm1()
        e_slope = e_slope + abs(weight) * z.exp() * 1.01 * e_lp
    if y is not None:
        E, q, lnSy, E1 = softmax_of(y, t, excluded)
        moved = E - D  # d - dy
        mean = (p * moved).sum(1, keepdim=True)
        e_moved = (5 * D + 5 * E) * U
        e_mean = (p * (e_moved + moved.abs() * (4 * D + 78) * U)).sum(1, keepdim=True) \
            + mean.abs() * (4 * D1 + 59) * U
        kl = mean - lnS + lnSy
        e_kl = e_mean + e_lp + (4 * E1 + 58) * U
    loss = loss + weight * kl
    e_loss = e_loss + abs(weight) * e_kl
    got = {n: (v[:, 0], e[:, 0] + U * (v[:, 0].abs() + e[:, 0]) + 2.0 ** -126)
           for n, v, e in (("loss", loss, e_loss), ("log_prob", lp, e_lp), ("kl", kl, e_kl))}
    if g is None:
        return got
    # the slope and the mean are stored in 32 bits; g / t, the products
    gs = g[:, None] / t
    r = (4 * D + 4 * D1 + 62) * U
    grad = -gs * slope * p
    err = gs.abs() * p * (slope.abs() * (r + 5 * U) + e_slope)
    if y is not None:
        gk = gs * weight
        grad = grad + gk * p * (moved - mean)
        err = err + gk.abs() * p * ((moved - mean).abs() * (r + 8 * U) + e_moved + 2 * e_mean
                                    + moved.abs() * U)
        err = err + 2 * U * gk.abs() * p * (moved - mean).abs()
    err = err + 3 * U * gs.abs() * slope.abs() * p
    own = torch.zeros_like(p).scatter_(1, at, 1.0)
    grad = grad + own * gs * slope
    err = err + own * gs.abs() * (slope.abs() * 5 * U + e_slope)
    # below 2^-126 an exponential may be 0, whatever multiplies it
    err = err + 2.0 ** -110 * gs.abs() * (1 + slope.abs() + (moved.abs() if y is not None else 0))
    if excluded is not None:
        grad, err = grad.masked_fill(excluded, 0.0), err.masked_fill(excluded, 0.0)
    got["grad"] = (grad, err)
    return got


def allowed(grad, err, dtype):
    tol = err + HALF_STEP[dtype] * (grad.abs() + err) + TINY[dtype]
    return torch.where((grad == 0) & (err == 0), 0.0, tol)


def case(rows, cols, dtype, seed, excluded=False, drift=0.3):
    """Inputs: every row takes part, and no ratio is within 1e-3 of a bound of [0.8, 1.3]."""
    g = torch.Generator().manual_seed(1000 * seed + 7 * rows + cols)
    x = (2.0 * torch.randn(rows, cols, generator=g)).to(dtype)
    y = (x.float() + drift * torch.randn(rows, cols, generator=g)).to(dtype)
    given = torch.randint(0, cols, (rows,), generator=g)
    ex = None
    if excluded:
        ex = torch.rand(rows, cols, generator=g) < 0.2
        ex[torch.arange(rows), given] = False
    adv = torch.randn(rows, generator=g)
    ratio = torch.rand(rows, generator=g) * 1.2 + 0.4
    ratio = torch.where((ratio - 0.8).abs() < 1e-3, ratio + 0.01, ratio)
    ratio = torch.where((ratio - 1.3).abs() < 1e-3, ratio + 0.01, ratio)
    t = float(torch.tensor((1.0, 0.7, 1.7)[seed % 3]))  # as 32 bits hold it
    D, _, lnS, _ = softmax_of(x.double(), t, ex)
    lp = (-D.gather(1, given[:, None]) - lnS)[:, 0]
    old = (lp - ratio.double().log()).float()
    ref_lp = (lp + 0.4 * torch.randn(rows, generator=g)).float()
    weight = torch.randn(rows, generator=g)
    return dict(x=x, y=y, given=given, ex=ex, adv=adv, old=old, ref_lp=ref_lp, weight=weight, t=t)


LO, HI, KL = (float(torch.tensor(v)) for v in (0.2, 0.3, 0.06))
