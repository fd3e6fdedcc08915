"""More ranking operators on given inputs: what is measured, in plain form and exactly.

Four operators beside those of perf/operators.py, for answers from catalogues of half
their size and for training on what users did with the answers:

  quantise  factor rows in 4 bits (e2m1 values, a power-of-two scale for each 32 of them),
            and read back
  product   scores = rows . items^T with both sides in 4 bits, the rows quantised within
            the call
  policy    per row of scores over the catalogue: the clipped policy loss of an item that
            was shown, with a divergence from a reference, and its gradient
  dropout   elements of factors dropped by a counter-based generator, in the forward and
            the backward pass

Sizes are those of the workloads in workloads/synth.py (480,000 users, 18,000, 10,000,
625,000 and 5,000,000 items, k = 64 and 128) and generic ones.  Inputs are drawn on the GPU
from the seed.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32  # values that share a scale


def listed():
    return [
        # a batch of users' factors of an odd width, read back for a second look
        dict(name="quantise_batch", kind="quantise", rows=1_999, k=200, type="bf16", out="f32"),
        # a large catalogue's factors laid out once
        dict(name="quantise_catalogue", kind="quantise", rows=625_000, k=128, type="f32",
             out="bf16"),
        # one request over the largest catalogue, k = 64
        dict(name="product_one_user", kind="product", rows=1, items=5_000_000, k=64, type="f32",
             out="f32"),
        # a batch of requests over the benchmark's catalogue, k = 64
        dict(name="product_batch", kind="product", rows=2_048, items=18_000, k=64, type="f32",
             out="bf16"),
        # odd sizes: tens of users, rows that end inside a block
        dict(name="product_ragged", kind="product", rows=37, items=100_003, k=200, type="bf16",
             out="f16"),
        # wide rows (a tower's output in place of factors): the product itself counts
        dict(name="product_wide", kind="product", rows=4_096, items=8_192, k=4_096, type="bf16",
             out="bf16"),
        # a small update as answers come in: the divergence estimated from the shown items
        dict(name="policy_step_small", kind="policy", mode="step", rows=16, cols=18_000,
             type="f32", kl="shown", temperature=1.0, excluded=False),
        # a training batch over the benchmark's catalogue; what users have rated is left out
        dict(name="policy_step_batch", kind="policy", mode="step", rows=2_047, cols=18_000,
             type="bf16", kl="full", temperature=0.7, excluded=True),
        # evaluation: how far the policy has moved, no gradient, an odd catalogue
        dict(name="policy_heldout", kind="policy", mode="value", rows=4_001, cols=10_007,
             type="f32", kl="full", temperature=1.0, excluded=False),
        # few rows of a large catalogue, through autograd, an odd length
        dict(name="policy_autograd_long", kind="policy", mode="autograd", rows=33, cols=625_001,
             type="f32", kl="full", temperature=1.3, excluded=False),
        # a batch of users' factors in the forward pass
        dict(name="dropout_batch", kind="dropout", mode="value", rows=4_096, k=64, type="f32",
             p=0.1),
        # all users' factors, forward and backward
        dict(name="dropout_factors", kind="dropout", mode="autograd", rows=480_000, k=64,
             type="bf16", p=0.2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One user to 4,096, one item to five million, k from 1 to 4,096."""
    kind = rng.choice(["quantise", "product", "product", "policy", "policy", "dropout"])
    type_ = rng.choice(["f32", "bf16", "f16"])
    if kind == "quantise":
        k = _log(rng, 1, 4_096)
        return dict(kind=kind, rows=_log(rng, 1, 80_000_000 // k), k=k, type=type_,
                    out=rng.choice(["f32", "bf16", "f16"]))
    if kind == "product":
        k = _log(rng, 1, 4_096)
        rows = _log(rng, 1, 4_096)
        most = min(5_000_000, 300_000_000 // k, 40_000_000 // rows, 130_000_000_000 // (rows * k))
        return dict(kind=kind, rows=rows, items=_log(rng, 1, max(1, most)), k=k, type=type_,
                    out=rng.choice(["f32", "bf16", "f16"]))
    if kind == "policy":
        cols = _log(rng, 1, 5_000_000)
        rows = _log(rng, 1, min(4_096, max(1, 20_000_000 // cols)))
        return dict(kind=kind, mode=rng.choice(["value", "step", "autograd"]), rows=rows,
                    cols=cols, type=type_, kl=rng.choice(["none", "shown", "full", "full"]),
                    temperature=rng.choice([1.0, 0.7, 1.3]), excluded=rng.random() < 0.5)
    k = _log(rng, 1, 1_024)
    return dict(kind=kind, mode=rng.choice(["value", "autograd"]),
                rows=_log(rng, 1, 30_000_000 // k), k=k, type=type_,
                p=rng.choice([0.0, 0.1, 0.2, 0.5]))


# ------------------------------------------------------------------ inputs

def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _blocks(k):
    return (k + BLOCK - 1) // BLOCK


def _quantised(x):
    """Rows (fp32) in blocks of 32, the last one filled up with zeros: per block a scale
    2^e, e = floor(log2(largest magnitude)) - 2, and the quotients rounded to the nearest of
    0, 0.5, 1, 1.5, 2, 3, 4 and 6 (ties to the one whose last bit is even, larger ones to
    6).  Returns the quotients [rows, blocks, 32] and e + 127 [rows, blocks]."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x, (0, _blocks(k) * BLOCK - k)).view(rows, _blocks(k), BLOCK)
    most = x.abs().amax(2)
    code = torch.where(most > 0, most.frexp().exponent - 1 - 2 + 127, 0).clamp(0, 254)
    v = x * ((254 - code) << 23).view(torch.float32)[:, :, None]
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp_max(6.0), v), code


def _packed(q, code):
    """The layout in memory: a sign and three bits a value, the even one of two in the
    lower half of their byte; a byte a scale."""
    a = q.abs()
    nibble = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a * 0.5 + 4)).to(torch.uint8)
    nibble |= torch.signbit(q).to(torch.uint8) << 3
    nibble = nibble.view(q.shape[0], -1, 2)
    return nibble[:, :, 0] | nibble[:, :, 1] << 4, code.to(torch.uint8)


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    kind, type_ = case["kind"], TYPES[case["type"]]
    s = {"case": case}
    if kind == "dropout":
        s["x"] = torch.randn(case["rows"], case["k"], generator=g, device=dev).to(type_)
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (seed + 1) % (1 << 62), 1_000_003 * seed
        if case["mode"] == "autograd":
            s["x"].requires_grad_()
            s["grad"] = torch.randn(case["rows"], case["k"], generator=g, device=dev).to(type_)
        return s
    if kind in ("quantise", "product"):
        rows = torch.randn(case["rows"], case["k"], generator=g, device=dev)
        rows *= torch.rand(case["rows"], 1, generator=g, device=dev) + 0.1
        if case["rows"] > 8:
            rows[5] = 0.0  # a user without ratings
        s["rows"] = rows.to(type_)
        if kind == "product":
            items = torch.randn(case["items"], case["k"], generator=g, device=dev)
            items *= torch.rand(case["items"], 1, generator=g, device=dev) + 0.1
            s["items"], s["item_scale"] = _packed(*_quantised(items))
        return s
    rows, cols, t = case["rows"], case["cols"], case["temperature"]
    x = 2.0 * torch.randn(rows, cols, generator=g, device=dev)
    x += torch.randn(cols, generator=g, device=dev)  # an item's popularity
    y = x + 0.3 * torch.randn(rows, cols, generator=g, device=dev)  # before training
    x, y = x.to(type_), y.to(type_)
    given = torch.randint(0, cols, (rows,), generator=g, device=dev, dtype=torch.int32)
    s["excluded"] = None
    if case["excluded"]:
        s["excluded"] = torch.rand(rows, cols, generator=g, device=dev) < 0.01
        s["excluded"][torch.arange(rows, device=dev), given.long()] = False
        if rows > 8:
            s["excluded"][3] = True  # a user who has rated everything
            given[4] = -1  # a row that fills the batch up
    s["scores"], s["given"] = x.requires_grad_(case["mode"] == "autograd"), given
    # log probabilities of the shown items when they were shown, and before training
    z = y.float() / t
    if s["excluded"] is not None:
        z = z.masked_fill(s["excluded"], -math.inf)
    before = z.gather(1, given.clamp_min(0).long()[:, None])[:, 0] - z.logsumexp(1)
    before = torch.where(before > -math.inf, before, -1.0)
    s["old_log_prob"] = before + 0.1 * torch.randn(rows, generator=g, device=dev)
    s["advantage"] = torch.randn(rows, generator=g, device=dev)
    s["reference"] = y if case["kl"] == "full" else None
    s["reference_log_prob"] = before if case["kl"] == "shown" else None
    s["kl_weight"] = 0.0 if case["kl"] == "none" else 0.05
    s["weight"] = torch.rand(rows, generator=g, device=dev)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return _calls(s) if own else _plain(s)


def _calls(s):
    from paper_2304_13724_amd import ranking

    case = s["case"]
    if case["kind"] == "quantise":
        q, scale = ranking.quantize_rows_mx4(s["rows"])
        return ranking.dequantize_rows_mx4(q, scale, case["k"], dtype=TYPES[case["out"]])
    if case["kind"] == "product":
        return ranking.mx4_scores(s["rows"], s["items"], s["item_scale"],
                                  dtype=TYPES[case["out"]])
    if case["kind"] == "dropout":
        y = ranking.dropout(s["x"], case["p"], s["seed"], s["offset"])
        if case["mode"] == "value":
            return y
        return {"y": y, "grad": torch.autograd.grad(y, s["x"], s["grad"])[0]}
    options = dict(reference=s["reference"], reference_log_prob=s["reference_log_prob"],
                   kl_weight=s["kl_weight"], clip_low=0.2, clip_high=0.25,
                   temperature=case["temperature"], excluded=s["excluded"])
    at = (s["scores"], s["given"], s["advantage"], s["old_log_prob"])
    if case["mode"] == "step":
        r, grad = ranking.policy_loss_and_grad(*at, s["weight"], **options)
        return {"loss": r.loss, "log_prob": r.log_prob, "kl": r.kl, "grad": grad}
    r = ranking.policy_loss(*at, **options)
    got = {"loss": r.loss, "log_prob": r.log_prob, "kl": r.kl}
    if case["mode"] == "autograd":
        got["grad"] = torch.autograd.grad(r.loss, s["scores"], s["weight"])[0]
    return got


def _plain(s):
    return {"quantise": _plain_quantise, "product": _plain_product, "policy": _plain_policy,
            "dropout": _plain_dropout}[s["case"]["kind"]](s)


def _values(q, code):
    """Quotients and scale codes -> rows of values."""
    return (q * (code << 23).view(torch.float32)[:, :, None]).view(q.shape[0], -1)


def _plain_quantise(s):
    return _values(*_quantised(s["rows"].float()))[:, :s["case"]["k"]].to(TYPES[s["case"]["out"]])


def _plain_product(s):
    q = s["items"]
    q = torch.stack((q & 15, q >> 4), 2).view(q.shape[0], -1).int()
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=q.device)
    table = torch.cat((table, -table))
    items = table.index_select(0, q.view(-1)).view(q.shape[0], -1, BLOCK)
    items = _values(items, s["item_scale"].int())
    return (_values(*_quantised(s["rows"].float())) @ items.t()).to(TYPES[s["case"]["out"]])


def _plain_policy(s):
    case, t, given = s["case"], s["case"]["temperature"], s["given"].long()
    x = s["scores"].detach().float()
    if s["excluded"] is not None:
        x = x.masked_fill(s["excluded"], -math.inf)
    top = x.amax(1)
    top = torch.where(top > -math.inf, top, 0.0)
    d = (x - top[:, None]) / t
    e = d.exp()
    total = e.sum(1, dtype=torch.float64)
    some = total > 0
    part = some & (given >= 0)
    total = torch.where(some, total, 1.0)
    at = given.clamp_min(0)[:, None]
    # a row's own numbers in 64 bits: the divergence is a small difference of large ones
    log_prob = d.gather(1, at)[:, 0].double() - total.log()
    ratio = (log_prob - s["old_log_prob"].double()).exp()
    advantage = s["advantage"].double()
    free, held = ratio * advantage, ratio.clamp(1 - 0.2, 1 + 0.25) * advantage
    loss, slope = -torch.minimum(free, held), torch.where(free <= held, -free, 0.0)
    kl = torch.zeros_like(loss)
    if s["reference_log_prob"] is not None:
        z = s["reference_log_prob"].double() - log_prob
        kl = z.expm1() - z
        slope = slope - s["kl_weight"] * z.expm1()
    if s["reference"] is not None:
        y = s["reference"].float()
        if s["excluded"] is not None:
            y = y.masked_fill(s["excluded"], -math.inf)
        y_top = y.amax(1)
        y_d = (y - torch.where(y_top > -math.inf, y_top, 0.0)[:, None]) / t
        y_total = y_d.exp().sum(1, dtype=torch.float64)
        moved = torch.where(e > 0, d - y_d, 0.0)
        mean = (e * moved).sum(1, dtype=torch.float64) / total
        kl = mean - total.log() + torch.where(some, y_total, 1.0).log()
    loss = loss + s["kl_weight"] * kl
    got = {"loss": torch.where(part, loss, 0.0).float(),
           "log_prob": torch.where(given >= 0, torch.where(some, log_prob, -math.inf), 0.0).float(),
           "kl": torch.where(part, kl, 0.0).float()}
    if case["mode"] == "value":
        return got
    p = e / total.float()[:, None]
    slope = torch.where(part, slope, 0.0).float()[:, None]
    grad = -slope * p
    if s["reference"] is not None:
        grad += s["kl_weight"] * p * (moved - torch.where(part, mean, 0.0).float()[:, None])
    grad.scatter_add_(1, at, slope)
    grad = torch.where(part[:, None], grad * (s["weight"] / t)[:, None], 0.0)
    if s["excluded"] is not None:
        grad = grad.masked_fill(s["excluded"], 0.0)
    got["grad"] = grad.to(s["scores"].dtype)
    return got


def _plain_words(seed, offset, count, device):
    """Words 0..count-1 of the generator Philox4x32 with ten rounds (Salmon, Moraes, Dror
    and Shaw, 2011): four for each counter from `offset` on, the seed as its key."""
    low = (1 << 32) - 1

    def times(a, b):  # the upper and lower 32 bits of a 32-bit number times a constant
        lo, hi = a * (b & 0xFFFF), a * (b >> 16)
        mid = lo + ((hi & 0xFFFF) << 16)
        return (hi >> 16) + (mid >> 32), mid & low

    c = offset + torch.arange((count + 3) // 4, device=device)
    x = [c & low, c >> 32 & low, torch.zeros_like(c), torch.zeros_like(c)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        h0, l0 = times(x[0], 0xD2511F53)
        h1, l1 = times(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack(x, 1).view(-1)[:count]


def _plain_dropout(s):
    case, x = s["case"], s["x"].detach()
    kept = _plain_words(s["seed"], s["offset"], x.numel(), x.device) >= int(case["p"] * (1 << 32))
    kept = kept.view(x.shape)

    def drop(x):
        return torch.where(kept, x.float() * (1.0 / (1.0 - case["p"])), 0.0).to(x.dtype)

    return drop(x) if case["mode"] == "value" else {"y": drop(x), "grad": drop(s["grad"])}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind == "quantise":
        n, laid = case["rows"] * case["k"], case["rows"] * _blocks(case["k"]) * 17
        return {"bytes": n * (BYTES[case["type"]] + BYTES[case["out"]]) + 2 * laid, "flops": 3 * n}
    if kind == "product":
        rows, items, k = case["rows"], case["items"], case["k"]
        return {"bytes": rows * k * BYTES[case["type"]] + items * _blocks(k) * 17
                + rows * items * BYTES[case["out"]], "flops": 2 * rows * items * k}
    if kind == "dropout":
        n = case["rows"] * case["k"] * (1 if case["mode"] == "value" else 2)
        return {"bytes": 2 * n * BYTES[case["type"]], "flops": 12 * n}
    cells, full = case["rows"] * case["cols"], case["kl"] == "full"
    read = cells * (BYTES[case["type"]] * (2 if full else 1) + (1 if case["excluded"] else 0))
    write = 0 if case["mode"] == "value" else cells * BYTES[case["type"]]
    return {"bytes": read + write + 32 * case["rows"],
            "flops": cells * ((10 if full else 4) + (0 if case["mode"] == "value" else 6))}


# ------------------------------------------------------------------ in 64 bits

def _power(e):
    """2^e in 64 bits, exactly."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_values(x):
    """What rows stand for in 4 bits: the nearest representable value, by a search."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -k % BLOCK)).view(rows, -1, BLOCK)
    most = x.abs().amax(2, keepdim=True)
    exponent = torch.where(most > 0, torch.frexp(most).exponent - 1, 0)
    scale = _power(exponent - 2)
    a = x.abs() / scale
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64,
                        device=x.device)
    upper = torch.searchsorted((grid[1:] + grid[:-1]) / 2, a.contiguous())  # ties to the lower one
    tie = (a == ((grid[1:] + grid[:-1]) / 2)[upper.clamp_max(6)]) & (upper < 7)
    upper = torch.where(tie & (upper % 2 == 1), upper + 1, upper)
    return (torch.sign(x) * grid[upper] * scale).view(rows, -1)[:, :k]


def _exact_words(seed, offset, count):
    """The generator's words once more, in unsigned 64-bit numbers on the host."""
    low = np.uint64(0xFFFFFFFF)
    c = np.uint64(offset) + np.arange((count + 3) // 4, dtype=np.uint64)
    a0, a1, a2, a3 = c & low, c >> np.uint64(32), np.zeros_like(c), np.zeros_like(c)
    for i in range(10):
        k0 = np.uint64((seed + i * 0x9E3779B9) & 0xFFFFFFFF)
        k1 = np.uint64(((seed >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)
        u, v = a0 * np.uint64(0xD2511F53), a2 * np.uint64(0xCD9E8D57)
        a0, a1 = (v >> np.uint64(32)) ^ a1 ^ k0, v & low
        a2, a3 = (u >> np.uint64(32)) ^ a3 ^ k1, u & low
    words = np.empty((len(c), 4), dtype=np.uint32)
    for i, a in enumerate((a0, a1, a2, a3)):
        words[:, i] = a
    return words.reshape(-1)[:count]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantise":
        return _exact_values(s["rows"])
    if case["kind"] == "product":
        q, k = s["items"], case["k"]
        sign = 1.0 - 2.0 * (torch.stack((q >> 3 & 1, q >> 7), 2).view(q.shape[0], -1).double())
        m = torch.stack((q & 7, q >> 4 & 7), 2).view(q.shape[0], -1)
        # three bits: two of exponent, one of fraction
        e, f = (m >> 1).int(), (m & 1).double()
        items = sign * torch.where(e == 0, f / 2, (1.0 + f / 2) * _power(e - 1))
        items = items.view(q.shape[0], -1, BLOCK)
        items = items * _power(s["item_scale"].long()[:, :, None] - 127)
        return _exact_values(s["rows"]) @ items.view(q.shape[0], -1)[:, :k].t().contiguous()
    if case["kind"] == "dropout":
        words = _exact_words(s["seed"], s["offset"], s["x"].numel())
        kept = torch.from_numpy(words >= case["p"] * 2.0**32).to(s["x"].device).view(s["x"].shape)
        factor = kept.double() / (1.0 - case["p"])
        y = s["x"].detach().double() * factor
        return y if case["mode"] == "value" else {"y": y, "grad": s["grad"].double() * factor}
    t, rows = case["temperature"], case["rows"]
    z = s["scores"].detach().double() / t
    if s["excluded"] is not None:
        z[s["excluded"]] = -math.inf
    z.requires_grad_()
    part = ((z > -math.inf).any(1) & (s["given"] >= 0)).detach()
    # rows that take part, by automatic differentiation
    use = part.nonzero()[:, 0]
    log_p = torch.log_softmax(z[use], 1)
    log_prob = log_p.gather(1, s["given"][use].long()[:, None])[:, 0]
    ratio, advantage = (log_prob - s["old_log_prob"][use].double()).exp(), s["advantage"][use].double()
    loss = -torch.minimum(ratio * advantage, ratio.clamp(0.8, 1.25) * advantage)
    kl = torch.zeros_like(loss)
    if s["reference_log_prob"] is not None:
        u = s["reference_log_prob"][use].double() - log_prob
        kl = u.exp() - u - 1
    if s["reference"] is not None:
        zy = s["reference"][use].double() / t
        if s["excluded"] is not None:
            zy[s["excluded"][use]] = -math.inf
        log_q = torch.log_softmax(zy, 1)
        left = log_p > -math.inf
        kl = (log_p.exp() * torch.where(left, log_p - torch.where(left, log_q, 0.0), 0.0)).sum(1)
    loss = loss + s["kl_weight"] * kl
    none = torch.zeros(rows, dtype=torch.float64, device=z.device)
    empty = torch.where(s["given"] >= 0, -math.inf, none)
    got = {"loss": none.index_copy(0, use, loss.detach()),
           "log_prob": empty.index_copy(0, use, log_prob.detach()),
           "kl": none.index_copy(0, use, kl.detach())}
    if case["mode"] == "value":
        return got
    grad = torch.zeros_like(z)
    if len(use):
        (grad,) = torch.autograd.grad(loss, z, s["weight"][use].double())
    got["grad"] = grad.nan_to_num(0.0) / t
    return got
