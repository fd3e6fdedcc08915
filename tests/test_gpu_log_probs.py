"""Log probabilities, entropy and top alternatives, and their gradient, against
the formulas in 64 bits (on the CPU), at the sizes, strides and values where a
one-pass kernel can go wrong."""
import math

import numpy as np
import pytest

from paper_2304_13724_amd import bgmf, ranking

import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# d = (x - M)/t is rounded twice, exp is good to one unit, and a sum of positive
# terms keeps their relative error plus that of its additions (at most some
# thousand in a row per accumulator): ln S is off by about 1e-6 times the mean
# |d| under p (below 10) plus 2e-6; the entropy's second sum by as much times |d|
LOG_TOL = dict(rtol=1e-6, atol=1e-5)
ENTROPY_TOL = dict(rtol=1e-6, atol=3e-5)


def reference(x, given, top, t, excluded):
    """In 64 bits, row by row; x: the rounded scores as a float64 array."""
    rows, cols = x.shape
    lp, ent, m, s = (np.zeros(rows) for _ in range(4))
    ti = np.full((rows, top), -1, np.int32)
    tl = np.full((rows, top), -np.inf)
    for r in range(rows):
        v = x[r].copy()
        if excluded is not None:
            v[excluded[r]] = -np.inf
        kept = v[v != -np.inf]
        g = -1 if given is None else int(given[r])
        if kept.size == 0:
            lp[r] = 0.0 if g == -1 else -np.inf if 0 <= g < cols else np.nan
            m[r] = -np.inf
            continue
        m[r] = np.nanmax(kept) if not np.isnan(kept).all() else np.nan
        with np.errstate(invalid="ignore", over="ignore"):
            d = (v - m[r]) / t
            d[v == -np.inf] = -np.inf
            e = np.exp(d)
            s[r] = e.sum()
            ent[r] = math.log(s[r]) - np.where(e == 0, 0.0, e * np.where(e == 0, 0, d)).sum() / s[r]
            if g == -1:
                lp[r] = 0.0
            else:
                lp[r] = d[g] - math.log(s[r]) if 0 <= g < cols else np.nan
            ranked = np.where(np.isnan(v), -np.inf, v)
            order = np.lexsort((np.arange(cols), -ranked))[:top]
            order = order[ranked[order] > -np.inf]
            ti[r, :order.size] = order
            tl[r, :order.size] = d[order] - math.log(s[r])
    return lp, ent, ti, tl, m, s


def check(x, given=None, top=0, t=1.0, excluded=None, scores=None):
    """x: CPU tensor; scores: the tensor on the GPU to pass (default: x copied)."""
    scores = x.cuda() if scores is None else scores
    ex = None if excluded is None else excluded.cuda()
    g = None if given is None else torch.as_tensor(given, dtype=torch.int32).cuda()
    r = ranking.log_probs(scores, g, top=top, temperature=t, excluded=ex)
    lp, ent, ti, tl, m, s = reference(x.double().numpy(), given, top, t,
                                      None if excluded is None else excluded.numpy())
    got = [y.cpu().numpy() for y in r]
    np.testing.assert_array_equal(got[2], ti)
    np.testing.assert_allclose(got[0], lp, **LOG_TOL)
    np.testing.assert_allclose(got[1], ent, **ENTROPY_TOL)
    np.testing.assert_allclose(got[3], tl, **LOG_TOL)
    finite = np.isfinite(s)
    np.testing.assert_array_equal(got[4][finite], m[finite].astype(np.float32))
    np.testing.assert_allclose(got[5], s, rtol=1e-5)
    return r


def draw(rows, cols, dtype, seed, sigma=2.0):
    g = torch.Generator().manual_seed(seed)
    x = sigma * torch.randn(rows, cols, generator=g)
    return x.to(TYPES[dtype])


def some_given(rows, cols, seed):
    rng = np.random.default_rng(seed)
    return rng.integers(-1, cols, rows) if cols else np.full(rows, -1)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,top", [
    (1, 1, 1), (1, 1, 128), (3, 2, 5), (2, 3, 0), (5, 7, 7), (4, 8, 3), (2, 63, 63), (3, 64, 10),
    (3, 65, 128), (2, 255, 20), (2, 256, 1), (3, 1000, 128), (2, 1023, 50), (2, 1025, 10),
    (2, 4095, 10), (1, 4097, 128), (7, 10007, 20), (1, 18000, 10), (3, 65537, 100), (300, 50, 5),
    (1, 300001, 64), (2, 131072, 10)])
def test_sizes(dtype, rows, cols, top):
    x = draw(rows, cols, dtype, rows * 7 + cols)
    check(x, some_given(rows, cols, cols), top=top)
    g = torch.Generator().manual_seed(cols)
    ex = torch.rand(rows, cols, generator=g) < 0.3
    check(x, some_given(rows, cols, cols + 1), top=top, t=0.7, excluded=ex)


def test_few_items_are_left():
    """Almost everything excluded: fewer left than alternatives asked for."""
    x = draw(6, 20011, "f32", 3)
    ex = torch.ones(6, 20011, dtype=torch.bool)
    ex[1, 777] = False
    ex[2, ::4001] = False
    ex[3, :50] = False
    ex[4, 19990:] = False
    ex[5, ::40] = False
    check(x, [5, 777, 4001, -1, 3, 80], top=40, excluded=ex)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_nothing_left(dtype):
    x = draw(4, 700, dtype, 5)
    x[1] = -math.inf
    ex = torch.zeros(4, 700, dtype=torch.bool)
    ex[2] = True
    r = check(x, [3, 3, -1, 700], top=3, excluded=ex)
    assert r.log_prob[1].item() == -math.inf and r.entropy[1].item() == 0
    assert r.log_prob[2].item() == 0 and math.isnan(r.log_prob[3].item())
    out = ranking.log_probs_backward(
        x.cuda(), torch.tensor([3, 3, -1, 5], dtype=torch.int32).cuda(), r.row_max, r.row_sum,
        r.entropy, torch.ones(4).cuda(), torch.ones(4).cuda(), excluded=ex.cuda())
    assert torch.isfinite(out.float()).all() and not out[1:3].any() and out[0].any()


def test_no_items_and_no_rows():
    r = ranking.log_probs(torch.empty(3, 0).cuda(), torch.tensor([-1, 0, 2]).int().cuda(), top=4)
    assert r.log_prob[0].item() == 0 and torch.isnan(r.log_prob[1:]).all()
    assert not r.entropy.any() and (r.top_item == -1).all()
    assert (r.top_log_prob == -math.inf).all() and (r.row_max == -math.inf).all()
    r = ranking.log_probs(torch.empty(0, 9).cuda(), torch.empty(0).int().cuda(), top=2)
    assert r.log_prob.shape == (0,) and r.top_item.shape == (0, 2)
    for shape in ((3, 0), (0, 9)):
        z = torch.zeros(shape[0]).cuda()
        assert ranking.log_probs_backward(torch.empty(shape).cuda(), z.int(), z, z, z, z).shape == shape


@pytest.mark.parametrize("dtype", list(TYPES))
def test_extreme_values(dtype):
    """The type's lowest and largest values, infinities, signed zeros, and
    garbage in excluded places."""
    low, high = torch.finfo(TYPES[dtype]).min, torch.finfo(TYPES[dtype]).max
    x = draw(8, 3001, dtype, 11)
    ex = torch.zeros(8, 3001, dtype=torch.bool)
    x[0] = low
    x[1, ::2] = low
    x[2, 100:] = -math.inf
    x[3, ::7] = high
    x[4] = torch.tensor([0.0, -0.0]).repeat(1501)[:3001]
    x[5, ::3], ex[5, ::3] = math.nan, True
    x[6, 1::3], ex[6, 1::3] = math.inf, True
    x[7] = high
    x[7, 5] = low
    for t in (1.0, 0.5, 2.0):
        check(x, [7, 3, 200, 7, 9, 1, 0, 6], top=30, t=t, excluded=ex)


@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_not_a_number_or_infinite(value):
    x = draw(3, 5000, "f32", 13)
    x[1, 1234] = value
    x[2] = value
    r = ranking.log_probs(x.cuda(), torch.tensor([5, 5, -1]).int().cuda(), top=5)
    lp, ent, ti, tl, _, _ = reference(x.double().numpy(), [5, 5, -1], 5, 1.0, None)
    np.testing.assert_array_equal(r.top_item.cpu().numpy(), ti)
    assert math.isnan(r.log_prob[1].item()) and r.log_prob[2].item() == 0.0
    assert torch.isnan(r.entropy[1:]).all() and torch.isfinite(r.entropy[0])
    kept = r.top_item[1:] >= 0
    assert torch.isnan(r.top_log_prob[1:][kept]).all()
    assert (r.top_log_prob[1:][~kept] == -math.inf).all()


@pytest.mark.parametrize("cols", [500, 18000, 200003])
def test_orders_and_ties(cols):
    """Rows whose best items lie together, at a fixed distance, or are many:
    equal scores go to the lower item."""
    j = torch.arange(cols)
    rows = [torch.zeros(cols), j.float(), -j.float(), (j % 1024 == 3).float(), (j % 4 == 1).float(),
            (j % 256).float(), (j // 1000).float(), torch.where(j >= cols - 30, 5.0, 0.0),
            (j % 1024 < 40).float() * (1000 - (j // 1024).float()), (j % 2048 < 16).float()]
    x = torch.stack(rows)
    for top in (1, 10, 128):
        check(x, [0] * len(rows), top=top)
        check((x / 8).bfloat16(), [0] * len(rows), top=top)


def test_temperature_extremes():
    x = draw(4, 999, "f32", 17)
    for t in (1e-4, 1e4, 1e30):
        check(x, [1, 2, 3, 4], top=5, t=t)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("offset,stride", [(0, 1009), (1, 1009), (3, 1016), (8, 1024), (5, 1001)])
def test_strides_and_alignment(dtype, offset, stride):
    flat = torch.empty(offset + 6 * stride, dtype=TYPES[dtype])
    flat.fill_(math.nan)
    x = flat[offset:].view(6, stride)[:, :1001]
    x.copy_(draw(6, 1001, dtype, stride))
    scores = flat.cuda()[offset:].view(6, stride)[:, :1001]
    exf = torch.ones(7 + 6 * 1003, dtype=torch.uint8)
    ex = exf[7:].view(6, 1003)[:, :1001]
    ex.copy_((torch.rand(6, 1001, generator=torch.Generator().manual_seed(2)) < 0.2).byte() * 3)
    g = some_given(6, 1001, 1)
    check(x, g, top=9, scores=scores)
    r = ranking.log_probs(scores, torch.as_tensor(g).int().cuda(), top=9,
                          excluded=exf.cuda()[7:].view(6, 1003)[:, :1001])
    want = reference(x.double().numpy(), g, 9, 1.0, ex.numpy() != 0)
    np.testing.assert_array_equal(r.top_item.cpu().numpy(), want[2])
    np.testing.assert_allclose(r.log_prob.cpu().numpy(), want[0], **LOG_TOL)


def test_broadcast_rows():
    """One row of scores, and one of exclusions, for every user (row stride 0)."""
    x = draw(1, 3000, "f32", 23)
    ex = torch.rand(1, 3000, generator=torch.Generator().manual_seed(3)) < 0.5
    r = ranking.log_probs(x.cuda().expand(5, -1), torch.arange(5).int().cuda(), top=4,
                          excluded=ex.cuda().expand(5, -1))
    want = reference(x.double().numpy().repeat(5, 0), range(5), 4, 1.0, ex.numpy().repeat(5, 0))
    np.testing.assert_array_equal(r.top_item.cpu().numpy(), want[2])
    np.testing.assert_allclose(r.log_prob.cpu().numpy(), want[0], **LOG_TOL)


def test_offsets_beyond_32_bits():
    """Rows further apart than 2^31 elements (2^32 bytes)."""
    stride = (1 << 31) + 16
    flat = torch.empty(2 * stride + 3000, dtype=torch.bfloat16, device="cuda")
    scores = flat.as_strided((3, 3000), (stride, 1))
    x = draw(3, 3000, "bf16", 29)
    scores.copy_(x.cuda())
    g = [11, 12, 13]
    r = check(x, g, top=5, scores=scores)
    gl = torch.ones(3).cuda()
    ranking.log_probs_backward(scores, torch.tensor(g).int().cuda(), r.row_max, r.row_sum, None, gl,
                               out=scores)
    small = ranking.log_probs_backward(x.cuda(), torch.tensor(g).int().cuda(), r.row_max,
                                       r.row_sum, None, gl)
    assert torch.equal(scores, small)


def test_long_rows():
    """The largest catalogue: five million items, few rows."""
    g = torch.Generator(device="cuda").manual_seed(31)
    x = 2.0 * torch.randn(2, 5_000_000, generator=g, device="cuda")
    check(x.cpu(), [4_999_999, 17], top=50, scores=x)


def test_same_bits_twice_and_on_another_stream():
    x = draw(3, 200003, "bf16", 37).cuda()
    g = torch.tensor([1, 2, 3]).int().cuda()
    a = ranking.log_probs(x, g, top=20)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = x * 1
        b = ranking.log_probs(y, g, top=20)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_graph_replays():
    x = draw(4, 70001, "f32", 41).cuda()
    g = torch.tensor([1, 2, 3, -1]).int().cuda()
    gl = torch.full((4,), -0.25).cuda()
    ranking.log_probs(x, g, top=8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = ranking.log_probs(x, g, top=8)
        d = ranking.log_probs_backward(x, g, r.row_max, r.row_sum, r.entropy, gl, gl)
    for seed in range(3):
        x.copy_(draw(4, 70001, "f32", 100 + seed).cuda())
        graph.replay()
        torch.cuda.synchronize()
        e = ranking.log_probs(x, g, top=8)
        f = ranking.log_probs_backward(x, g, e.row_max, e.row_sum, e.entropy, gl, gl)
        assert all(torch.equal(p, q) for p, q in zip(r, e)) and torch.equal(d, f)


# --- gradient -----------------------------------------------------------------

def grad_reference(x, given, t, excluded, gl, gh):
    v = x.clone()
    if excluded is not None:
        v[excluded] = -math.inf
    z = v / t
    lp = torch.log_softmax(z, 1)
    p = lp.exp()
    h = -torch.where(p > 0, p * lp, 0.0).sum(1, keepdim=True)
    grad = torch.where(p > 0, -gh[:, None] * p * (torch.where(p > 0, lp, 0.0) + h), 0.0)
    use = (given >= 0).double() * gl
    grad -= use[:, None] * p
    at = torch.arange(x.shape[0])
    grad[at, given.clamp_min(0)] += use
    if excluded is not None:
        grad[excluded] = 0.0
    return grad / t


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (5, 17), (2, 255), (4, 1024), (3, 4099),
                                       (2, 18000), (1, 100003), (700, 33)])
def test_gradient(dtype, rows, cols):
    x = draw(rows, cols, dtype, rows + cols)
    rng = torch.Generator().manual_seed(cols)
    given = torch.randint(-1, cols, (rows,), generator=rng).int()
    gl, gh = torch.randn(rows, generator=rng), torch.randn(rows, generator=rng)
    ex = torch.rand(rows, cols, generator=rng) < 0.2
    ex[torch.arange(rows), given.clamp_min(0).long()] = False
    for t, mask, ge in ((1.0, None, None), (0.7, ex, gh), (1.7, None, gh), (1.0, ex, None)):
        xc, gc = x.cuda(), given.cuda()
        mc = None if mask is None else mask.cuda()
        r = ranking.log_probs(xc, gc, temperature=t, excluded=mc)
        got = ranking.log_probs_backward(xc, gc, r.row_max, r.row_sum, r.entropy, gl.cuda(),
                                         None if ge is None else ge.cuda(), temperature=t,
                                         excluded=mc)
        want = grad_reference(x.double(), given.long(), t, mask, gl.double(),
                              torch.zeros(rows).double() if ge is None else ge.double())
        # p is off by 3e-6 of itself, the entropy by 3e-5; one rounding to the type
        unit = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}[dtype]
        size = (gl.abs() + (0 if ge is None else 20 * ge.abs())).double()[:, None] / t
        tol = unit * want.abs() + 1e-5 * size * torch.ones_like(want) * 0.5 + 2.0 ** -24
        assert ((got.cpu().double() - want).abs() <= tol).all()
        again = xc.clone()
        ranking.log_probs_backward(again, gc, r.row_max, r.row_sum, r.entropy, gl.cuda(),
                                   None if ge is None else ge.cuda(), temperature=t, excluded=mc,
                                   out=again)
        assert torch.equal(again, got)


def test_gradient_against_differences():
    """Through autograd, against central differences of the 64-bit formulas."""
    rows, cols, t, h = 3, 41, 0.8, 1e-5
    x = draw(rows, cols, "f32", 43)
    given = np.array([5, -1, 40])
    ex = torch.rand(rows, cols, generator=torch.Generator().manual_seed(1)) < 0.2
    ex[0, 5] = ex[2, 40] = False
    a, b = torch.tensor([0.3, 2.0, -1.0]), torch.tensor([0.5, -0.2, 1.0])
    leaf = x.cuda().requires_grad_()
    r = ranking.log_probs(leaf, torch.as_tensor(given).int().cuda(), top=3, temperature=t,
                          excluded=ex.cuda())
    ((r.log_prob * a.cuda()).sum() + (r.entropy * b.cuda()).sum()).backward()

    def loss(v):
        lp, ent = reference(v, given, 0, t, ex.numpy())[:2]
        return (lp * a.numpy()).sum() + (ent * b.numpy()).sum()

    base = x.double().numpy()
    for i in range(rows):
        for j in range(cols):
            up, down = base.copy(), base.copy()
            up[i, j] += h
            down[i, j] -= h
            assert abs(leaf.grad[i, j].item() - (loss(up) - loss(down)) / (2 * h)) < 2e-5


def test_gradient_through_one_output_only():
    x = draw(4, 100, "f32", 47)
    given = torch.tensor([1, 2, 3, 4]).int()
    for part in (0, 1):
        leaf = x.cuda().requires_grad_()
        ranking.log_probs(leaf, given.cuda())[part].sum().backward()
        zero, one = torch.zeros(4).double(), torch.ones(4).double()
        want = grad_reference(x.double(), given.long(), 1.0, None, *((one, zero), (zero, one))[part])
        assert (leaf.grad.cpu().double() - want).abs().max() < 1e-5


def test_given_outside_makes_the_row_nan():
    x = draw(3, 50, "f32", 53).cuda()
    g = torch.tensor([50, -2, 7]).int().cuda()
    r = ranking.log_probs(x, g)
    assert torch.isnan(r.log_prob[:2]).all() and torch.isfinite(r.log_prob[2])
    d = ranking.log_probs_backward(x, g, r.row_max, r.row_sum, None, torch.ones(3).cuda())
    assert torch.isnan(d[:2]).all() and torch.isfinite(d[2]).all()


# --- refusals -------------------------------------------------------------------

def test_refusals():
    x = torch.zeros(4, 10, device="cuda")
    g = torch.zeros(4, dtype=torch.int32, device="cuda")
    z = torch.zeros(4, device="cuda")
    for bad in (x.double(), x[0], x.t(), x.cpu(), x.int()):
        with pytest.raises(ValueError):
            ranking.log_probs(bad, None)
    for bad in (g.long(), g[:3], g.cpu(), torch.zeros(8, dtype=torch.int32, device="cuda")[::2]):
        with pytest.raises(ValueError):
            ranking.log_probs(x, bad)
    for bad in (torch.zeros(4, 9, dtype=torch.bool, device="cuda"), x, torch.zeros(4, 10).bool()):
        with pytest.raises(ValueError):
            ranking.log_probs(x, g, excluded=bad)
    for top in (-1, ranking.TOP_MAX + 1):
        with pytest.raises(ValueError):
            ranking.log_probs(x, g, top=top)
    for t in (0.0, -1.0, math.inf, math.nan, 1e-45):
        with pytest.raises(bgmf.BgmfError) as e:
            ranking.log_probs(x, g, temperature=t)
        assert e.value.code == bgmf.BGMF_E_ARG
    with pytest.raises(bgmf.BgmfError):
        ranking.log_probs_backward(x, None, z, z, None, z)
    with pytest.raises(bgmf.BgmfError):
        ranking.log_probs_backward(x, g, z, z, None, z, z)
    for bad in (torch.zeros(4, 10, device="cuda").half(), torch.zeros(4, 9, device="cuda"),
                torch.zeros(1, 10, device="cuda").expand(4, -1)):
        with pytest.raises(ValueError):
            ranking.log_probs_backward(x, g, z, z, None, z, out=bad)
