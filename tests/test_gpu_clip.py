"""Clipping by the global norm against the formula in 64 bits."""
import math

import pytest

from paper_2304_13724_amd import bgmf, ranking

import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -22, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def grads_of(sizes, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=g)).to(TYPES[d])
            for n, d in zip(sizes, dtype if isinstance(dtype, list) else [dtype] * len(sizes))]


def check(grads, most, on=None, out=None):
    """The norm is one rounding (and a square root) from the 64-bit one; the
    factor takes one division and the product one more rounding."""
    on = [g.cuda() for g in grads] if on is None else on
    norm = math.sqrt(sum(g.double().square().sum().item() for g in grads))
    got = ranking.clip_grad_norm(on, most, out=out)
    assert abs(got.item() - norm) <= 2.0 ** -22 * norm
    factor = most / norm if norm > most else 1.0
    for g, h in zip(grads, on if out is None else out):
        want = g.double() * factor
        tol = UNIT[g.dtype] * want.abs() + 2.0 ** -24 * (g.dtype == torch.float16)
        assert ((h.cpu().double() - want).abs() <= tol).all()
        if factor == 1.0:
            assert torch.equal(h.cpu(), g)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sizes", [[1], [7], [8192], [8193, 1], [100_003], [5, 0, 17, 1],
                                   [3] * 59, [11] * 60, [13] * 61, [2] * 121, [1000] * 300,
                                   [1, 500_001, 2, 30_000, 3]])
def test_sizes(dtype, sizes):
    grads = grads_of(sizes, dtype, len(sizes) + sum(sizes))
    check(grads, 0.5)
    check(grads, 1e6)


def test_mixed_types_and_matrices():
    grads = [g.reshape(-1, 64) for g in grads_of([64 * 1000, 64 * 333, 64 * 7], ["f32", "bf16", "f16"],
                                                 1)]
    check(grads, 1.0)
    out = [torch.empty_like(g.cuda()) for g in grads]
    on = [g.cuda() for g in grads]
    check(grads, 1.0, on=on, out=out)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(on, grads))  # inputs unchanged


@pytest.mark.parametrize("dtype", list(TYPES))
def test_views_into_one_bucket(dtype):
    """Odd sizes one after another: every alignment of a start."""
    sizes = [1, 2, 3, 5, 8191, 7, 8193, 20_001, 1, 9, 4097]
    flat = torch.cat(grads_of(sizes, dtype, 5))
    on = list(flat.cuda().split(sizes))
    to = torch.empty(sum(sizes) + 3, dtype=TYPES[dtype], device="cuda")[3:]
    check(list(flat.split(sizes)), 0.25, on=on, out=list(to.split(sizes)))
    check(list(flat.split(sizes)), 0.25, on=on)


def test_row_strides():
    """Columns of a wider matrix: what lies between is neither read nor written."""
    wide = torch.full((57, 100), math.nan, device="cuda")
    g = grads_of([57 * 33], "f32", 7)[0].view(57, 33)
    view = wide[:, 11:44]
    view.copy_(g)
    check([g], 1.0, on=[view])
    assert torch.isnan(wide[:, :11]).all() and torch.isnan(wide[:, 44:]).all()
    view.copy_(g)
    check([g], 1.0, on=[view], out=[torch.empty(57, 33, device="cuda")])
    to = torch.full((57, 40), 3.0, device="cuda")
    check([g], 1.0, on=[g.cuda()], out=[to[:, :33]])
    assert (to[:, 33:] == 3.0).all()


def test_large_and_small_values():
    """Squares that 32 bits cannot hold."""
    check(grads_of([5000], "f32", 9, 1e30), 1.0)
    check(grads_of([5000], "f32", 10, 1e-30), 1e-29)
    check([torch.zeros(100)], 1.0)
    check([torch.zeros(100)], 0.0)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad):
    grads = grads_of([1000, 500], "f32", 11)
    grads[1][77] = bad
    on = [g.cuda() for g in grads]
    norm = ranking.clip_grad_norm(on, 1.0).item()
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    assert all(torch.equal(a.cpu().nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(on, grads))


def test_zero_max_norm_and_infinite_max_norm():
    check(grads_of([500], "f32", 12), 0.0)
    check(grads_of([500], "f32", 13), math.inf)


def test_offsets_beyond_32_bits():
    """A gradient of more than 2^32 bytes, its large values at the end."""
    n = (1 << 31) + 12_345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-3:] = torch.tensor([3.0, 4.0, 12.0])
    g[5] = 84.0
    assert ranking.clip_grad_norm([g], 42.5).item() == 85.0
    assert g[-3:].tolist() == [1.5, 2.0, 6.0] and g[5].item() == 42.0


def test_same_bits_twice_graphs_and_streams():
    g = [x.cuda() for x in grads_of([70_001, 3, 900], "f32", 14)]
    out = [torch.empty_like(x) for x in g]
    ranking.clip_grad_norm(g, 1.0, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = ranking.clip_grad_norm(g, 1.0, out=out)
    for seed in range(3):
        for x, y in zip(g, grads_of([70_001, 3, 900], "f32", 20 + seed)):
            x.copy_(y.cuda())
        graph.replay()
        torch.cuda.synchronize()
        first = [norm.clone()] + [x.clone() for x in out]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = [torch.empty_like(x) for x in g]
            again = [ranking.clip_grad_norm(g, 1.0, out=other)] + other
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_refusals():
    g = torch.ones(10, 10, device="cuda")
    for bad in ([], [g.cpu()], [g.double()], [g, g.int()], [g.t()[:5]], [g[:, ::2]],
                [g[:1].expand(10, -1)]):
        with pytest.raises(ValueError):
            ranking.clip_grad_norm(bad, 1.0)
    for out in ([], [g[:5]], [g.half()], [g.cpu()], [g[:1].expand(10, -1)]):
        with pytest.raises(ValueError):
            ranking.clip_grad_norm([g], 1.0, out=out)
    for most in (-1.0, math.nan):
        with pytest.raises(bgmf.BgmfError) as e:
            ranking.clip_grad_norm([g], most)
        assert e.value.code == bgmf.BGMF_E_ARG
    assert (g == 1).all()
