"""Sizes at which a workgroup goes on to a second tile, row or part of the table,
with what it has in registers or LDS from the first."""
import pytest

from paper_2304_13724_amd import ranking

import torch

pytestmark = pytest.mark.gpu

GROUPS = 1 << 20  # workgroups of a launch, at most


def draw8(rows, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-127, 128, (rows, k), generator=g, device="cuda", dtype=torch.int8)
    q[:, 0] = 127  # so that values q a have bytes q, whatever the scale
    return q, torch.rand(rows, generator=g, device="cuda") + 0.5


def product(q, a, w, b):
    """Exact sums in doubles, then fp32."""
    return (q.double() @ w.double().t()).float() * a[:, None] * b[None]


# more tiles than workgroups at a time, and several steps of k in each tile
@pytest.mark.parametrize("rows,items,k", [(1030, 12000, 200), (200, 70001, 130), (60, 140_000, 200),
                                          (64, 140_003, 65)])
def test_product_second_tile_of_several_steps(rows, items, k):
    q, a = draw8(rows, k, 1)
    w, b = draw8(items, k, 2)
    assert torch.equal(ranking.quantized_scores(q, w, b, a), product(q, a, w, b))


# values that the tiles quantise themselves, more tiles than workgroups
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,items,k", [(4000, 3000, 64), (4000, 2999, 50), (520, 21_000, 33)])
def test_product_of_values_second_tile(rows, items, k, dtype):
    q, _ = draw8(rows, k, 3)
    w, b = draw8(items, k, 4)
    x = q.to(dtype)  # scale 1
    x[7] = 0.0
    x[8, 3] = float("nan")
    one = torch.ones(rows, device="cuda")
    want = product(q, one, w, b)
    want[7], want[8] = 0.0, float("nan")
    got = ranking.quantized_scores(x, w, b)
    assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


def windows(rows, cols, seed, dtype=torch.float32):
    """Overlapping rows: row r is elements r .. r + cols of one vector."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    line = (2 * torch.randn(rows + cols, generator=g, device="cuda")).to(dtype)
    return line.as_strided((rows, cols), (1, 1))


# by four, 16 and 64 lanes to a row, and a workgroup to a row
@pytest.mark.parametrize("k,per_group", [(3, 64), (37, 16), (150, 4), (2100, 1)])
def test_quantize_more_rows_than_workgroups(k, per_group):
    rows = GROUPS * per_group + 777
    x = windows(rows, k, k)
    q, scale = ranking.quantize_rows(x)
    step = max(1, (1 << 27) // k)
    for r in range(0, rows, step):
        part = x[r:r + step].contiguous()
        want = part.abs().amax(1) / torch.full((), 127.0, device="cuda")
        assert torch.equal(scale[r:r + step], want)
        bytes_ = torch.round(part / want[:, None]).clamp(-127, 127)
        assert torch.equal(q[r:r + step], bytes_.to(torch.int8))


# a wave to a row, and a workgroup to a row.  The bounds are those of the tests
# of log_probs: ln S is good to about 1e-6 of the mean |d| plus 2e-6
@pytest.mark.parametrize("cols,top", [(5, 3), (2100, 3), (2100, 0)])
def test_log_probs_more_rows_than_workgroups(cols, top):
    rows = GROUPS + 50_007
    x = windows(rows, cols, cols)
    given = torch.randint(-1, cols, (rows,), device="cuda", dtype=torch.int32,
                          generator=torch.Generator(device="cuda").manual_seed(1))
    r = ranking.log_probs(x, given, top=top)
    step = (1 << 25) // cols
    for i in range(0, rows, step):
        z, g = x[i:i + step].double(), given[i:i + step].long()
        lp = torch.log_softmax(z, 1)
        want = torch.where(g < 0, 0.0, lp.gather(1, g.clamp_min(0)[:, None])[:, 0])
        assert (r.log_prob[i:i + step] - want).abs().max() < 2e-5
        assert (r.entropy[i:i + step] + (lp.exp() * lp).sum(1)).abs().max() < 5e-5
        assert torch.equal(r.row_max[i:i + step], z.amax(1).float())
        if top:
            best = lp.topk(top, 1)
            assert (r.top_log_prob[i:i + step] - best.values).abs().max() < 2e-5
            # (equal scores may come in another order than topk's)
            at = r.top_item[i:i + step].long()
            assert torch.equal(z.gather(1, at), z.gather(1, best.indices))


def test_gradient_more_rows_than_workgroups():
    rows, cols = GROUPS + 50_007, 5
    x = windows(rows, cols, 9)
    given = torch.arange(rows, device="cuda", dtype=torch.int32) % cols
    gl = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    r = ranking.log_probs(x, given)
    got = ranking.log_probs_backward(x, given, r.row_max, r.row_sum, None, gl)
    want = -torch.softmax(x.double(), 1) * gl[:, None]
    want[torch.arange(rows, device="cuda"), given.long()] += gl
    # p is good to (4 D + 4 D1 + 62) 2^-24 of itself, D below 20: 1.4e-5
    p = torch.softmax(x.double(), 1)
    own = torch.nn.functional.one_hot(given.long(), cols)
    assert ((got - want).abs() <= 1.4e-5 * gl[:, None] * (p + own) + 2.0 ** -126).all()


# the table's 120 slots that travel with a kernel, and the batches of an upload:
# dense gradients take one slot, others two
@pytest.mark.parametrize("dense,strided", [(119, 0), (120, 0), (121, 0), (240, 0), (241, 0), (118, 1),
                                           (119, 1), (119, 3), (120, 1), (0, 60), (0, 61), (0, 70),
                                           (1, 121), (239, 2), (500, 11)])
def test_clip_table_batches(dense, strided):
    g = torch.Generator().manual_seed(dense * 1000 + strided)
    wide = torch.randn(23, 9 * max(strided, 1) + 2, generator=g)
    flat = torch.randn(sum(range(1, dense + 1)) + 9000, generator=g)

    def parts(flat, wide):
        sizes = list(range(1, dense + 1))
        got = list(flat[:sum(sizes)].split(sizes)) if dense else []
        got.insert(dense // 2, flat[sum(sizes):])  # one of more than a chunk
        for i in range(strided):
            got.insert((3 * i + 1) % (len(got) + 1), wide[:, 9 * i:9 * i + 8])
        return got

    fc, wc = flat.cuda(), wide.cuda()
    before = parts(flat, wide)
    norm = sum(p.double().square().sum() for p in before).sqrt().item()
    got = ranking.clip_grad_norm(parts(fc, wc), 1.0)
    assert abs(got.item() - norm) <= 2.0 ** -22 * norm
    for p, h in zip(before, parts(fc, wc)):
        want = p.double() / norm
        assert ((h.cpu().double() - want).abs() <= 2.0 ** -21 * want.abs()).all()
    between = torch.ones(wide.shape[1], dtype=torch.bool)
    for i in range(strided):
        between[9 * i:9 * i + 8] = False
    assert torch.equal(wc.cpu()[:, between], wide[:, between])
