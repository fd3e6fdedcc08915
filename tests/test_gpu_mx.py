"""Rows in 4 bits with block scales: bytes equal to the definition's, and the
product of two such matrices, exact where its sums are."""
import numpy as np
import pytest

from paper_2304_13724_amd import bgmf, ranking

import torch

from mx_values import GRID, blocks_of, draw, quantized, values

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def check_rows(x, on=None):
    q, scale = ranking.quantize_rows_mx4(x.cuda() if on is None else on)
    want_q, want_s = quantized(x)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
    return q, scale


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 7), (5, 32), (17, 64), (2, 100), (33, 128),
                                    (4, 255), (3, 256), (9, 1000), (2, 4096), (1, 20001),
                                    (1000, 33), (70, 520)])
def test_quantize_rows(dtype, rows, k):
    x = draw(rows, k, TYPES[dtype], rows + k)
    q, scale = check_rows(x)
    want = torch.from_numpy(values(q.cpu().numpy(), scale.cpu().numpy()))
    for out in TYPES.values():
        got = ranking.dequantize_rows_mx4(q, scale, k, dtype=out)
        assert torch.equal(got.cpu(), want[:, :k].to(out)) and got.shape == (rows, k)
    assert torch.equal(ranking.dequantize_rows_mx4(q, scale).cpu().double(), want)


def special_rows():
    x = draw(24, 96, torch.float32, 1)
    x[0] = 0.0
    x[1, 7] = float("nan")
    x[2, 95] = float("inf")
    x[3, 40] = -float("inf")
    x[4] = 0.0
    x[4, 33] = -3.0
    x[5] = 1e-45
    x[6] = torch.finfo(torch.float32).max
    x[7] = 2e-38 * torch.randn(96, generator=torch.Generator().manual_seed(3))
    x[8] = 3e-42 * torch.arange(96)
    x[9] = -0.0
    x[10] = torch.arange(96) / 8 - 6  # ties
    x[11] = (torch.arange(96) / 8 - 6) * 2.0 ** -120
    x[12] = (torch.arange(96) / 8 - 6) * 2.0 ** -130
    x[13] = (torch.arange(96) / 8 - 6) * 2.0 ** 124
    x[14] = torch.linspace(4.0, 8.0, 96)  # past 6 X: the largest value
    x[15] = torch.nextafter(torch.arange(96) / 8 - 6, torch.tensor(9.0))
    x[16] = torch.nextafter(torch.arange(96) / 8 - 6, torch.tensor(-9.0))
    for i in range(17, 24):  # the edges of the scale's range, and of powers of two
        x[i] = torch.nextafter(torch.tensor(2.0 ** (i - 20)), torch.tensor(float(i > 20) * 99))
        x[i, ::3] = 2.0 ** (-124 - i % 4)
    return x


def test_quantize_special_rows():
    x = special_rows()
    q, scale = check_rows(x)
    want = torch.from_numpy(values(q.cpu().numpy(), scale.cpu().numpy())).float()
    got = ranking.dequantize_rows_mx4(q, scale).cpu()
    assert torch.equal(got.nan_to_num(7.5), want.nan_to_num(7.5))
    for t in (torch.bfloat16, torch.float16):
        check_rows(x.to(t))


def test_every_byte_and_scale():
    """All 16 values at all 256 scales, there and (as bytes) from values to bytes."""
    scale = torch.arange(256, dtype=torch.uint8)[:, None].contiguous()
    q = torch.arange(256, dtype=torch.uint8).repeat(1, 1).expand(256, 256)[:, ::16].contiguous()
    q = (q | torch.arange(16, dtype=torch.uint8)).contiguous()
    want = values(q.numpy(), scale.numpy())
    got = ranking.dequantize_rows_mx4(q.cuda(), scale.cuda()).cpu().double().numpy()
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(got, want.astype(np.float32).astype(np.float64))


def test_quantize_strides():
    flat = draw(1, 3 + 6 * 77, torch.float16, 2)[0]
    x, on = flat[3:].view(6, 77)[:, :61], flat.cuda()[3:].view(6, 77)[:, :61]
    check_rows(x, on)
    one = draw(1, 45, torch.float32, 4)
    check_rows(one.expand(9, 45), one.cuda().expand(9, 45))


# --- the product -----------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 5, 3), (2, 17, 16), (1, 1000, 64), (3, 333, 64), (16, 129, 64),
         (17, 100, 65), (31, 257, 50), (33, 64, 200), (64, 1000, 128), (65, 999, 127),
         (128, 128, 128), (129, 257, 129), (130, 131, 1000), (200, 300, 2047), (256, 512, 1024),
         (1, 4099, 4096), (5, 70, 20001), (300, 1025, 64), (513, 770, 320), (1, 20011, 100),
         (1, 70_001, 64), (4, 300_001, 33), (1030, 1200, 200), (64, 40_001, 96), (20, 3000, 2500),
         (600, 2100, 1500)]


def exact_rows(rows, k, seed):
    """Values of the grid with scale 1 in every block: sums are exact in fp32."""
    g = torch.Generator().manual_seed(seed)
    x = torch.from_numpy(GRID)[torch.randint(0, 8, (rows, k), generator=g)].float()
    x *= torch.randint(0, 2, (rows, k), generator=g) * 2 - 1
    x[:, ::32] = 4.0
    return x


@pytest.mark.parametrize("rows,items,k", SIZES)
def test_product_exact(rows, items, k):
    """Multiples of 1/4 below 2^22 in every partial sum (k <= 20,001 of 36): whatever the
    order of the sums, fp32 holds them."""
    x, v = exact_rows(rows, k, rows), exact_rows(items, k, items + 1)
    want = (x.double() @ v.double().t()).float()
    w, b = ranking.quantize_rows_mx4(v.cuda())
    q, a = ranking.quantize_rows_mx4(x.cuda())
    assert torch.equal(ranking.mx4_scores(x.cuda(), w, b).cpu(), want)
    assert torch.equal(ranking.mx4_scores(q, w, b, a).cpu(), want)
    for t in (torch.bfloat16, torch.float16):
        assert torch.equal(ranking.mx4_scores(x.cuda().to(t), w, b, dtype=t).cpu(), want.to(t))


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("rows,items,k", SIZES)
def test_product(out, rows, items, k):
    """Each of at most 32 ceil(k / 32) additions is off by at most a step (2^-23, rounded
    whichever way) of the sum of magnitudes, and the result by half a step of its type."""
    x, v = draw(rows, k, torch.float32, rows), draw(items, k, torch.float32, items)
    w, b = (torch.from_numpy(t) for t in quantized(v))
    q, a = (torch.from_numpy(t) for t in quantized(x))
    xv, vv = torch.from_numpy(values(q.numpy(), a.numpy())), torch.from_numpy(
        values(w.numpy(), b.numpy()))
    want = xv @ vv.t()
    size = xv.abs() @ vv.abs().t()
    t = TYPES[out]
    err = 32 * blocks_of(k) * 2.0 ** -23 * size
    tol = err + torch.finfo(t).eps / 2 * (want.abs() + err) + (2.0 ** -25 if out == "f16" else 0)
    c = ranking.Catalogue(v.cuda(), bits=4)
    want_here = want.to(t).double() if out == "f16" else want  # past 65,504: infinite
    for got in (ranking.mx4_scores(x.cuda(), w.cuda(), b.cuda(), dtype=t),
                ranking.mx4_scores(q.cuda(), w.cuda(), b.cuda(), a.cuda(), dtype=t),
                c.scores(x.cuda(), t)):
        g = got.cpu().double()
        both = torch.isfinite(want_here) & torch.isfinite(g)
        assert ((g - want).abs()[both] <= tol[both]).all()
        edge = want.abs() > 65_000 if out == "f16" else torch.zeros_like(both)
        assert (both | edge).all()


# more tiles than workgroups at a time, of 128 x 128 and of 128 x 64, in one and in
# several steps, and long rows in tiles of 256 x 256 with rows, items and blocks left over
LARGE = [(3000, 5003, 64), (2999, 5000, 40), (3001, 4999, 200), (2100, 6001, 300),
         (60, 140_003, 64), (64, 140_000, 200), (2900, 2801, 2048), (2817, 2900, 2100),
         (3000, 3001, 2300), (300, 18_000, 4090), (257, 16_500, 2049)]


@pytest.mark.parametrize("rows,items,k", LARGE)
def test_product_exact_large(rows, items, k):
    g = torch.Generator(device="cuda").manual_seed(rows)
    grid = torch.from_numpy(GRID).float().cuda()

    def draw_exact(n):
        x = grid[torch.randint(0, 8, (n, k), generator=g, device="cuda")]
        x = x * (torch.randint(0, 2, (n, k), generator=g, device="cuda") * 2 - 1)
        x[:, ::32] = 4.0
        return x * 2.0 ** (torch.arange(n, device="cuda") % 3)[:, None]  # scales of its own

    x, v = draw_exact(rows), draw_exact(items)
    want = (x.double() @ v.double().t()).float()
    w, b = ranking.quantize_rows_mx4(v)
    q, a = ranking.quantize_rows_mx4(x)
    assert torch.equal(ranking.mx4_scores(x, w, b), want)
    assert torch.equal(ranking.mx4_scores(q, w, b, a), want)
    # items apart, with NaN scales and other bytes between them
    blocks = blocks_of(k)
    wide = torch.full((items, 17 * blocks + 11), 255, dtype=torch.uint8, device="cuda")
    wide[:, 3:3 + 16 * blocks], wide[:, 7 + 16 * blocks:7 + 17 * blocks] = w, b
    got = ranking.mx4_scores(x.bfloat16(), wide[:, 3:3 + 16 * blocks],
                             wide[:, 7 + 16 * blocks:7 + 17 * blocks], dtype=torch.bfloat16)
    assert torch.equal(got, want.bfloat16())
    # NaN blocks at the ends: their own rows and items alone
    x[rows - 1, k - 1], v[0, 0], v[items - 1, k - 1] = float("nan"), float("inf"), float("nan")
    got = ranking.mx4_scores(x, *ranking.quantize_rows_mx4(v))
    want[rows - 1], want[:, 0], want[:, items - 1] = float("nan"), float("nan"), float("nan")
    assert torch.equal(got.nan_to_num(7.5), want.nan_to_num(7.5))


@pytest.mark.parametrize("rows,items,k", [(1, 70, 64), (3, 300, 96), (40, 500, 70), (200, 300, 64),
                                          (300, 600, 600), (5, 9000, 128)])
def test_product_blocks_that_stand_for_nan(rows, items, k):
    """They make their user's or item's scores NaN, and no others: not through the
    padding of a row, the next row's bytes or a neighbour in the tile."""
    x, v = draw(rows, k, torch.float32, 1), draw(items, k, torch.float32, 2)
    clean = ranking.mx4_scores(x.cuda(), *ranking.quantize_rows_mx4(v.cuda()))
    bad_r, bad_j = sorted({0, rows // 2, rows - 1}), sorted({1, items // 3, items - 2, items - 1})
    for i, r in enumerate(bad_r):
        x[r, (i * 37 + 3) % k] = float("nan")
    for i, j in enumerate(bad_j):
        v[j, (i * 31 + k - 1) % k] = float("inf")
    q, a = ranking.quantize_rows_mx4(x.cuda())
    got = [ranking.mx4_scores(x.cuda(), *ranking.quantize_rows_mx4(v.cuda())),
           ranking.mx4_scores(q, *ranking.quantize_rows_mx4(v.cuda()), a)]
    for g in got:
        want = clean.clone()
        want[bad_r] = float("nan")
        want[:, bad_j] = float("nan")
        assert torch.equal(g.nan_to_num(7.0), want.nan_to_num(7.0))


def test_product_zero_rows_and_wide_scales():
    x, v = draw(40, 96, torch.float32, 1), draw(300, 96, torch.float32, 2)
    x[3] = 0.0
    v[7] = 0.0
    x[5] = 2.0 ** -100
    v[9] = 2.0 ** 90
    v[10] = 2.0 ** 120
    x[6] = 2.0 ** 120
    got = ranking.Catalogue(v.cuda(), bits=4).scores(x.cuda()).cpu()
    assert (got[3] == 0).all() and (got[:, 7] == 0).all()
    assert got[5, 9] == 96 * 2.0 ** -10 and got[6, 10] == float("inf")


def test_product_strides_and_output():
    k, rows, items = 100, 21, 333
    x, v = draw(rows, k, torch.float32, 1), draw(items, k, torch.float32, 2)
    w, b = ranking.quantize_rows_mx4(v.cuda())
    want = ranking.mx4_scores(x.cuda(), w, b)
    wide = torch.full((items, 64 + 21), 255, dtype=torch.uint8, device="cuda")
    wide[:, 3:67], wide[:, 70:74] = w, b
    assert torch.equal(ranking.mx4_scores(x.cuda(), wide[:, 3:67], wide[:, 70:74]), want)
    q, a = ranking.quantize_rows_mx4(x.cuda())
    long = torch.full((rows, 64 + 13), 255, dtype=torch.uint8, device="cuda")
    long[:, 5:69], long[:, 71:75] = q, a
    out = torch.full((rows, items + 9), 7.0, device="cuda")
    got = ranking.mx4_scores(long[:, 5:69], w, b, long[:, 71:75], out=out[:, 2:items + 2])
    assert torch.equal(got, want) and got.data_ptr() == out[:, 2:].data_ptr()
    assert (out[:, :2] == 7).all() and (out[:, items + 2:] == 7).all()
    # one item many times over, one user many times over
    assert torch.equal(ranking.mx4_scores(x[:1].cuda().expand(50, k), w, b), want[:1].expand(50, items))
    got = ranking.mx4_scores(x.cuda(), w[:1].expand(70, 64), b[:1].expand(70, 4))
    assert torch.equal(got, want[:, :1].expand(rows, 70))


@pytest.mark.parametrize("rows,items,k", [(70_000, 3, 40), (2_100_000, 1, 33), (3, 1, 4096),
                                          (0, 5, 64), (5, 0, 64)])
def test_product_extremes(rows, items, k):
    x = exact_rows(max(min(rows, 1000), 1), k, 1).repeat(max(rows // 1000, 1), 1)[:rows].cuda()
    v = exact_rows(max(items, 1), k, 2)[:items].cuda()
    w, b = ranking.quantize_rows_mx4(v)
    got = ranking.mx4_scores(x, w, b)
    assert torch.equal(got, x @ v.t()) and got.shape == (rows, items)


def test_items_past_32_bits_of_bytes():
    """More than 2^32 bytes of items: the last ones' scores are their own."""
    items, blocks = 270_000, 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.randint(0, 256, (items, blocks * 16), generator=g, device="cuda", dtype=torch.uint8)
    b = torch.full((items, blocks), 127, device="cuda", dtype=torch.uint8)
    x = exact_rows(2, blocks * 32, 3).cuda()
    got = ranking.mx4_scores(x, w, b)
    at = [0, 1, 134_217, 134_218, items - 2, items - 1]
    part = ranking.dequantize_rows_mx4(w[at].contiguous(), b[at].contiguous())
    assert torch.equal(got[:, at], (x.double() @ part.double().t()).float())


def test_captured_with_other_inputs_on_replay():
    x = draw(40, 64, torch.float32, 1).cuda()
    c = ranking.Catalogue(draw(3000, 64, torch.float32, 2).cuda(), bits=4)
    c.scores(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.scores(x, torch.bfloat16)
    for seed in range(4):
        x.copy_(draw(40, 64, torch.float32, 10 + seed))
        graph.replay()
        assert torch.equal(got, c.scores(x, torch.bfloat16))
        torch.cuda.synchronize()


def test_on_another_stream():
    x = draw(100, 64, torch.float32, 1).cuda()
    c = ranking.Catalogue(draw(3000, 64, torch.float32, 2).cuda(), bits=4)
    want = c.scores(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [c.scores(x) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_scores_have_no_derivative_and_say_so():
    users = draw(3, 64, torch.float32, 1).cuda().requires_grad_()
    c = ranking.Catalogue(draw(7, 64, torch.float32, 2).cuda(), bits=4)
    s = c.scores(users)
    assert s.requires_grad and torch.equal(s.detach(), c.scores(users.detach()))
    with pytest.raises(RuntimeError, match="derivative"):
        s.sum().backward()
    with pytest.raises(ValueError, match="out"):
        ranking.mx4_scores(users, c.items, c.scale, out=torch.empty(3, 7, device="cuda"))


def test_refusals_on_the_gpu():
    x = draw(4, 64, torch.float32, 1).cuda()
    q, s = ranking.quantize_rows_mx4(x)
    for call in (lambda: ranking.mx4_scores(x[:, :20], q, s), lambda: ranking.mx4_scores(q, q, s),
                 lambda: ranking.mx4_scores(x, q, s, s), lambda: ranking.mx4_scores(x, q, s[:3]),
                 lambda: ranking.mx4_scores(x, q[:, :16], s), lambda: ranking.mx4_scores(x, x, s),
                 lambda: ranking.mx4_scores(x, q, s, dtype=torch.int8),
                 lambda: ranking.mx4_scores(x.double(), q, s),
                 lambda: ranking.mx4_scores(x, q.cpu(), s.cpu()),
                 lambda: ranking.mx4_scores(x, q, s, out=torch.empty(4, 5, device="cuda")),
                 lambda: ranking.dequantize_rows_mx4(q, s, 32),
                 lambda: ranking.dequantize_rows_mx4(q, s, 65),
                 lambda: ranking.dequantize_rows_mx4(q, s[:, :1]),
                 lambda: ranking.quantize_rows_mx4(x.t()[:, :3]),
                 lambda: ranking.quantize_rows_mx4(x[:, :0]),
                 lambda: ranking.Catalogue(x, bits=5)):
        with pytest.raises(ValueError):
            call()
    flat = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    items = flat[:128].view(4, 32)
    out = flat[64:128].view(torch.float32).view(4, 4)
    with pytest.raises(bgmf.BgmfError, match="shares memory"):
        ranking.mx4_scores(x, items, s, out=out)
