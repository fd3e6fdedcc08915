"""Rows in 8-bit integers and the product of two such matrices: integers and
products equal to the definition's, bit for bit."""
import numpy as np
import pytest

from paper_2304_13724_amd import bgmf, ranking

import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def quantized(x):
    """The definition, in numpy: both quotients rounded to fp32."""
    x = x.float().numpy()
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        bad = ~np.isfinite(x).all(1)
        scale = (np.abs(x).max(1) / np.float32(127)).astype(np.float32)
        q = np.rint(x / scale[:, None])
        q = np.clip(np.where((scale > 0)[:, None] & ~bad[:, None], q, 0), -127, 127)
        return np.nan_to_num(q).astype(np.int8), np.where(bad, np.float32(np.nan), scale)


def draw(rows, k, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, k, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))
    return x.to(TYPES[dtype])


def product(q, a, items, b, dtype):
    """float(sum) * a * b in fp32, rounded to the type; the sum exact in 64 bits
    (in doubles, exact below 2^53)."""
    total = torch.from_numpy(q.astype(np.float64)) @ torch.from_numpy(items.astype(np.float64)).t()
    out = total.float() * torch.from_numpy(a)[:, None] * torch.from_numpy(b)[None]
    return out.to(dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 7), (5, 16), (17, 64), (2, 100), (33, 128),
                                    (4, 255), (3, 256), (9, 1000), (2, 4096), (1, 20001)])
def test_quantize_rows(dtype, rows, k):
    x = draw(rows, k, dtype, rows + k)
    q, scale = ranking.quantize_rows(x.cuda())
    want_q, want_s = quantized(x)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
    assert q.stride(0) % 16 == 0 or rows == 1


def test_quantize_special_rows():
    x = draw(10, 300, "f32", 1)
    x[0] = 0.0
    x[1, 7] = float("nan")
    x[2, 299] = float("inf")
    x[3] = 0.0
    x[3, 5] = -3.0
    x[4] = 1e-45
    x[5] = torch.finfo(torch.float32).max
    x[6] = 2e-38 * torch.randn(300)
    x[7] = torch.arange(300) - 149.5  # ties
    x[8] = 3e-42
    x[9] = -0.0
    q, scale = ranking.quantize_rows(x.cuda())
    want_q, want_s = quantized(x)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)


def test_quantize_strides():
    flat = draw(1, 3 + 6 * 77, "f16", 2)[0]
    x, on = flat[3:].view(6, 77)[:, :61], flat.cuda()[3:].view(6, 77)[:, :61]
    q, scale = ranking.quantize_rows(on)
    want_q, want_s = quantized(x)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)


SIZES = [(1, 1, 1), (1, 5, 3), (2, 17, 16), (1, 1000, 64), (3, 333, 64), (16, 129, 64),
         (17, 100, 65), (31, 257, 50), (33, 64, 200), (64, 1000, 128), (65, 999, 127),
         (128, 128, 128), (129, 257, 129), (130, 131, 1000), (200, 300, 2047), (256, 512, 1024),
         (1, 4099, 4096), (5, 70, 20001), (300, 1025, 64), (513, 770, 320), (1, 20011, 100)]


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("rows,items,k", SIZES)
def test_product(out, rows, items, k):
    x, v = draw(rows, k, "f32", rows), draw(items, k, "f32", items)
    q, a = quantized(x)
    w, b = quantized(v)
    wc, bc = torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda()
    want = product(q, a, w, b, TYPES[out])
    got = ranking.quantized_scores(x.cuda(), wc, bc, dtype=TYPES[out])
    assert torch.equal(got.cpu(), want)
    got = ranking.quantized_scores(torch.from_numpy(q).cuda(), wc, bc, torch.from_numpy(a).cuda(),
                                   dtype=TYPES[out])
    assert torch.equal(got.cpu(), want)
    c = ranking.Catalogue(v.cuda())  # rows of 16-byte multiples
    assert torch.equal(c.scores(x.cuda(), TYPES[out]).cpu(), want)


# the kernels' other ways: tiles of 128 and 64 items and users, long k shared by
# the waves of a workgroup, less than 128 items or 16 bytes for many users
@pytest.mark.parametrize("rows,items,k", [
    (100, 20000, 72), (100, 20001, 64), (1030, 4100, 96), (1030, 4099, 201), (64, 4097, 64),
    (20, 300, 777), (64, 2000, 600), (33, 8200, 512), (17, 8193, 640), (200, 100, 64),
    (70, 127, 130), (5, 3, 5), (300, 2, 7), (40, 15, 1), (16, 33000, 520)])
def test_product_other_tiles(rows, items, k):
    x, v = draw(rows, k, "f32", rows + 1), draw(items, k, "f32", items + 1)
    q, a = quantized(x)
    w, b = quantized(v)
    want = product(q, a, w, b, torch.float32)
    wc, bc = torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda()
    assert torch.equal(ranking.quantized_scores(x.cuda(), wc, bc).cpu(), want)
    assert torch.equal(ranking.Catalogue(v.cuda()).scores(x.cuda()).cpu(), want)


def on_gpu(rows, items, k, seed, pad=0):
    """Bytes, scales and the product in doubles, all on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw8 = lambda n, wide: torch.randint(-127, 128, (n, wide), generator=g, device="cuda",  # noqa: E731
                                          dtype=torch.int8)
    q, w = draw8(rows, k), draw8(items, k + pad)[:, :k]
    a, b = (torch.rand(n, generator=g, device="cuda") for n in (rows, items))
    total = q.double() @ w.double().t()
    return q, a, w, b, total.float() * a[:, None] * b[None]


# many items: several tiles for each wave, the last ones overlapping, and items
# that the caches cannot hold
@pytest.mark.parametrize("rows,items,k,pad", [
    (1, 524_293, 64, 0), (1, 600_001, 50, 0), (16, 524_300, 48, 0), (3, 524_301, 128, 0),
    (2, 530_000, 100, 0), (1, 3_200_001, 64, 0), (2, 1_700_003, 128, 0), (1, 600_001, 50, 14),
    (40, 524_301, 64, 0)])
def test_product_many_items(rows, items, k, pad):
    q, a, w, b, want = on_gpu(rows, items, k, k + rows, pad)
    assert torch.equal(ranking.quantized_scores(q, w, b, a), want)
    # values whose bytes are q with scale a: the largest of each row is 127
    x = q.float()
    x[:, 0] = 127.0
    got = ranking.quantized_scores(x * a[:, None], w, b)
    r, s = ranking.quantize_rows(x * a[:, None])
    assert torch.equal(got, ranking.quantized_scores(r, w, b, s))


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("rows,items,k,pad", [
    (4096, 4096, 512, 0), (4000, 4099, 528, 0), (3841, 4111, 521, 0), (4096, 4352, 640, 0),
    (4000, 4200, 513, 3), (5000, 4100, 1000, 8), (4097, 4097, 1152, 16)])
def test_product_large_tiles(out, rows, items, k, pad):
    q, a, w, b, want = on_gpu(rows, items, k, k, pad)
    got = ranking.quantized_scores(q, w, b, a, dtype=TYPES[out])
    assert torch.equal(got, want.to(TYPES[out]))


def test_product_of_millions_of_users():
    """More users than a launch has blocks for."""
    q, a, w, b, want = on_gpu(65535 * 32 + 37, 20, 16, 1)
    assert torch.equal(ranking.quantized_scores(q, w, b, a), want)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_product_of_16_bit_rows(dtype):
    for rows, items, k in ((1, 500, 64), (40, 130, 200), (150, 260, 96)):
        x, v = draw(rows, k, dtype, rows), draw(items, k, dtype, items)
        q, a = quantized(x)
        w, b = quantized(v)
        c = ranking.Catalogue(v.cuda())
        assert torch.equal(c.scores(x.cuda()).cpu(), product(q, a, w, b, torch.float32))


@pytest.mark.parametrize("rows", [1, 7, 40, 200])
def test_product_strides(rows):
    """Row strides of every operand, at odd addresses; -128 is a valid byte; what
    lies between the rows is neither read into a sum nor written."""
    rng = np.random.default_rng(rows)
    items, k = 301, 77
    a = torch.from_numpy(rng.integers(-128, 128, 5 + rows * 83, dtype=np.int8))
    b = torch.from_numpy(rng.integers(-128, 128, 3 + items * 79, dtype=np.int8))
    sa, sb = (torch.from_numpy(rng.random(n, dtype=np.float32)) for n in (rows, items))
    view = lambda t, off, n, stride: t[off:].view(n, stride)[:, :k]  # noqa: E731
    out = torch.full((1 + rows * 311,), 7.0, device="cuda")
    to = out[1:].view(rows, 311)[:, :items]
    ranking.quantized_scores(view(a.cuda(), 5, rows, 83), view(b.cuda(), 3, items, 79), sb.cuda(),
                             sa.cuda(), out=to)
    want = product(view(a, 5, rows, 83).numpy(), sa.numpy(), view(b, 3, items, 79).numpy(),
                   sb.numpy(), torch.float32)
    assert torch.equal(to.cpu(), want)
    assert (out[1:].view(rows, 311)[:, items:] == 7.0).all() and out[0].item() == 7.0


def test_product_broadcast_rows():
    g = torch.Generator().manual_seed(9)
    q = torch.randint(-127, 128, (1, 64), dtype=torch.int8, generator=g)
    w = torch.randint(-127, 128, (90, 64), dtype=torch.int8, generator=g)
    one = torch.ones(90)
    got = ranking.quantized_scores(q.cuda().expand(20, -1), w.cuda(), one.cuda(),
                                   torch.ones(20).cuda())
    want = product(q.numpy().repeat(20, 0), np.ones(20, np.float32), w.numpy(), one.numpy(),
                   torch.float32)
    assert torch.equal(got.cpu(), want)


def test_longest_sums_stay_exact():
    k = bgmf.BGMF_PRODUCT_K_MAX
    for rows in (1, 20):
        a = torch.full((rows, k), -128, dtype=torch.int8).cuda()
        b = torch.full((3, k), -128, dtype=torch.int8).cuda()
        got = ranking.quantized_scores(a, b, torch.ones(3).cuda(), torch.ones(rows).cuda())
        assert (got == float(np.float32(k * 128 * 128))).all()


def test_nan_rows_stay_nan_and_zero_rows_zero():
    x = draw(5, 64, "f32", 3)
    x[1, 3] = float("nan")
    x[2] = 0.0
    c = ranking.Catalogue(draw(40, 64, "f32", 4).cuda())
    s = c.scores(x.cuda())
    assert torch.isnan(s[1]).all() and not s[2].any() and torch.isfinite(s[[0, 3, 4]]).all()


def test_offsets_beyond_32_bits():
    """Item rows and output rows further apart than 2^32 bytes."""
    x = draw(3, 64, "f32", 5)
    v = draw(2, 64, "f32", 6)
    q, a = quantized(x)
    w, b = quantized(v)
    far = (1 << 32) + 64
    items = torch.empty(far + 64, dtype=torch.int8, device="cuda").as_strided((2, 64), (far, 1))
    items.copy_(torch.from_numpy(w).cuda())
    wide = (1 << 31) + 16
    out = torch.empty(2 * wide + 2, dtype=torch.float16, device="cuda").as_strided((3, 2), (wide, 1))
    ranking.quantized_scores(x.cuda(), items, torch.from_numpy(b).cuda(), dtype=torch.float16,
                             out=out)
    assert torch.equal(out.cpu(), product(q, a, w, b, torch.float16))


def test_no_rows_and_no_items():
    c = ranking.Catalogue(torch.empty(0, 64).cuda())
    assert c.scores(torch.ones(3, 64).cuda()).shape == (3, 0)
    c = ranking.Catalogue(torch.ones(5, 64).cuda())
    assert c.scores(torch.empty(0, 64).cuda()).shape == (0, 5)


def test_graph_replays_and_streams():
    x = draw(20, 96, "f32", 7).cuda()
    c = ranking.Catalogue(draw(500, 96, "f32", 8).cuda())
    c.scores(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = c.scores(x)
    for seed in range(3):
        x.copy_(draw(20, 96, "f32", 50 + seed).cuda())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, c.scores(x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = c.scores(x)
    side.synchronize()
    assert torch.equal(y, z)


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    w = torch.zeros(9, 64, dtype=torch.int8, device="cuda")
    b = torch.zeros(9, device="cuda")
    with pytest.raises(ValueError):
        ranking.quantize_rows(torch.zeros(3, 0, device="cuda"))
    with pytest.raises(ValueError):
        ranking.quantize_rows(x.t())
    with pytest.raises(ValueError):
        ranking.quantize_rows(w)
    for args in ((x[:, :63], w, b), (x, w.float(), b), (x, w, b[:8]), (x, w, b.half()),
                 (x, w, b, torch.zeros(4, device="cuda")), (x.to(torch.int8), w, b), (x.cpu(), w, b),
                 (x.double(), w, b), (x, w.t(), b)):
        with pytest.raises(ValueError):
            ranking.quantized_scores(*args)
    with pytest.raises(ValueError):
        ranking.quantized_scores(x, w, b, dtype=torch.float64)
    with pytest.raises(ValueError):
        ranking.quantized_scores(x, w, b, out=torch.zeros(4, 8, device="cuda"))
    k = bgmf.BGMF_PRODUCT_K_MAX + 1
    with pytest.raises(bgmf.BgmfError) as e:
        ranking.quantized_scores(torch.zeros(1, k, device="cuda"),
                                 torch.zeros(1, k, dtype=torch.int8, device="cuda"), b[:1])
    assert e.value.code == bgmf.BGMF_E_ARG


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,items,k", [
    (17, 128, 64), (17, 129, 1), (64, 18000, 64), (65, 300, 50), (100, 20000, 48), (513, 700, 33),
    (130, 20001, 64), (1000, 130, 16), (30, 4097, 17), (700, 30000, 64)])
def test_values_quantised_within_the_product(dtype, rows, items, k):
    """The same scores whether the product or quantize_rows made the bytes."""
    x = draw(rows, k, dtype, rows)
    if rows > 20:
        x[3], x[5, 0] = 0.0, float("nan")
    v = draw(items, k, "f32", items)
    c = ranking.Catalogue(v.cuda())
    r, s = ranking.quantize_rows(x.cuda())
    one = c.scores(x.cuda())
    two = ranking.quantized_scores(r, c.items, c.scale, s)
    assert torch.equal(one.nan_to_num(7.0), two.nan_to_num(7.0))
    q, a = quantized(x)
    np.testing.assert_array_equal(r.cpu().numpy(), q)
    np.testing.assert_array_equal(s.cpu().numpy(), a)
    w, b = quantized(v)
    want = product(q, a, w, b, torch.float32)
    assert torch.equal(one.cpu().nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("rows", [1, 3, 20, 70, 300])
@pytest.mark.parametrize("k", [3, 8, 16, 50, 64, 600])
def test_broadcast_and_overlapping_items(rows, k):
    """Item rows with a stride of 0 (one item's bytes, fewer than a load's 16
    among them) and of 1."""
    x = draw(rows, k, "f32", rows + k)
    q, a = quantized(x)
    line = torch.randint(-127, 128, (400 + k,), dtype=torch.int8,
                         generator=torch.Generator().manual_seed(k))
    for stride in (0, 1):
        # the last item's last byte is the last of its memory
        flat = line[:k + 299 * stride].clone()
        b = torch.rand(300, generator=torch.Generator().manual_seed(1))
        items = flat.as_strided((300, k), (stride, 1))
        on = flat.cuda().as_strided((300, k), (stride, 1))
        want = product(q, a, items.contiguous().numpy(), b.numpy(), torch.float32)
        assert torch.equal(ranking.quantized_scores(x.cuda(), on, b.cuda()).cpu(), want)
        got = ranking.quantized_scores(torch.from_numpy(q).cuda(), on, b.cuda(),
                                       torch.from_numpy(a).cuda())
        assert torch.equal(got.cpu(), want)
