"""The 4-bit product of users in tiles of 64 that end where the laid-out users end."""
import pytest

from paper_2304_13724_amd import ranking

import torch

from mx_values import GRID

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [20, 64])
@pytest.mark.parametrize("rows", [193, 256, 449, 512, 705, 768])
def test_users_up_to_the_last_tile(rows, k):
    """Values of the grid times 1, 2 and 4: every partial sum is exact in fp32."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    grid = torch.from_numpy(GRID).float().cuda()
    for items in (129, 1_000, 128 * (254 // ((rows + 127) // 128))):
        x, v = (grid[torch.randint(0, 8, (n, k), generator=g, device="cuda")]
                * 2.0 ** (torch.arange(n, device="cuda") % 3)[:, None] for n in (rows, items))
        want = (x.double() @ v.double().t()).float()
        w, b = ranking.quantize_rows_mx4(v)
        q, a = ranking.quantize_rows_mx4(x)
        assert torch.equal(ranking.dequantize_rows_mx4(q, a, k), x)
        assert torch.equal(ranking.mx4_scores(x, w, b), want)
        assert torch.equal(ranking.mx4_scores(q, w, b, a), want)
