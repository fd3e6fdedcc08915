"""Users whose factors are not as wide as the catalogue's items."""
import pytest

from paper_2304_13724_amd import ranking

import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("k,users", [(60, 64), (64, 60), (1, 32), (33, 64), (50, 49)])
def test_other_widths_are_refused(bits, k, users):
    """Within a block of 4-bit columns too."""
    g = torch.Generator().manual_seed(k)
    c = ranking.Catalogue(torch.randn(9, k, generator=g).cuda(), bits=bits)
    u = torch.randn(3, users, generator=g).cuda()
    for call in (c.scores, c.rank):
        with pytest.raises(ValueError, match="columns"):
            call(u)
    assert c.scores(torch.randn(3, k, generator=g).cuda()).shape == (3, 9)
