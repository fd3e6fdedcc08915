"""Outputs beside their inputs in one allocation: columns of a wider matrix are
valid, shared elements are refused."""
import pytest

from paper_2304_13724_amd import bgmf, ranking

import torch

pytestmark = pytest.mark.gpu


def test_columns_beside_the_scores():
    wide = torch.randn(5, 210, generator=torch.Generator().manual_seed(1)).cuda()
    x, out = wide[:, :100], wide[:, 105:205]
    given = torch.tensor([1, 2, 3, 4, -1]).int().cuda()
    r = ranking.log_probs(x.contiguous(), given)
    one = torch.ones(5, device="cuda")
    args = (given, r.row_max, r.row_sum, r.entropy, one, one)
    want = ranking.log_probs_backward(x.contiguous(), *args)
    ranking.log_probs_backward(x, *args, out=out)
    assert torch.equal(out, want)
    for shared in (wide[:, 1:101], wide[:, 99:199], wide.flatten()[30:530].view(5, 100)):
        with pytest.raises(bgmf.BgmfError, match="shares memory"):
            ranking.log_probs_backward(x, *args, out=shared)


def test_scores_beside_the_users():
    wide = torch.randn(6, 64 + 30, generator=torch.Generator().manual_seed(2)).cuda()
    c = ranking.Catalogue(torch.randn(30, 64, generator=torch.Generator().manual_seed(3)).cuda())
    users = wide[:, :64]
    want = c.scores(users)
    ranking.quantized_scores(users, c.items, c.scale, out=wide[:, 64:])
    assert torch.equal(wide[:, 64:], want)
    for shared in (wide[:, 63:93], wide[:, :30]):
        with pytest.raises(bgmf.BgmfError, match="shares memory"):
            ranking.quantized_scores(users, c.items, c.scale, out=shared)
