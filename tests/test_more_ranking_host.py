"""Refusals of the 4-bit, policy and dropout calls at the C boundary, before
anything reaches a device (the addresses are never used), and the generator's
known answers."""
import pytest

from paper_2304_13724_amd import bgmf

from philox import block
from test_ranking_host import A, BF16, F32, I8, refused

MX4 = 4


def test_known_answers_of_the_generator():
    """Those published with it for ten rounds of Philox4x32."""
    for counter, key, want in (
            ([0] * 4, (0, 0), [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
            ([0xFFFFFFFF] * 4, (0xFFFFFFFF,) * 2,
             [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD])):
        assert [int(v) for v in block(counter, key)] == want


@pytest.mark.parametrize("change", [
    dict(type=I8), dict(type=MX4), dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(k=1 << 30),
    dict(x=0), dict(x=A + 1), dict(stride=-1), dict(q=0), dict(q_stride=47), dict(scale=0),
    dict(scale_stride=2), dict(q=A), dict(scale=2 * A + 5)])
def test_quantize_rows_mx(change):
    refused(bgmf.bgmf_quantize_rows_mx, (A, BF16, 4, 70, 70, 2 * A, 48, 3 * A, 3, 0),
            ("x", "type", "rows", "k", "stride", "q", "q_stride", "scale", "scale_stride",
             "stream"), change)


@pytest.mark.parametrize("change", [
    dict(out_type=I8), dict(rows=-1), dict(k=0), dict(q=0), dict(q_stride=-1), dict(scale=0),
    dict(scale_stride=-1), dict(out=0), dict(out=3 * A + 1), dict(out_stride=69), dict(out=A)])
def test_dequantize_rows_mx(change):
    refused(bgmf.bgmf_dequantize_rows_mx, (A, 48, 2 * A, 3, 4, 70, 3 * A, F32, 70, 0),
            ("q", "q_stride", "scale", "scale_stride", "rows", "k", "out", "out_type",
             "out_stride", "stream"), change)


PRODUCT = ("x", "type", "rows", "k", "stride", "row_scale", "row_scale_stride", "items",
           "item_count", "items_stride", "item_scale", "item_scale_stride", "out", "out_type",
           "out_stride", "ws", "ws_bytes", "stream")


def product_args():
    return (A, F32, 4, 64, 64, 0, 0, 2 * A, 50, 32, 3 * A, 2, 4 * A, F32, 50, 5 * A, 1 << 40, 0)


@pytest.mark.parametrize("change", [
    dict(type=I8), dict(type=5), dict(out_type=MX4), dict(rows=-1), dict(rows=1 << 31),
    dict(item_count=-1), dict(item_count=1 << 31), dict(k=0), dict(k=1 << 20), dict(x=0),
    dict(x=A + 2), dict(stride=-1), dict(items=0), dict(items_stride=-1), dict(item_scale=0),
    dict(item_scale_stride=-1), dict(out=0), dict(out=4 * A + 2), dict(out_stride=49),
    dict(row_scale=A), dict(type=MX4), dict(type=MX4, row_scale=A, row_scale_stride=-1),
    dict(ws=0), dict(ws=A + 128), dict(out=A), dict(out=2 * A), dict(out=3 * A)])
def test_mx_scores(change):
    refused(bgmf.bgmf_mx_scores, product_args(), PRODUCT, change)


POLICY = ("scores", "type", "rows", "cols", "stride", "reference", "reference_stride", "excluded",
          "ex_stride", "given", "advantage", "old", "reference_log_prob", "t", "clip_low",
          "clip_high", "kl_weight", "loss", "log_prob", "kl", "state", "g_loss", "out",
          "out_stride", "ws", "ws_bytes", "stream")


def policy_args():
    return (A, F32, 4, 100, 100, 2 * A, 100, 0, 0, 3 * A, 4 * A, 5 * A, 0, 1.0, 0.2, 0.2, 0.1,
            6 * A, 7 * A, 8 * A, 0, 0, 9 * A, 100, 10 * A, 1 << 40, 0)


@pytest.mark.parametrize("change", [
    dict(type=I8), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(rows=1 << 31),
    dict(cols=1 << 31), dict(scores=0), dict(scores=A + 2), dict(stride=-1), dict(stride=1 << 60),
    dict(reference=2 * A + 1), dict(reference_stride=-1), dict(excluded=A, ex_stride=-5),
    dict(given=0), dict(advantage=0), dict(old=0), dict(reference_log_prob=A), dict(t=0.0),
    dict(t=-1.0), dict(t=float("nan")), dict(t=float("inf")), dict(t=1e-45), dict(clip_low=-0.1),
    dict(clip_low=1.5), dict(clip_low=float("nan")), dict(clip_high=-0.1),
    dict(clip_high=float("nan")), dict(kl_weight=float("nan")), dict(kl_weight=float("inf")),
    dict(out=9 * A + 2), dict(out_stride=99), dict(out=A, out_stride=101),
    dict(out=2 * A, out_stride=101), dict(out=A + 4), dict(out=3 * A), dict(out=4 * A),
    dict(out=5 * A), dict(out=6 * A), dict(out=7 * A), dict(out=8 * A),
    dict(out=11 * A, state=11 * A + 64), dict(out=11 * A, g_loss=11 * A)])
def test_policy_loss(change):
    refused(bgmf.bgmf_policy_loss, policy_args(), POLICY, change)


@pytest.mark.parametrize("change", [dict(ws=0), dict(ws=A + 8)])
def test_policy_loss_of_rows_that_need_a_workspace(change):
    args = {**dict(zip(POLICY, policy_args())), "cols": 100_000, "stride": 100_000,
            "reference_stride": 100_000, "out": 1 << 40, "out_stride": 100_000, "scores": 1 << 41,
            "reference": 1 << 42}
    refused(bgmf.bgmf_policy_loss, args.values(), POLICY, change)


@pytest.mark.parametrize("change", [
    dict(type=I8), dict(rows=-1), dict(scores=0), dict(stride=-1), dict(out=0), dict(out=9 * A + 3),
    dict(out_stride=99), dict(state=0), dict(given=0), dict(t=0.0), dict(kl_weight=float("nan")),
    dict(out=A, out_stride=101), dict(out=4 * A), dict(out=3 * A)])
def test_policy_loss_grad(change):
    args = (A, F32, 4, 100, 100, 2 * A, 100, 0, 0, 3 * A, 1.0, 0.1, 4 * A, 0, 9 * A, 100, 0)
    refused(bgmf.bgmf_policy_loss_grad, args,
            ("scores", "type", "rows", "cols", "stride", "reference", "reference_stride",
             "excluded", "ex_stride", "given", "t", "kl_weight", "state", "g_loss", "out",
             "out_stride", "stream"), change)


@pytest.mark.parametrize("change", [
    dict(type=I8), dict(rows=-1), dict(rows=1 << 31), dict(cols=-1), dict(cols=1 << 40), dict(x=0),
    dict(x=A + 1), dict(stride=-1), dict(p=-0.1), dict(p=1.5), dict(p=float("nan")),
    dict(more=A + 4), dict(out=0), dict(out=2 * A + 2), dict(out_stride=99),
    dict(out=A, out_stride=101), dict(out=A + 4), dict(more=2 * A + 8)])
def test_dropout(change):
    refused(bgmf.bgmf_dropout, (A, F32, 4, 100, 100, 0.5, 1, 2, 0, 2 * A, 100, 0),
            ("x", "type", "rows", "cols", "stride", "p", "seed", "offset", "more", "out",
             "out_stride", "stream"), change)


def test_workspaces():
    need = bgmf.bgmf_mx_scores_workspace(4, 50, 64, F32)
    args = dict(zip(PRODUCT, product_args()))
    refused(bgmf.bgmf_mx_scores, {**args, "ws_bytes": need - 1}.values(), PRODUCT, {},
            bgmf.BGMF_E_BUDGET)
    for rows, cols in ((4, 100), (1, 5_000_000)):
        need = bgmf.bgmf_policy_loss_workspace(rows, cols)
        args = {**dict(zip(POLICY, policy_args())), "rows": rows, "cols": cols, "stride": cols,
                "reference_stride": cols, "out": 1 << 40, "out_stride": cols, "reference": 1 << 41}
        refused(bgmf.bgmf_policy_loss, {**args, "ws_bytes": need - 1}.values(), POLICY, {},
                bgmf.BGMF_E_BUDGET)
    assert bgmf.bgmf_mx_scores_workspace(0, 10, 64, F32) == 0
    assert bgmf.bgmf_mx_scores_workspace(5, 10, -1, F32) == 0
    assert bgmf.bgmf_policy_loss_workspace(0, 10) == 0
    assert bgmf.bgmf_policy_loss_workspace(5, -1) == 0


def test_tensors_that_do_not_fit_are_refused_without_a_gpu():
    import torch
    from paper_2304_13724_amd import ranking
    x, given = torch.zeros(4, 32), torch.zeros(4, dtype=torch.int32)
    q, s = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)
    for call in (lambda: ranking.quantize_rows_mx4(x), lambda: ranking.quantize_rows_mx4(None),
                 lambda: ranking.dequantize_rows_mx4(q, s), lambda: ranking.mx4_scores(x, q, s),
                 lambda: ranking.mx4_scores(x.requires_grad_(), q, s),
                 lambda: ranking.Catalogue(x, bits=4), lambda: ranking.Catalogue(x, bits=2),
                 lambda: ranking.mx4_scores(x, q, s, dtype=torch.int8),
                 lambda: ranking.policy_loss(x.detach(), given, x[:, 0], x[:, 0]),
                 lambda: ranking.policy_loss([1.0], given, x[:, 0], x[:, 0]),
                 lambda: ranking.policy_loss_and_grad(x, given, x[:, 0], x[:, 0]),
                 lambda: ranking.dropout(x, 0.5, 1), lambda: ranking.dropout(None, 0.5, 1),
                 lambda: ranking.dropout(x, 0.5, 1, None)):
        with pytest.raises(ValueError):
            call()
