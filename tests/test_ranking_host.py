"""Refusals of the ranking calls at the C boundary, before anything reaches a
device (the addresses are never used), and their workspace sizes."""
import ctypes

import pytest

from paper_2304_13724_amd import bgmf

A = 1 << 20  # an aligned address that no call may touch
F32, BF16, F16, I8 = 0, 1, 2, 3


def refused(call, args, names, change, code=bgmf.BGMF_E_ARG):
    args = dict(zip(names, args))
    assert set(change) <= set(args)
    with pytest.raises(bgmf.BgmfError) as e:
        call(*{**args, **change}.values())
    assert e.value.code == code
    assert call.__name__ in str(e.value)


LOG_PROBS = ("scores", "type", "rows", "cols", "stride", "excluded", "ex_stride", "given", "t",
             "top", "log_prob", "entropy", "row_max", "row_sum", "top_item", "top_log_prob", "ws",
             "ws_bytes", "stream")


@pytest.mark.parametrize("change", [
    dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(rows=1 << 31),
    dict(cols=1 << 31), dict(stride=-1), dict(stride=1 << 60), dict(scores=0), dict(scores=A + 2),
    dict(excluded=A, ex_stride=-5), dict(t=0.0), dict(t=-1.0), dict(t=float("nan")),
    dict(t=float("inf")), dict(t=1e-45), dict(top=-1), dict(top=129), dict(given=0),
    dict(top=3, top_item=0), dict(top=3, top_log_prob=0)])
def test_log_probs(change):
    args = (A, F32, 4, 100, 100, 0, 0, A, 1.0, 2, A, A, A, A, A, A, A, 1 << 40, 0)
    refused(bgmf.bgmf_log_probs, args, LOG_PROBS, change)


GRAD = ("scores", "type", "rows", "cols", "stride", "excluded", "ex_stride", "given", "t",
        "row_max", "row_sum", "entropy", "g_log_prob", "g_entropy", "out", "out_stride", "stream")


@pytest.mark.parametrize("change", [
    dict(type=3), dict(rows=-1), dict(scores=0), dict(stride=-1), dict(out=0), dict(out=A + 3),
    dict(out_stride=99), dict(row_max=0), dict(row_sum=0), dict(given=0), dict(entropy=0),
    dict(t=0.0), dict(out=A, out_stride=101)])
def test_log_probs_grad(change):
    args = (A, F32, 4, 100, 100, 0, 0, A, 1.0, A, A, A, A, A, 2 * A, 100, 0)
    refused(bgmf.bgmf_log_probs_grad, args, GRAD, change)


@pytest.mark.parametrize("change", [
    dict(type=I8), dict(rows=-1), dict(k=0), dict(k=1 << 31), dict(x=0), dict(x=A + 1),
    dict(stride=-1), dict(q=0), dict(q_stride=63), dict(scale=0)])
def test_quantize_rows(change):
    refused(bgmf.bgmf_quantize_rows, (A, BF16, 4, 64, 64, A, 64, A, 0),
            ("x", "type", "rows", "k", "stride", "q", "q_stride", "scale", "stream"), change)


PRODUCT = ("x", "type", "rows", "k", "stride", "row_scale", "items", "item_count", "items_stride",
           "item_scale", "out", "out_type", "out_stride", "ws", "ws_bytes", "stream")


@pytest.mark.parametrize("change", [
    dict(type=4), dict(out_type=I8), dict(rows=-1), dict(item_count=-1), dict(rows=1 << 31),
    dict(item_count=1 << 31), dict(k=0), dict(k=131072), dict(x=0), dict(x=A + 2),
    dict(stride=-1), dict(items=0), dict(items_stride=-1), dict(item_scale=0), dict(out=0),
    dict(out=A + 2), dict(out_stride=49), dict(row_scale=A), dict(type=I8), dict(ws=0),
    dict(ws=A + 128)])
def test_quantized_scores(change):
    args = (A, F32, 4, 64, 64, 0, A, 50, 64, A, A, F32, 50, A, 1 << 40, 0)
    refused(bgmf.bgmf_quantized_scores, args, PRODUCT, change)


def test_workspaces_too_small():
    need = bgmf.bgmf_quantized_scores_workspace(4, 50, 64, F32)
    args = (A, F32, 4, 64, 64, 0, A, 50, 64, A, A, F32, 50, A, need - 1, 0)
    refused(bgmf.bgmf_quantized_scores, args, PRODUCT, {}, bgmf.BGMF_E_BUDGET)
    need = bgmf.bgmf_clip_grad_norm_workspace(1)
    grads = (bgmf.Grad * 1)(bgmf.Grad(A, A, 1, 5, 5, 5, F32))
    refused(bgmf.bgmf_clip_grad_norm, (grads, 1, 1.0, A, A, need - 1, 0), CLIP, {},
            bgmf.BGMF_E_BUDGET)
    need = bgmf.bgmf_log_probs_workspace(1, 5_000_000, 10)
    if need:
        args = (A, F32, 1, 5_000_000, 5_000_000, 0, 0, A, 1.0, 10, A, A, A, A, A, A, A, need - 1, 0)
        refused(bgmf.bgmf_log_probs, args, LOG_PROBS, {}, bgmf.BGMF_E_BUDGET)


CLIP = ("grads", "count", "max_norm", "norm", "ws", "ws_bytes", "stream")


@pytest.mark.parametrize("change", [
    dict(count=-1), dict(count=1 << 31), dict(grads=None), dict(max_norm=-1.0),
    dict(max_norm=float("nan")), dict(norm=0), dict(ws=0), dict(ws=A + 8)])
def test_clip_arguments(change):
    grads = (bgmf.Grad * 2)(*[bgmf.Grad(A, A, 2, 5, 5, 5, F32)] * 2)
    refused(bgmf.bgmf_clip_grad_norm, (grads, 2, 1.0, A, A, 1 << 40, 0), CLIP, change)


@pytest.mark.parametrize("grad", [
    (A, A, 2, 5, 5, 5, I8), (0, A, 2, 5, 5, 5, F32), (A, 0, 2, 5, 5, 5, F32),
    (A + 1, A, 2, 5, 5, 5, F32), (A, A + 2, 2, 5, 5, 5, F32), (A, A, -1, 5, 5, 5, F32),
    (A, A, 2, -5, 5, 5, F32), (A, A, 2, 5, 4, 5, F32), (A, 2 * A, 2, 5, 5, 4, F32),
    (A, A, 2, 5, 5, 6, F32), (A, A, 1 << 40, 1 << 40, 1 << 40, 1 << 40, F32)])
def test_clip_gradients(grad):
    grads = (bgmf.Grad * 2)(bgmf.Grad(A, A, 2, 5, 5, 5, F32), bgmf.Grad(*grad))
    refused(bgmf.bgmf_clip_grad_norm, (grads, 2, 1.0, A, A, 1 << 40, 0), CLIP, {})
    assert "gradient 1" in bgmf.bgmf_last_error(None)


def test_the_table_entry_has_the_header_s_layout():
    assert ctypes.sizeof(bgmf.Grad) == 56 and bgmf.Grad.type.offset == 48


def test_workspace_sizes_of_degenerate_calls():
    assert bgmf.bgmf_log_probs_workspace(0, 10, 1) == 0
    assert bgmf.bgmf_log_probs_workspace(-1, 10, 1) == 0
    assert bgmf.bgmf_quantized_scores_workspace(0, 10, 64, F32) == 0
    assert bgmf.bgmf_quantized_scores_workspace(5, 10, -1, F32) == 0
    assert bgmf.bgmf_clip_grad_norm_workspace(-1) == 0


def test_tensors_that_do_not_fit_are_refused_without_a_gpu():
    import torch
    from paper_2304_13724_amd import ranking
    x = torch.zeros(4, 8)
    for call in (lambda: ranking.log_probs(x), lambda: ranking.log_probs([1.0, 2.0]),
                 lambda: ranking.log_probs(x.requires_grad_()),
                 lambda: ranking.log_probs_backward(x, None, x[0], x[0], None, None),
                 lambda: ranking.quantize_rows(x), lambda: ranking.quantize_rows(None),
                 lambda: ranking.Catalogue(x), lambda: ranking.quantized_scores(x, x, x[0]),
                 lambda: ranking.quantized_scores(x, x, x[0], dtype=torch.int8),
                 lambda: ranking.clip_grad_norm([], 1.0), lambda: ranking.clip_grad_norm([x], 1.0),
                 lambda: ranking.clip_grad_norm([None], 1.0)):
        with pytest.raises(ValueError):
            call()
