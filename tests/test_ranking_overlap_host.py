"""Outputs that share memory with an input, refused at the C boundary (every
call here is refused: no address is used)."""
import pytest

from paper_2304_13724_amd import bgmf

A = 1 << 20
F32, F16, I8 = 0, 2, 3


def refused(call, *args):
    with pytest.raises(bgmf.BgmfError, match="shares memory") as e:
        call(*args)
    assert e.value.code == bgmf.BGMF_E_ARG


# 4 x 100 scores at A, 400 or more bytes apart; every other input far away
@pytest.mark.parametrize("stride,out,out_stride", [
    (100, A + 4, 100), (100, A - 4, 100), (100, A + 1596, 100), (100, A - 1596, 100),
    (150, A + 396, 150), (150, A + 204, 150), (150, A + 400, 250), (0, A + 396, 100)])
def test_gradient_and_scores(stride, out, out_stride):
    refused(bgmf.bgmf_log_probs_grad, A, F32, 4, 100, stride, 0, 0, 2 * A, 1.0, 3 * A, 4 * A, 5 * A,
            6 * A, 7 * A, out, out_stride, 0)


@pytest.mark.parametrize("which", range(7))
def test_gradient_and_other_inputs(which):
    """excluded, given, row_max, row_sum, entropy and both gradients."""
    at = [(2 + i) * A for i in range(7)]
    at[which] = 9 * A + 8
    excluded, given, row_max, row_sum, entropy, g_log_prob, g_entropy = at
    refused(bgmf.bgmf_log_probs_grad, A, F16, 4, 100, 100, excluded, 100, given, 1.0, row_max,
            row_sum, entropy, g_log_prob, g_entropy, 9 * A, 100, 0)


@pytest.mark.parametrize("q,scale", [(A, 5 * A), (A + 511, 5 * A), (A - 127, 5 * A),
                                     (4 * A, A + 8), (4 * A, 4 * A + 4)])
def test_quantize_rows(q, scale):
    refused(bgmf.bgmf_quantize_rows, A, F32, 2, 64, 64, q, 64, scale, 0)


@pytest.mark.parametrize("out", [A, A + 1020, A - 796, 2 * A, 2 * A - 796, 2 * A + 3196, 3 * A + 196])
def test_quantized_scores(out):
    """4 x 50 scores; 4 users at A, 50 items at 2 A, their scales at 3 A."""
    refused(bgmf.bgmf_quantized_scores, A, F32, 4, 64, 64, 0, 2 * A, 50, 64, 3 * A, out, F32, 50,
            8 * A, 1 << 40, 0)
