"""Ranking with learned factors, on PyTorch tensors.

Answers: quantise the item factors once (``Catalogue``), score users over the
whole catalogue, and take log probabilities, entropy and the best items
(``log_probs``).  Training on choices in place of ratings: ``log_probs`` is
differentiable, and ``clip_grad_norm`` bounds the gradients' global norm.

Every function checks its tensors (ValueError for those that do not fit,
BgmfError for what the library refuses), runs the library's kernels
(include/bgmf.h) on the current stream of the tensors' device and returns
without waiting.  There is no fallback: importing this module raises if
_ranking.so is missing.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Sequence, Tuple

from . import bgmf  # before torch: one HIP runtime in the process

import torch

from . import _ranking

TOP_MAX = bgmf.BGMF_TOP_MAX

_TYPES = {torch.float32: bgmf.BGMF_TYPE_F32, torch.bfloat16: bgmf.BGMF_TYPE_BF16,
          torch.float16: bgmf.BGMF_TYPE_F16}


class LogProbs(NamedTuple):
    """Results of ``log_probs``, one entry (or row of ``top``) per row of scores."""
    log_prob: torch.Tensor      # of the given item
    entropy: torch.Tensor
    top_item: torch.Tensor      # int32 [rows, top], -1 where fewer items are left
    top_log_prob: torch.Tensor  # [rows, top]
    row_max: torch.Tensor       # the largest score, and the sum of exp((x - max) / temperature):
    row_sum: torch.Tensor       # what log_probs_backward needs


# the current stream's address without a Stream object, where PyTorch offers it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        return 0  # which the call refuses
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _checked(result):
    if type(result) is int:  # a status code
        bgmf._check(None, result)
    return result


def _in_graph(*tensors) -> bool:
    """Whether autograd would want the derivative of a call on these tensors."""
    if torch.is_grad_enabled():
        for t in tensors:
            if isinstance(t, torch.Tensor) and t.requires_grad:
                return True
    return False


class _NoDerivative(torch.autograd.Function):
    """Results of a call that has no derivative: a backward pass that reaches
    them raises, as with PyTorch's functions that have none."""
    @staticmethod
    def forward(ctx, name, call, *tensors):
        ctx.name = name
        results = call()
        for r in results if isinstance(results, tuple) else (results,):
            if not r.is_floating_point():
                ctx.mark_non_differentiable(r)
        return results

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{ctx.name} has no derivative: call it under torch.no_grad(), or on "
                           "detached tensors")


def _without_derivative(name, call, out, *tensors):
    if not _in_graph(*tensors):
        return _checked(call())
    if out is not None:
        raise ValueError(f"{name}: out takes no part in a graph, and one of the tensors requires "
                         "grad")
    return _NoDerivative.apply(name, lambda: _checked(call()), *tensors)


# --- log probabilities ----------------------------------------------------------

def _forward(scores, given, top, temperature, excluded) -> LogProbs:
    return LogProbs(*_checked(_ranking.log_probs(scores, given, top, temperature, excluded,
                                                 _stream(scores))))


def log_probs_backward(scores: torch.Tensor, given: Optional[torch.Tensor], row_max: torch.Tensor,
                       row_sum: torch.Tensor, entropy: Optional[torch.Tensor],
                       grad_log_prob: Optional[torch.Tensor],
                       grad_entropy: Optional[torch.Tensor] = None, *, temperature: float = 1.0,
                       excluded: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient with respect to the scores of a loss whose gradients with
    respect to ``log_prob`` and ``entropy`` are given (None: zero), from the
    results of ``log_probs``.  ``out`` may be the scores themselves.  Has no
    derivative of its own."""
    return _without_derivative(
        "log_probs_backward", lambda: _ranking.log_probs_backward(
            scores, given, row_max, row_sum, entropy, grad_log_prob, grad_entropy, temperature,
            excluded, out, _stream(scores)),
        out, scores, row_max, row_sum, entropy, grad_log_prob, grad_entropy)


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, scores, given, top, temperature, excluded):
        r = _forward(scores, given, top, temperature, excluded)
        ctx.save_for_backward(scores, given, excluded, r.row_max, r.row_sum, r.entropy)
        ctx.temperature = temperature
        ctx.mark_non_differentiable(r.top_item, r.top_log_prob, r.row_max, r.row_sum)
        ctx.set_materialize_grads(False)
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_log_prob, g_entropy, *_):
        scores, given, excluded, row_max, row_sum, entropy = ctx.saved_tensors
        if g_log_prob is None and g_entropy is None:
            return None, None, None, None, None
        g = [None if x is None else x.resolve_neg().contiguous() for x in (g_log_prob, g_entropy)]
        if given is None:
            g[0] = None
        grad = log_probs_backward(scores, given, row_max, row_sum, entropy, g[0], g[1],
                                  temperature=ctx.temperature, excluded=excluded)
        return grad, None, None, None, None


def log_probs(scores: torch.Tensor, given: Optional[torch.Tensor] = None, *, top: int = 0,
              temperature: float = 1.0, excluded: Optional[torch.Tensor] = None) -> LogProbs:
    """Softmax of every row of ``scores`` (float32, bfloat16 or float16) at a
    temperature, without its probabilities being stored: the log probability
    of the row's ``given`` item (int32; -1: none, log_prob 0), the entropy and
    the ``top`` items with their log probabilities, ties to the lower item.
    ``excluded`` (bool or uint8, the shape of the scores): items to leave out.
    Differentiable with respect to the scores through log_prob and entropy.
    include/bgmf.h says what empty rows, infinities and NaN give."""
    if torch.is_grad_enabled() and isinstance(scores, torch.Tensor) and scores.requires_grad:
        return LogProbs(*_LogProbs.apply(scores, given, top, temperature, excluded))
    return _forward(scores, given, top, temperature, excluded)


# --- scores in 8-bit integers ---------------------------------------------------

def quantize_rows(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows in 8-bit integers: (q int8, scale float32) with x ~ q * scale,
    scale the row's largest magnitude / 127.  The rows of q start on 16-byte
    boundaries (q is a view of a wider tensor where k needs it).  Has no
    derivative."""
    return _without_derivative("quantize_rows", lambda: _ranking.quantize_rows(x, _stream(x)),
                               None, x)


def quantized_scores(rows: torch.Tensor, items: torch.Tensor, item_scale: torch.Tensor,
                     row_scale: Optional[torch.Tensor] = None, *,
                     dtype: torch.dtype = torch.float32,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scores rows . items^T with both in 8-bit integers, times row_scale and
    item_scale, as ``dtype``.  ``rows``: int8 with ``row_scale``, or float32,
    bfloat16 or float16 without it, quantised in the call as by
    ``quantize_rows``.  ``items``: int8 with ``item_scale``.  Has no
    derivative."""
    code = _TYPES.get(dtype)
    if code is None:
        raise ValueError(f"dtype must be float32, bfloat16 or float16: {dtype}")
    return _without_derivative(
        "quantized_scores", lambda: _ranking.quantized_scores(
            rows, items, item_scale, row_scale, code, out, _stream(rows)),
        out, rows, item_scale, row_scale)


class Catalogue:
    """Item factors (m x k, such as a model's V) in 8-bit integers, laid out
    once, to score and rank them for users."""

    def __init__(self, items: torch.Tensor):
        self.items, self.scale = quantize_rows(items)

    def scores(self, users: torch.Tensor, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """Scores of user factors (rows x k) over all items."""
        return quantized_scores(users, self.items, self.scale, dtype=dtype)

    def rank(self, users: torch.Tensor, given: Optional[torch.Tensor] = None, *, top: int = 10,
             temperature: float = 1.0, excluded: Optional[torch.Tensor] = None) -> LogProbs:
        """The best items for each user, with the log probability of a given
        item and the entropy, as by ``log_probs``, but without a derivative
        with respect to the users: the scores are in 8-bit integers."""
        return log_probs(self.scores(users), given, top=top, temperature=temperature,
                         excluded=excluded)


# --- clipping -------------------------------------------------------------------

def clip_grad_norm(grads: Sequence[torch.Tensor], max_norm: float,
                   out: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
    """Scales gradients (float32, bfloat16 or float16, mixed or not) so that
    their global norm is at most max_norm, in place or into ``out``; returns
    the norm before (a float32 tensor on the GPU).  A norm that is not finite
    leaves the gradients as they are.  Each must be contiguous, or 2-D with
    adjacent row elements, and none may share written memory with another (the
    same gradient twice, say): BgmfError.  The results are in no graph."""
    grads = list(grads)
    return _checked(_ranking.clip_grad_norm(grads, max_norm, None if out is None else list(out),
                                            _stream(grads[0]) if grads else 0))
