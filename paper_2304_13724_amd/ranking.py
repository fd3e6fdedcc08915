"""Ranking with learned factors, on PyTorch tensors.

Answers: quantise the item factors once (``Catalogue``, in 8 or 4 bits), score
users over the whole catalogue, and take log probabilities, entropy and the best
items (``log_probs``).  Training on choices in place of ratings: ``log_probs`` is
differentiable, ``dropout`` drops elements of the factors, and ``clip_grad_norm``
bounds the gradients' global norm.  Training on what users did with the answers:
``policy_loss``.

Every function checks its tensors (ValueError for those that do not fit, an
``out`` that is part of a graph among them; BgmfError for what the library
refuses), runs the library's kernels (include/bgmf.h) on the current stream of
the tensors' device and returns without waiting.  There is no fallback:
importing this module raises if _ranking.so is missing.

Calls can be captured into a graph, backward passes too, as long as no autograd
graph from before the capture still holds the same leaves (PyTorch adds up a
leaf's gradient on the stream of the first).
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Sequence, Tuple

from . import bgmf  # before torch: one HIP runtime in the process

import torch

from . import _ranking

TOP_MAX = bgmf.BGMF_TOP_MAX

_TYPES = {torch.float32: bgmf.BGMF_TYPE_F32, torch.bfloat16: bgmf.BGMF_TYPE_BF16,
          torch.float16: bgmf.BGMF_TYPE_F16}


def _type_code(dtype) -> int:
    code = _TYPES.get(dtype)
    if code is None:
        raise ValueError(f"dtype must be float32, bfloat16 or float16: {dtype}")
    return code


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
_ranking.set_stream_function(
    _raw_stream or (lambda device: torch.cuda.current_stream(device).cuda_stream))


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
    code = _type_code(dtype)
    return _without_derivative(
        "quantized_scores", lambda: _ranking.quantized_scores(
            rows, items, item_scale, row_scale, code, out, _stream(rows)),
        out, rows, item_scale, row_scale)


# --- scores in 4 bits -----------------------------------------------------------

def quantize_rows_mx4(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows in 4 bits with a power-of-two scale for each block of 32 columns
    (the MXFP4 format): (q uint8 [rows, 16 blocks], scale uint8 [rows,
    blocks]), the last block filled up with zeros.  include/bgmf.h has the
    rounding and the layout.  The results are bytes, in no graph."""
    return _checked(_ranking.quantize_rows_mx(x, _stream(x)))


def dequantize_rows_mx4(q: torch.Tensor, scale: torch.Tensor, k: Optional[int] = None, *,
                        dtype: torch.dtype = torch.float32,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values that rows in 4 bits stand for, [rows, k] as ``dtype``.
    ``k``: columns, None for whole blocks."""
    return _checked(_ranking.dequantize_rows_mx(q, scale, k, _type_code(dtype), out, _stream(q)))


def mx4_scores(rows: torch.Tensor, items: torch.Tensor, item_scale: torch.Tensor,
               row_scale: Optional[torch.Tensor] = None, *, dtype: torch.dtype = torch.float32,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scores rows . items^T with both in 4 bits, summed in float32, as
    ``dtype``.  ``rows``: uint8 with ``row_scale``, or float32, bfloat16 or
    float16 without it, quantised in the call as by ``quantize_rows_mx4``.
    ``items``: uint8 with ``item_scale``; their rows are whole blocks, and rows
    that end within the last one stand for zeros there.  Has no derivative."""
    code = _type_code(dtype)
    return _without_derivative(
        "mx4_scores", lambda: _ranking.mx_scores(rows, items, item_scale, row_scale, code, out,
                                                 _stream(rows)),
        out, rows)


class Catalogue:
    """Item factors (m x k, such as a model's V) in 8-bit integers, or with
    ``bits=4`` in 4 bits with block scales (half the memory and the traffic, a
    coarser score), laid out once, to score and rank them for users."""

    def __init__(self, items: torch.Tensor, bits: int = 8):
        if bits not in (4, 8):
            raise ValueError(f"bits must be 8 or 4: {bits}")
        self.bits = bits
        self.items, self.scale = quantize_rows(items) if bits == 8 else quantize_rows_mx4(items)
        self.k = items.shape[1]  # (4-bit items know their blocks alone)

    def scores(self, users: torch.Tensor, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """Scores of user factors (rows x k) over all items."""
        if self.bits == 4:
            if isinstance(users, torch.Tensor) and users.shape[1:] != (self.k,):
                raise ValueError(f"users must be rows of {self.k} columns, as the items are: "
                                 f"{tuple(users.shape)}")
            return mx4_scores(users, self.items, self.scale, dtype=dtype)
        return quantized_scores(users, self.items, self.scale, dtype=dtype)

    def rank(self, users: torch.Tensor, given: Optional[torch.Tensor] = None, *, top: int = 10,
             temperature: float = 1.0, excluded: Optional[torch.Tensor] = None) -> LogProbs:
        """The best items for each user, with the log probability of a given
        item and the entropy, as by ``log_probs``, but without a derivative
        with respect to the users: the scores are in 8-bit integers (or 4
        bits)."""
        return log_probs(self.scores(users), given, top=top, temperature=temperature,
                         excluded=excluded)


# --- learning from what users did with the answers ------------------------------

class PolicyLoss(NamedTuple):
    """Results of ``policy_loss``, one entry per row of scores."""
    loss: torch.Tensor
    log_prob: torch.Tensor  # of the shown item
    kl: torch.Tensor        # divergence from the reference, 0 without one


def _only_scores(name, *tensors):
    if _in_graph(*tensors):
        raise ValueError(f"{name} has a derivative with respect to the scores alone, and another "
                         "of its tensors requires grad (call .detach())")


def policy_loss(scores: torch.Tensor, given: torch.Tensor, advantage: torch.Tensor,
                old_log_prob: torch.Tensor, *, reference: Optional[torch.Tensor] = None,
                reference_log_prob: Optional[torch.Tensor] = None, kl_weight: float = 0.0,
                clip_low: float = 0.2, clip_high: float = 0.2, temperature: float = 1.0,
                excluded: Optional[torch.Tensor] = None) -> PolicyLoss:
    """Clipped policy loss of the items that were shown, row by row:
    -min(rho A, clip(rho, 1 - clip_low, 1 + clip_high) A) + kl_weight kl with
    rho = exp(log_prob - old_log_prob), without the softmax's probabilities
    being stored.  ``scores`` (float32, bfloat16 or float16): the policy's, over
    the catalogue; ``given`` (int32): the shown item, -1 for a row that fills
    the batch up; ``advantage`` A and ``old_log_prob`` (float32): its log
    probability when it was shown.  ``reference``: another policy's scores, for
    the whole divergence, or ``reference_log_prob`` (float32): its log
    probabilities of the shown items, for an estimate.  Differentiable with
    respect to the scores through ``loss``.  include/bgmf.h says what empty
    rows, infinities and NaN give."""
    _only_scores("policy_loss", advantage, old_log_prob, reference, reference_log_prob)
    return PolicyLoss(*_checked(_ranking.policy_loss(
        scores, given, advantage, old_log_prob, reference, reference_log_prob, kl_weight, clip_low,
        clip_high, temperature, excluded, None, None, _stream(scores))))


def policy_loss_and_grad(scores: torch.Tensor, given: torch.Tensor, advantage: torch.Tensor,
                         old_log_prob: torch.Tensor, weight: Optional[torch.Tensor] = None, *,
                         reference: Optional[torch.Tensor] = None,
                         reference_log_prob: Optional[torch.Tensor] = None,
                         kl_weight: float = 0.0, clip_low: float = 0.2, clip_high: float = 0.2,
                         temperature: float = 1.0, excluded: Optional[torch.Tensor] = None,
                         out: Optional[torch.Tensor] = None
                         ) -> Tuple[PolicyLoss, torch.Tensor]:
    """The results of ``policy_loss`` and the gradient of sum(weight * loss)
    with respect to the scores (``weight`` float32, one entry per row; None:
    ones), which are read once for both where a row fits a workgroup's
    registers.  ``out`` may be the scores themselves, in a graph too.  For a loop that passes
    the gradient on itself (``logits.backward(grad)``): the results are in no
    graph."""
    _only_scores("policy_loss_and_grad", advantage, old_log_prob, reference, reference_log_prob,
                 weight)
    loss, log_prob, kl, grad = _checked(_ranking.policy_loss_and_grad(
        scores, given, advantage, old_log_prob, reference, reference_log_prob, kl_weight, clip_low,
        clip_high, temperature, excluded, weight, out, _stream(scores)))
    return PolicyLoss(loss, log_prob, kl), grad


# --- dropout --------------------------------------------------------------------

def dropout(x: torch.Tensor, p: float, seed: int, offset=0, *,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Elements of ``x`` (float32, bfloat16 or float16; contiguous, or 2-D with
    adjacent row elements) set to 0 with probability ``p``, the others times
    1 / (1 - p).  Which ones depends on ``seed``, ``offset`` (in [0, 2^64)) and
    the element's place alone (include/bgmf.h has the generator), so no mask is
    stored: the backward pass draws it again.  A call uses the offsets from
    ``offset`` up to ``offset + ceil(x.numel() / 4)``.  ``offset`` may be an
    int64 tensor of one element on the GPU, read when the kernel runs: a
    captured graph that adds to it drops other elements on each replay (it must
    not change between a forward and its backward pass, which raises).  ``out``
    may be ``x`` itself."""
    return _checked(_ranking.dropout(x, p, seed, offset, out, _stream(x)))


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
