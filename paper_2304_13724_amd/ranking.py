"""Ranking with learned factors, on PyTorch tensors.

Answers: quantise the item factors once (``Catalogue``), score users over the
whole catalogue, and take log probabilities, entropy and the best items
(``log_probs``).  Training on choices in place of ratings: ``log_probs`` is
differentiable, and ``clip_grad_norm`` bounds the gradients' global norm.

Every function checks its tensors, runs the library's kernels
(include/bgmf.h) on the current stream of the tensors' device and returns
without waiting; there is no fallback.
"""
from __future__ import annotations

import contextlib
from typing import NamedTuple, Optional, Sequence, Tuple

from . import bgmf  # before torch: one HIP runtime in the process

import numpy as np
import torch

TOP_MAX = bgmf.BGMF_TOP_MAX

_TYPES = {torch.float32: bgmf.BGMF_TYPE_F32, torch.bfloat16: bgmf.BGMF_TYPE_BF16,
          torch.float16: bgmf.BGMF_TYPE_F16}
_BYTES = {torch.int8: bgmf.BGMF_TYPE_I8}
_ROW_TYPES = {**_TYPES, **_BYTES}


class LogProbs(NamedTuple):
    """Results of ``log_probs``, one entry (or row of ``top``) per row of scores."""
    log_prob: torch.Tensor      # of the given item
    entropy: torch.Tensor
    top_item: torch.Tensor      # int32 [rows, top], -1 where fewer items are left
    top_log_prob: torch.Tensor  # [rows, top]
    row_max: torch.Tensor       # the largest score, and the sum of exp((x - max) / temperature):
    row_sum: torch.Tensor       # what log_probs_backward needs


# --- checks -------------------------------------------------------------------

def _matrix(t: torch.Tensor, name: str, types) -> int:
    """Checks a 2-D device tensor with adjacent row elements; its type's code."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    code = types.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} has type {t.dtype}; one of "
                         f"{', '.join(str(x) for x in types)} is needed")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent (call .contiguous())")
    return code


def _vector(t: torch.Tensor, name: str, like: torch.Tensor, count: int, dtype) -> None:
    if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.shape[0] != count:
        raise ValueError(f"{name} must be a 1-D tensor of length {count}")
    if t.dtype != dtype or t.get_device() != like.get_device():
        raise ValueError(f"{name} must be {dtype} on {like.device}")
    if count > 1 and t.stride(0) != 1:
        raise ValueError(f"{name} must be contiguous")


def _output(t: torch.Tensor, name: str, like: torch.Tensor, shape, dtype) -> None:
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != like.device:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)} on {like.device}")
    if (shape[1] > 1 and t.stride(1) != 1) or (shape[0] > 1 and t.stride(0) < shape[1]):
        raise ValueError(f"{name}: rows must not overlap and their elements must be adjacent")


def _excluded(t: Optional[torch.Tensor], like: torch.Tensor) -> Tuple[int, int]:
    if t is None:
        return 0, 0
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.bool, torch.uint8):
        raise ValueError("excluded must be a bool or uint8 tensor")
    if t.shape != like.shape or t.device != like.device:
        raise ValueError("excluded must have the shape and the device of the scores")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("excluded: the elements of a row must be adjacent (call .contiguous())")
    return t.data_ptr(), t.stride(0)


_HERE = contextlib.nullcontext()
# the current stream's address without a Stream object, where PyTorch offers it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on(t: torch.Tensor):
    """The context in which a launch for t's device is made."""
    at = t.get_device()
    return _HERE if at == torch.cuda.current_device() else torch.cuda.device(at)


def _stream(t: torch.Tensor) -> int:
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _workspace(nbytes: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device) if nbytes else None


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


# --- log probabilities ----------------------------------------------------------

def _forward(scores, given, top, temperature, excluded) -> LogProbs:
    code = _matrix(scores, "scores", _TYPES)
    rows, cols = scores.shape
    if given is not None:
        _vector(given, "given", scores, rows, torch.int32)
    ex, ex_stride = _excluded(excluded, scores)
    top = int(top)
    if not 0 <= top <= TOP_MAX:
        raise ValueError(f"top must be in [0, {TOP_MAX}]")
    dev = scores.device
    log_prob, entropy, row_max, row_sum = torch.empty((4, rows), device=dev).unbind(0)
    top_item = torch.empty((rows, top), dtype=torch.int32, device=dev)
    top_log_prob = torch.empty((rows, top), device=dev)
    nbytes = bgmf.bgmf_log_probs_workspace(rows, cols, top)
    ws = _workspace(nbytes, scores)
    with _on(scores):
        bgmf.bgmf_log_probs(
            scores.data_ptr(), code, rows, cols, scores.stride(0), ex, ex_stride, _ptr(given),
            temperature, top, log_prob.data_ptr() if given is not None else 0,
            entropy.data_ptr(), row_max.data_ptr(), row_sum.data_ptr(), _ptr(top_item),
            _ptr(top_log_prob), _ptr(ws), nbytes, _stream(scores))
    if given is None:
        log_prob.zero_()
    return LogProbs(log_prob, entropy, top_item, top_log_prob, row_max, row_sum)


def log_probs_backward(scores: torch.Tensor, given: Optional[torch.Tensor], row_max: torch.Tensor,
                       row_sum: torch.Tensor, entropy: Optional[torch.Tensor],
                       grad_log_prob: Optional[torch.Tensor],
                       grad_entropy: Optional[torch.Tensor] = None, *, temperature: float = 1.0,
                       excluded: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient with respect to the scores of a loss whose gradients with
    respect to ``log_prob`` and ``entropy`` are given (None: zero), from the
    results of ``log_probs``.  ``out`` may be the scores themselves."""
    code = _matrix(scores, "scores", _TYPES)
    rows, cols = scores.shape
    _vector(row_max, "row_max", scores, rows, torch.float32)
    _vector(row_sum, "row_sum", scores, rows, torch.float32)
    for t, name in ((entropy, "entropy"), (grad_log_prob, "grad_log_prob"),
                    (grad_entropy, "grad_entropy")):
        if t is not None:
            _vector(t, name, scores, rows, torch.float32)
    if given is not None:
        _vector(given, "given", scores, rows, torch.int32)
    ex, ex_stride = _excluded(excluded, scores)
    if out is None:
        out = torch.empty((rows, cols), dtype=scores.dtype, device=scores.device)
    else:
        _output(out, "out", scores, (rows, cols), scores.dtype)
    with _on(scores):
        bgmf.bgmf_log_probs_grad(
            scores.data_ptr(), code, rows, cols, scores.stride(0), ex, ex_stride, _ptr(given),
            temperature, row_max.data_ptr(), row_sum.data_ptr(), _ptr(entropy),
            _ptr(grad_log_prob), _ptr(grad_entropy), out.data_ptr(), out.stride(0),
            _stream(scores))
    return out


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
    def backward(ctx, g_log_prob, g_entropy, *_):
        scores, given, excluded, row_max, row_sum, entropy = ctx.saved_tensors
        if g_log_prob is None and g_entropy is None:
            return None, None, None, None, None
        g = [None if x is None else x.contiguous() for x in (g_log_prob, g_entropy)]
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
    temperature = float(temperature)
    if torch.is_grad_enabled() and scores.requires_grad:
        return LogProbs(*_LogProbs.apply(scores, given, top, temperature, excluded))
    return _forward(scores, given, top, temperature, excluded)


# --- scores in 8-bit integers ---------------------------------------------------

def quantize_rows(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows in 8-bit integers: (q int8, scale float32) with x ~ q * scale,
    scale the row's largest magnitude / 127.  The rows of q start on 16-byte
    boundaries (q is a view of a wider tensor where k needs it)."""
    code = _matrix(x, "x", _TYPES)
    rows, k = x.shape
    if k < 1:
        raise ValueError("x has rows of no elements")
    q = torch.empty((rows, -(-k // 16) * 16), dtype=torch.int8, device=x.device)[:, :k]
    scale = torch.empty(rows, device=x.device)
    with _on(x):
        bgmf.bgmf_quantize_rows(x.data_ptr(), code, rows, k, x.stride(0), q.data_ptr(),
                                q.stride(0), scale.data_ptr(), _stream(x))
    return q, scale


def quantized_scores(rows: torch.Tensor, items: torch.Tensor, item_scale: torch.Tensor,
                     row_scale: Optional[torch.Tensor] = None, *,
                     dtype: torch.dtype = torch.float32,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scores rows . items^T with both in 8-bit integers, times row_scale and
    item_scale, as ``dtype``.  ``rows``: int8 with ``row_scale``, or float32,
    bfloat16 or float16 without it, quantised in the call as by
    ``quantize_rows``.  ``items``: int8 with ``item_scale``."""
    code = _matrix(rows, "rows", _ROW_TYPES)
    _matrix(items, "items", _BYTES)
    n, k = rows.shape
    m = items.shape[0]
    if items.shape[1] != k or items.device != rows.device:
        raise ValueError("rows and items must have equally many columns, on one device")
    _vector(item_scale, "item_scale", rows, m, torch.float32)
    if (row_scale is None) != (rows.dtype != torch.int8):
        raise ValueError("row_scale goes with int8 rows and with no others")
    if row_scale is not None:
        _vector(row_scale, "row_scale", rows, n, torch.float32)
    if dtype not in _TYPES:
        raise ValueError(f"dtype must be float32, bfloat16 or float16: {dtype}")
    if out is None:
        out = torch.empty((n, m), dtype=dtype, device=rows.device)
    else:
        _output(out, "out", rows, (n, m), dtype)
    nbytes = bgmf.bgmf_quantized_scores_workspace(n, m, k, code)
    ws = _workspace(nbytes, rows)
    with _on(rows):
        bgmf.bgmf_quantized_scores(
            rows.data_ptr(), code, n, k, rows.stride(0), _ptr(row_scale), items.data_ptr(), m,
            items.stride(0), item_scale.data_ptr(), out.data_ptr(), _TYPES[dtype], out.stride(0),
            _ptr(ws), nbytes, _stream(rows))
    return out


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
        item and the entropy, as by ``log_probs``."""
        return log_probs(self.scores(users), given, top=top, temperature=temperature,
                         excluded=excluded)


# --- clipping -------------------------------------------------------------------

def _layout(t: torch.Tensor) -> Tuple[int, int, int]:
    """(rows, cols, row stride) that cover a gradient's elements."""
    if t.is_contiguous():
        return 1, t.numel(), t.numel()
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]:
        return t.shape[0], t.shape[1], t.stride(0)
    raise ValueError("a gradient is neither contiguous nor 2-D with adjacent row elements")


def clip_grad_norm(grads: Sequence[torch.Tensor], max_norm: float,
                   out: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
    """Scales gradients (float32, bfloat16 or float16, mixed or not) so that
    their global norm is at most max_norm, in place or into ``out``; returns
    the norm before (a float32 tensor on the GPU).  A norm that is not finite
    leaves the gradients as they are.  Each must be contiguous, or 2-D with
    adjacent row elements."""
    grads = list(grads)
    if not grads:
        raise ValueError("clip_grad_norm needs at least one gradient")
    dev = grads[0].get_device()
    out = grads if out is None else list(out)
    if len(out) != len(grads):
        raise ValueError("out must have a tensor for each gradient")
    sides = (grads,) if out is grads else (grads, out)
    codes = list(map(_TYPES.get, [g.dtype for g in grads]))
    # whole columns of the table at a time: a model has hundreds of gradients
    for side in sides:
        if dev < 0 or set(map(torch.Tensor.get_device, side)) != {dev}:
            raise ValueError("gradients and out must be on one GPU")
    if None in codes:
        raise ValueError("gradients must be float32, bfloat16 or float16")
    if out is not grads and codes != list(map(_TYPES.get, [o.dtype for o in out])):
        raise ValueError("out must have the gradients' types")
    table = np.zeros((len(grads), 7), dtype=np.int64)  # rows of bgmf_grad_t
    table[:, 0] = list(map(torch.Tensor.data_ptr, grads))
    table[:, 1] = table[:, 0] if out is grads else list(map(torch.Tensor.data_ptr, out))
    table[:, 6] = codes
    if all(all(map(torch.Tensor.is_contiguous, side)) for side in sides):
        sizes = list(map(torch.Tensor.numel, grads))
        if out is not grads and sizes != list(map(torch.Tensor.numel, out)):
            raise ValueError("out must have the gradients' sizes")
        table[:, 2] = 1
        table[:, 3:6] = np.array(sizes, dtype=np.int64)[:, None]
    else:
        for row, g, o in zip(table, grads, out):
            if g.shape != o.shape:
                raise ValueError("out must have the gradients' shapes")
            at, to = _layout(g), _layout(o)
            if at[0] != to[0]:  # one side has a row stride: both are taken as matrices
                at, to = ((t.shape[0], t.shape[1], t.stride(0)) for t in (g, o))
            row[2:6] = (*at, to[2])
    norm = torch.empty((), device=grads[0].device)
    nbytes = bgmf.bgmf_clip_grad_norm_workspace(len(grads))
    ws = _workspace(nbytes, grads[0])
    with _on(grads[0]):
        bgmf.bgmf_clip_grad_norm(table.ctypes.data, len(grads), float(max_norm), norm.data_ptr(),
                                 ws.data_ptr(), nbytes, _stream(grads[0]))
    return norm
