"""Log probabilities of given tokens, with entropy and top alternatives, and their gradient (include/adagc_ops.h).

    r = token_logprobs(logits, targets, top_k=5)
    loss = -r.logprob.sum() / n
    grad_logits = token_logprobs_backward(logits, targets, r.lse, r.entropy, grad_logprob=torch.full_like(r.logprob, -1 / n))

Calls only enqueue work, on `stream` (default: the current stream); outputs belong to that stream.  Tensors made or freed on
another stream have to be ordered by the caller, as with every entry point of this package.  There is no autograd here: tensors
that require a gradient are read (and written) as they are, results never require one, and the backward pass is a call of its own.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from .binding import check, lib, matrix_args, run_on, vector_ptr

MAX_TOP_K = 32


class TokenLogprobs(NamedTuple):
    logprob: Optional[torch.Tensor]      # [rows] fp32; None without targets
    lse: torch.Tensor                    # [rows] fp32
    entropy: torch.Tensor                # [rows] fp32
    top_logprob: Optional[torch.Tensor]  # [rows, top_k] fp32, descending; None for top_k = 0
    top_index: Optional[torch.Tensor]    # [rows, top_k] int32


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor], top_k: int = 0, stream=None) -> TokenLogprobs:
    """adagc_token_logprobs.  logits [rows, vocab] float32 or bfloat16 (any row stride); targets [rows] int64, negative =
    no target, or None for no log probabilities; -inf masks an entry."""
    return run_on(logits.device, stream, _token_logprobs, logits, targets, top_k)


def _token_logprobs(logits, targets, top_k, stream):
    p, dtype, rows, vocab, ld = matrix_args(logits, "logits")
    t = vector_ptr(targets, rows, torch.int64, logits.device, "targets")
    if not 0 <= top_k <= MAX_TOP_K:
        raise ValueError(f"top_k must lie in [0, {MAX_TOP_K}], got {top_k}")
    logprob, lse, entropy = logits.new_empty((3, rows), dtype=torch.float32).unbind(0)
    top = idx = top_p = idx_p = None
    if top_k:
        top, idx = logits.new_empty((rows, top_k), dtype=torch.float32), logits.new_empty((rows, top_k), dtype=torch.int32)
        top_p, idx_p = top.data_ptr(), idx.data_ptr()
    base, step = logprob.data_ptr(), 4 * rows
    check(lib().adagc_token_logprobs(p, dtype, rows, vocab, ld, t, None if t is None else base, base + step, base + 2 * step, top_k, top_p, idx_p,
                                     stream), "adagc_token_logprobs")
    return TokenLogprobs(None if targets is None else logprob, lse, entropy, top, idx)


def token_logprobs_backward(logits: torch.Tensor, targets: Optional[torch.Tensor], lse: torch.Tensor,
                            entropy: Optional[torch.Tensor] = None, grad_logprob: Optional[torch.Tensor] = None,
                            grad_lse: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                            out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """adagc_token_logprobs_backward.  The upstream gradients are [rows] float32 each, None = zero.  `out` may be `logits`
    itself (in place); by default a new tensor of the logits' dtype."""
    return run_on(logits.device, stream, _token_logprobs_backward, logits, targets, lse, entropy, grad_logprob, grad_lse, grad_entropy, out)


def _token_logprobs_backward(logits, targets, lse, entropy, grad_logprob, grad_lse, grad_entropy, out, stream):
    p, dtype, rows, vocab, ld = matrix_args(logits, "logits")
    dev, f32 = logits.device, torch.float32
    if grad_logprob is not None and targets is None:
        raise ValueError("grad_logprob needs targets")
    if grad_entropy is not None and entropy is None:
        raise ValueError("grad_entropy needs entropy")
    if out is None:
        out = torch.empty_like(logits) if logits.is_contiguous() else logits.new_empty((rows, vocab))
    q, odtype, orows, ovocab, old = matrix_args(out, "out")
    if (odtype, orows, ovocab, out.device) != (dtype, rows, vocab, dev):
        raise ValueError(f"out: expected {tuple(logits.shape)} {logits.dtype} on {dev}, got {tuple(out.shape)} {out.dtype} on {out.device}")
    check(lib().adagc_token_logprobs_backward(
        p, dtype, rows, vocab, ld, vector_ptr(targets, rows, torch.int64, dev, "targets"), vector_ptr(lse, rows, f32, dev, "lse"),
        vector_ptr(entropy, rows, f32, dev, "entropy"), vector_ptr(grad_logprob, rows, f32, dev, "grad_logprob"),
        vector_ptr(grad_lse, rows, f32, dev, "grad_lse"), vector_ptr(grad_entropy, rows, f32, dev, "grad_entropy"), q, old, stream),
        "adagc_token_logprobs_backward")
    return out
