"""The two ends of a pipeline and its residual stream on tensors: the first stage's
embedding, the last stage's log probabilities, and dropout where a branch joins the
stream (include/dpo.h).

They run around the blocks of ``ffn`` and follow its rules: weights are ``opt.stale(i)``,
gradients of weights go into ``opt.grads(i)`` (written, or with ``accumulate`` added);
tensors are on the current CUDA device, their last dimension contiguous and the others
flattening to rows; outputs are allocated unless given; calls go to PyTorch's current
stream or to ``stream=``; autograd does not see them; ValueError and TypeError for
tensors that do not fit, DpoError for what the library refuses.

    x = ends.embed(tokens[:, :-1], opt.stale(0).view(vocab, dim))
    x = ends.dropout_add(branch, x, 0.1, seed, site=layer)       # in every block
    lp, kept = ends.head_logprobs(x, w_head, tokens[:, 1:], keep=True)
    loss = -lp.logp.mean()
    dx = ends.head_logprobs_backward(dlogp, kept, x, w_head, tokens[:, 1:], lp, dw_head)
    dbranch = ends.dropout_backward(dx, 0.1, seed, site=layer)
    ends.embed_backward(dx, tokens[:, :-1], opt.grads(0).view(vocab, dim))

Token ids are int32 or int64 tensors, slices of a batch among them. An id outside the
vocabulary, -1 or -100 as well as one past its end, is padding: its embedding is a row of
zeros, its log probability 0, and neither has a gradient.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import ffn as _ffn
from .dpo import (DPO_EMBED_SPAN, DPO_MAX_TOP, dpo_dropout_args, dpo_embed_args, dpo_embed_backward_args,
                  dpo_embed_workspace, dpo_head_args, dpo_head_backward_args, dpo_head_workspace, dpo_ids,
                  dpo_logprobs_args, dpo_logprobs_backward_args, load)


def embed(ids, table, *, scale: float = 1.0, dtype=None, out=None, stream=None):
    """scale * table[ids], rounded once: shape ids.shape + (dim,), of the table's type, of
    ``dtype`` or of ``out`` (float32 or bfloat16)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return embed(ids, table, scale=scale, dtype=dtype, out=out)
    if dtype is not None and dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise TypeError(f"dtype {dtype} (float32 or bfloat16)")
    if dtype is not None and out is not None and out.dtype is not dtype:
        raise TypeError(f"out is {out.dtype}, not {dtype}")
    return _ffn._t.embed(ids, table, scale, -1 if dtype is None else dtype is torch.bfloat16, out)


def embed_backward(dy, ids, dtable, *, scale: float = 1.0, accumulate: bool = False, stream=None):
    """dtable, with the embedding's gradient written over all of it, or with ``accumulate``
    added to the rows of the ids met: the sum of scale * dy over each id's tokens, in fp32,
    in an order that the ids, their number and dim alone decide."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return embed_backward(dy, ids, dtable, scale=scale, accumulate=accumulate)
    return _ffn._t.embed_backward(dy, ids, dtable, scale, accumulate)


def dropout_add(x, residual, p: float, seed, *, site: int = 0, out=None, stream=None):
    """residual + dropout(x), or dropout(x) where residual is None. An element is dropped with
    probability p, to a multiple of 2^-16, and the others are divided by 1 - p. The mask is a
    function of (seed, site, row, column), so it is not kept: give each step its seed and
    each dropout in it a site. ``seed``: an integer, of which 64 bits count, or an int64 CUDA
    tensor of one element that is read when the kernel runs, for calls captured in a CUDA
    graph. ``out`` may be x or residual where these are two tensors."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return dropout_add(x, residual, p, seed, site=site, out=out)
    return _ffn._t.dropout(x, residual, p, seed, site, out)


def dropout_backward(dy, p: float, seed, *, site: int = 0, out=None, stream=None):
    """The gradient of dropout_add's x from that of its result, with the same p, seed and site;
    the residual's gradient is dy itself. ``out`` may be dy."""
    return dropout_add(dy, None, p, seed, site=site, out=out, stream=stream)


class LogProbs(NamedTuple):
    """Of rows of logits; shapes are the rows', with a last dimension of ``top`` or, for
    ``stats``, of two."""
    logp: Optional[torch.Tensor]       # of the given ids, 0 for padding; None without ids
    entropy: torch.Tensor              # in nats
    stats: torch.Tensor                # (max, log of the sum of e^(z - max)), for the backward
    top_logp: Optional[torch.Tensor]   # of the ``top`` most likely ids, descending
    top_ids: Optional[torch.Tensor]    # int64; ties go to the lowest id
    scale: float


def token_logprobs(logits, ids=None, *, scale: float = 1.0, top: int = 0, stream=None) -> LogProbs:
    """The log probability of each row's id under softmax(scale * logits), the entropy, and
    the ``top`` (at most 32) most likely ids, NaN after all others. Logits are float32 or bfloat16;
    -inf masks."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return token_logprobs(logits, ids, scale=scale, top=top)
    return LogProbs(*_ffn._t.token_logprobs(logits, ids, scale, top), scale)


def token_logprobs_backward(dlogp, logits, ids, lp: LogProbs, *, dentropy=None, dlogits=None,
                            stream=None):
    """dlogits from the gradients of lp.logp and, where given, of lp.entropy (float32, one per
    row). ``dlogits`` may be logits itself. A row whose gradients are 0 gets zeros, whatever
    its logits are."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return token_logprobs_backward(dlogp, logits, ids, lp, dentropy=dentropy, dlogits=dlogits)
    return _ffn._t.token_logprobs_backward(dlogp, logits, ids, lp.stats, lp.entropy, dentropy, lp.scale,
                                           dlogits)


def head_logprobs(x, w, ids=None, *, scale: float = 1.0, top: int = 0, keep: bool = False, stream=None):
    """(LogProbs, kept): ``token_logprobs`` of the logits x w^T, which are formed in fp32 from
    the bf16 stream and the bf16 weights of the head (vocab x dim). With ``keep`` what the
    backward needs is kept, an opaque tensor of 2 bytes a logit and a 64th more (0.53 GB of 8192
    tokens and a vocabulary of 32000), which every microbatch in flight holds; else it is None. With
    ``top`` a workspace of 4 bytes a logit is taken for the call."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return head_logprobs(x, w, ids, scale=scale, top=top, keep=keep)
    *out, kept = _ffn._t.head_logprobs(x, w, ids, scale, top, keep)
    return LogProbs(*out, scale), kept


def head_logprobs_backward(dlogp, kept, x, w, ids, lp: LogProbs, dw, *, dentropy=None,
                           accumulate: bool = False, dx=None, stream=None):
    """dx, from the gradients of lp.logp and, where given, of lp.entropy (float32, one per
    token), and the head's gradient written into dw (fp32 or bf16, ``opt.grads(i)`` reshaped),
    or with ``accumulate`` added to it. ``kept`` may be used again. A workspace of 2 bytes a logit is
    taken for the call."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return head_logprobs_backward(dlogp, kept, x, w, ids, lp, dw, dentropy=dentropy,
                                          accumulate=accumulate, dx=dx)
    if kept is None:
        raise ValueError("the forward kept nothing (keep=False)")
    if lp.logp is None:
        raise ValueError("the forward had no ids")
    return _ffn._t.head_logprobs_backward(dlogp, kept, x, w, ids, lp.logp, lp.entropy, lp.stats, dw,
                                          dentropy, lp.scale, accumulate, dx)


def status() -> int:
    """Error bits of the tensor-core kernels (0: healthy), those of the feed-forward ones
    included, until dpo.dpo_ffn_clear_status clears them; waits for the device."""
    return _ffn.status()


# The calls as they are in include/dpo.h; the functions above make them through dpo_tensors.

EXPORTS = ("dpo_embed", "dpo_embed_backward", "dpo_embed_workspace", "dpo_dropout", "dpo_logprobs",
           "dpo_logprobs_backward", "dpo_head", "dpo_head_backward", "dpo_head_workspace")

lib = load
