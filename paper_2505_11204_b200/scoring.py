"""Log probabilities of given tokens with entropy, differentiable (``randes.token_scores`` behind torch's autograd).

    logprob, entropy = token_log_probs(logits, targets)
    (-logprob.mean()).backward()

Forward and backward are one kernel each; nothing of the size of the logits is kept but the logits themselves.
"""
from __future__ import annotations

import torch

from . import randes


class _TokenLogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, scale):
        scores = randes.token_scores(logits, targets, scale=scale)
        ctx.save_for_backward(logits, targets, scores.stats)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return scores.logprob.clone(), scores.entropy.clone()      # (not views of what backward reads)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_logprob, g_entropy):
        if g_logprob is None and g_entropy is None:
            return None, None, None
        logits, targets, stats = ctx.saved_tensors
        rows = lambda g: None if g is None else g.to(torch.float32).contiguous()      # (a gradient of a sum arrives expanded)
        scores = randes.TokenScores(stats[0], stats[1], stats, None, None)
        return randes.token_scores_backward(logits, targets, scores, rows(g_logprob), rows(g_entropy), scale=ctx.scale), None, None


def token_log_probs(logits, targets, scale: float = 1.0):
    """(log probability of ``targets``, entropy) of every row of softmax(scale * logits), both fp32 [n] and differentiable.

    logits: [n, vocab] fp32 or bf16 CUDA tensor; targets: int64 [n], negative = not scored (0, no gradient)."""
    return _TokenLogProbs.apply(logits, targets, float(scale))
