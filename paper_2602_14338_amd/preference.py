"""A policy that learns from pairs of its own rollouts.

The curation keeps as many wrong as right rollouts of a query that has both (k_ratio = 1), which makes pairs: of each, the right
rollout is to be preferred to the wrong one.  The loss looks at how far the policy has moved towards either, as a whole, so a pair's
gradient needs all of its tokens: where they are in one batch of rows, one call does everything; over several micro-batches the
log-probs of all of them come first, then the loss on them, then each micro-batch's gradient.

Everything numeric happens in the library calls; this module has the pairs and the sequence of calls.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Callable, Optional, Tuple

import numpy as np
import torch

from . import binding
from .binding import PreferenceParams


def pairs_of_groups(rewards: np.ndarray, kept_index: np.ndarray, kept_offsets: np.ndarray, every: bool = False) -> Tuple[np.ndarray, np.ndarray]:
    """Right and wrong rollouts of each query as pairs (chosen, rejected), i32: the curation's kept rollouts in their order, the n-th right
    one with the n-th wrong one as long as there are both, or with ``every`` each right one with each wrong one."""
    chosen, rejected = [], []
    for lo, hi in zip(kept_offsets[:-1], kept_offsets[1:]):
        kept = np.asarray(kept_index[lo:hi], np.int32)
        right = np.asarray(rewards)[kept] > 0
        good, bad = kept[right], kept[~right]
        if every:
            chosen.append(np.repeat(good, bad.size))
            rejected.append(np.tile(bad, good.size))
        else:
            n = min(good.size, bad.size)
            chosen.append(good[:n])
            rejected.append(bad[:n])
    empty = [np.zeros(0, np.int32)]
    return np.concatenate(chosen or empty), np.concatenate(rejected or empty)


@dataclass
class PairLoss:
    """What a loss on pairs says about them: loss f32 [1], margins f32 [P] (positive: the preferred rollout has gained on the other),
    log ratios f32 [R]; and the policy's log-probs f32 [T]."""
    loss: torch.Tensor
    margin: torch.Tensor
    ratio: torch.Tensor
    logprob: torch.Tensor


def _empty(device: torch.device, *sizes: int):
    return [torch.empty(n, device=device) for n in sizes]


def loss_bwd(logits: torch.Tensor, V: int, targets: torch.Tensor, ref_logprob: Optional[torch.Tensor], token_rollout: torch.Tensor, R: int,
             chosen: torch.Tensor, rejected: torch.Tensor, params: PreferenceParams, dlogits: Optional[torch.Tensor],
             pair_weight: Optional[torch.Tensor] = None, grad_scale: float = 1.0, err_flag: Optional[torch.Tensor] = None) -> PairLoss:
    """Loss of the pairs whose tokens are all among the rows ``logits`` [T, ld], and its gradient into ``dlogits`` (may be ``logits``)."""
    T, P, dev = logits.shape[0], chosen.numel(), logits.device
    out = PairLoss(*_empty(dev, 1, P, R, T))
    ws = torch.empty(binding.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS_BWD, T=T, V=V, R=R, Q=P), dtype=torch.uint8, device=dev)
    binding.aero_preference_loss_bwd(logits, T, V, logits.shape[1], targets, ref_logprob, token_rollout, R, chosen, rejected, pair_weight, P,
                                     params, grad_scale, out.loss, out.margin, out.ratio, out.logprob, dlogits, ws, err_flag)
    return out


def loss_bwd_microbatches(token_rollout: torch.Tensor, logits_of: Callable[[int], torch.Tensor], targets_of: Callable[[int], torch.Tensor],
                          ref_logprob: Optional[torch.Tensor], dlogits_of: Callable[[int], Optional[torch.Tensor]], R: int,
                          chosen: torch.Tensor, rejected: torch.Tensor, params: PreferenceParams, V: int, ld: int,
                          pair_weight: Optional[torch.Tensor] = None, grad_scale: float = 1.0,
                          err_flag: Optional[torch.Tensor] = None) -> PairLoss:
    """The same over the micro-batches of ``token_rollout`` ([n_mb, mb_tokens], device int32), ``ref_logprob`` f32 [n_mb, mb_tokens].  ``*_of(k)``
    hand over the tensors of micro-batch k, logits twice: for the log-probs, and for the gradient (``dlogits_of`` may be None then: loss
    only).  Logits have to be finite here."""
    n_mb, mb = token_rollout.shape
    T, P, dev = n_mb * mb, chosen.numel(), token_rollout.device
    out = PairLoss(*_empty(dev, 1, P, R, T))
    lse, slope = _empty(dev, T, R)
    active = (token_rollout >= 0).to(torch.uint8)
    owner = torch.empty_like(token_rollout)   # rows without a sampled token take no part either
    for k in range(n_mb):
        at = slice(k * mb, (k + 1) * mb)
        y = targets_of(k)
        owner[k].copy_(token_rollout[k].masked_fill((y < 0) | (y >= V), -1))
        binding.aero_logprob_fwd(logits_of(k), mb, V, ld, y, active[k], out.logprob[at], None, lse[at], err_flag)
    ws = torch.empty(binding.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS, T=T, R=R, Q=P), dtype=torch.uint8, device=dev)
    binding.aero_preference_loss(out.logprob, T, ref_logprob, owner, R, chosen, rejected, pair_weight, P, params, out.loss, out.margin,
                                 out.ratio, slope, ws, err_flag)
    # a surrogate at a ratio of 1 has the gradient -adv of each log-prob
    adv, one, ignored = -slope, torch.ones(R, device=dev), torch.empty(1, device=dev)
    ws = torch.empty(max(binding.aero_workspace_bytes(binding.OP_GRPO_LOSS_BWD, T=mb, V=V, R=R), 1), dtype=torch.uint8, device=dev)
    for k in range(n_mb):
        dlogits = dlogits_of(k)
        if dlogits is not None:
            at = slice(k * mb, (k + 1) * mb)
            binding.aero_grpo_loss_bwd(logits_of(k), mb, V, ld, targets_of(k), lse[at], out.logprob[at], token_rollout[k], adv, one, R, 0.5, 0.5,
                                       grad_scale, ignored, None, None, dlogits, ws, None)
    return out
