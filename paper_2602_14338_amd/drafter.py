"""A drafter that follows the policy: what the calls around a drafter look like together.

Most of a step of the update is spent on rollouts.  A small model that proposes a few tokens at a time makes them cheaper: the
policy scores all of them at once and keeps those that it could have drawn itself, so the rollouts stay the policy's own.  The
policy moves with every update, and the drafter has to move with it; it learns from the logits rows that the policy computes in
any case, handed on as their K largest.

The drafter here is as small as one can be: one table that is both its embedding and its head, z_t = (scale E[x_t]) E^T.  A drafter
with layers in between differs in how the rows of ``hidden`` become logits, not in the calls.  The lists, the distillation, the
verification, the lookup and its gradient are library calls; the three products with the table are plain matrix products.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass
from typing import Callable, Optional, Tuple

import torch

from . import binding


def _workspace(op: int, device: torch.device, **sizes: int) -> torch.Tensor:
    return torch.empty(binding.aero_workspace_bytes(op, **sizes), dtype=torch.uint8, device=device)


@dataclass
class TeacherLists:
    """The policy's rows as a drafter learns from them: ids and log-probs of the K largest logits, and the rows' log-sum-exp."""
    index: torch.Tensor     # i32 [T, K]
    logprob: torch.Tensor   # f32 [T, K]
    lse: torch.Tensor       # f32 [T]


def teacher_lists(logits: torch.Tensor, V: int, K: int, row_active: Optional[torch.Tensor] = None) -> TeacherLists:
    """Lists of the policy's logits [T, ld], columns from V on ignored.  Rows with row_active == 0 get empty lists."""
    T, dev = logits.shape[0], logits.device
    out = TeacherLists(torch.empty((T, K), dtype=torch.int32, device=dev), torch.empty((T, K), device=dev), torch.empty(T, device=dev))
    binding.aero_topk_logprob(logits, T, V, logits.shape[1], row_active, K, out.index, out.logprob, out.lse,
                              _workspace(binding.OP_TOPK_LOGPROB, dev, T=T, V=V, H=K))
    return out


class Drafter:
    """Next-token drafter of one table [V, H] (bf16), embedding and head in one."""

    def __init__(self, table: torch.Tensor, scale: float = 1.0):
        self.table, self.scale = table, scale
        self.V, self.H = table.shape
        self.err = torch.zeros(1, dtype=torch.int32, device=table.device)   # bits of the calls, as err_flag collects them

    def hidden(self, ids: torch.Tensor) -> torch.Tensor:
        out = torch.empty((ids.numel(), self.H), dtype=self.table.dtype, device=self.table.device)
        binding.aero_embedding_fwd(self.table, self.V, self.H, ids, ids.numel(), self.scale, out, self.H, self.err)
        return out

    def logits(self, ids: torch.Tensor) -> torch.Tensor:
        """Rows [T, V] behind the tokens ids (i32 [T]; a negative id is padding)."""
        return self.hidden(ids) @ self.table.t()

    def loss_bwd(self, ids: torch.Tensor, teacher: TeacherLists, token_weight: torch.Tensor, dtable: Optional[torch.Tensor],
                 tail: int = binding.AERO_TAIL_BUCKET, grad_scale: float = 1.0) -> torch.Tensor:
        """Divergence of the rows behind ``ids`` from the lists, sum_t token_weight[t] L_t (f32 [1]), and, into ``dtable``
        [V, H], its gradient: what the head's product leaves, with the lookup's gradient added onto it."""
        T, K = teacher.index.shape
        dev = self.table.device
        x = self.hidden(ids)
        z = x @ self.table.t()
        loss = torch.empty(1, device=dev)
        dz = None if dtable is None else z   # in place
        binding.aero_distill_loss_bwd(z, T, self.V, self.V, teacher.index, teacher.logprob, K, token_weight, tail, grad_scale, loss, None,
                                      dz, _workspace(binding.OP_DISTILL_LOSS_BWD, dev, T=T, V=self.V), self.err)
        if dtable is not None:
            if dtable.dtype == torch.float32 and dz.dtype != torch.float32:
                torch.mm(dz.t(), x, out_dtype=torch.float32, out=dtable)   # as it is summed up: not rounded to the rows' type in between
            else:
                dtable.copy_(dz.t() @ x)
            dx = dz @ self.table
            binding.aero_embedding_bwd(dx, T, self.H, self.H, ids, self.V, self.scale, dtable,
                                       _workspace(binding.OP_EMBEDDING_BWD, dev, T=T, V=self.V, H=self.H), True, self.err)
        return loss

    def propose(self, last: torch.Tensor, G: int, generator: Optional[torch.Generator] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """G tokens behind each sequence's last one (i32 [B]): tokens i32 [B, G] and the rows [B, G, V] that they were drawn from."""
        B, dev = last.numel(), last.device
        tokens = torch.empty((B, G), dtype=torch.int32, device=dev)
        rows = torch.empty((B, G, self.V), dtype=self.table.dtype, device=dev)
        ids = last
        for g in range(G):
            z = self.logits(ids)
            _, ids, _ = verify(z.view(B, 1, self.V), None, None, None, self.V, generator, err_flag=self.err)   # nothing drafted: a draw
            ids = ids.view(B)
            tokens[:, g], rows[:, g] = ids, z
        return tokens, rows


def verify(target: torch.Tensor, draft: Optional[torch.Tensor], draft_tokens: Optional[torch.Tensor], draft_count: Optional[torch.Tensor],
           V: int, generator: Optional[torch.Generator] = None,
           err_flag: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """What the policy keeps of G drafted tokens, given its rows [B, G+1, ld] and the drafter's [B, G, ld] (None: the tokens were
    copied from somewhere): number kept i32 [B], tokens i32 [B, G+1] (the kept ones, one of the policy's own, -1 behind it) and their
    log-probs, which are the old_logprob of the update."""
    B, G, dev = target.shape[0], target.shape[1] - 1, target.device
    uniform = torch.rand((B, G), generator=generator, device=dev)
    noise = torch.empty((B, V), device=dev).exponential_(generator=generator).clamp_min_(torch.finfo(torch.float32).tiny)
    accepted = torch.empty(B, dtype=torch.int32, device=dev)
    tokens = torch.empty((B, G + 1), dtype=torch.int32, device=dev)
    logprob = torch.empty((B, G + 1), device=dev)
    binding.aero_verify_draft(target, draft, B, G, V, target.shape[2], draft_tokens, draft_count, uniform, noise, accepted, tokens, logprob,
                              _workspace(binding.OP_VERIFY_DRAFT, dev, T=B * (G + 1), V=V, Q=B), err_flag)
    return accepted, tokens, logprob


def generate(drafter: Drafter, policy: Callable[[torch.Tensor], torch.Tensor], last: torch.Tensor, G: int,
             generator: Optional[torch.Generator] = None):
    """One turn of drafting for each sequence: the policy is asked once for the rows behind the last token and the G drafted ones
    (``policy``: i32 [B, G+1] -> rows [B, G+1, ld]).  Returns accepted, tokens, logprob, the policy's rows, from which the
    drafter can learn, and the drafted tokens i32 [B, G], which with ``last`` are the tokens in front of those rows."""
    tokens, rows = drafter.propose(last, G, generator)
    target = policy(torch.cat((last.view(-1, 1), tokens), 1))
    if target.shape[2] != drafter.V:   # rows with padding columns: the drafter's get them as well
        rows = torch.nn.functional.pad(rows, (0, target.shape[2] - drafter.V))
    accepted, out, logprob = verify(target, rows, tokens, None, drafter.V, generator, drafter.err)
    return accepted, out, logprob, target, tokens


def main() -> None:
    """A made-up policy over pairs of tokens; the drafter learns it while it drafts for it."""
    ap = argparse.ArgumentParser(description=main.__doc__)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--sequences", type=int, default=256)
    ap.add_argument("--drafted", type=int, default=4)
    ap.add_argument("--top", type=int, default=64)
    ap.add_argument("--turns", type=int, default=200)
    ap.add_argument("--rate", type=float, default=0.01)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    new = lambda sigma: torch.randn((a.vocab, a.width), generator=gen, device="cuda") * sigma   # noqa: E731
    truth, drafter = new(0.35).bfloat16(), Drafter(new(0.1).bfloat16())
    master, first, second = drafter.table.float(), torch.zeros_like(new(0.0)), torch.zeros_like(new(0.0))
    dtable = torch.empty_like(master)
    last = torch.randint(0, a.vocab, (a.sequences,), generator=gen, device="cuda", dtype=torch.int32)
    for turn in range(a.turns):
        policy = lambda ids: (truth[ids.long()] @ truth.t())   # noqa: E731
        accepted, tokens, _, rows, drafted = generate(drafter, policy, last, a.drafted, gen)
        seen = torch.cat((last.view(-1, 1), drafted), 1).reshape(-1)
        lists = teacher_lists(rows.view(-1, rows.shape[2]), a.vocab, a.top)
        weight = torch.full((seen.numel(),), 1.0 / seen.numel(), device="cuda")
        loss = drafter.loss_bwd(seen, lists, weight, dtable)
        first.lerp_(dtable, 0.1)
        second.lerp_(dtable * dtable, 0.01)
        step = turn + 1
        master -= a.rate * (first / (1 - 0.9 ** step)) / ((second / (1 - 0.99 ** step)).sqrt() + 1e-12)
        drafter.table.copy_(master)
        last = tokens.gather(1, accepted.long().view(-1, 1)).view(-1)
        if turn % 20 == 0 or step == a.turns:
            print(f"turn {turn}: divergence {loss.item():.4f}, {accepted.float().mean().item():.2f} of {a.drafted} drafted tokens kept", flush=True)
    if drafter.err.item():
        raise SystemExit(f"error bits {drafter.err.item()}")


if __name__ == "__main__":
    main()
