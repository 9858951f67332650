"""The step that gradients end in: norm over all tensors, clipping, and Adam with decoupled weight decay, without a look at the
device in between.

Everything numeric happens in the library calls; this module holds the moments and the table that describes the tensors.  Gradients
and parameters are buffers that stay where they are (those that the loss calls write into); a step is two launches for tensors of one kind, and
can be captured: the count of steps and the factor on the rate are device words.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import binding
from .binding import AERO_MOMENT_BLOCK, AdamWParams, AeroError, TensorTable


class AdamW:
    """``params`` and ``grads``: tensors of the same sizes, f32, bf16 or fp16.  16-bit parameters are stepped on an f32 master of their own unless
    ``master`` is false (bf16 alone).  ``bits``: of the moments, 32 or 8.  ``stochastic``: 8-bit moments, and bf16
    parameters without a master, are rounded at random.  ``decay``: a number for each parameter that multiplies the weight decay."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.01, decay: Optional[Sequence[float]] = None, bits: int = 32, master: bool = True,
                 stochastic: bool = False, seed: int = 0, max_norm: float = 0.0):
        if bits not in (8, 32):
            raise AeroError(f"moments have 8 or 32 bits, not {bits}")
        if len(params) != len(grads) or (decay is not None and len(decay) != len(params)):
            raise AeroError("params, grads and decay differ in number")
        if not params:
            raise AeroError("no parameters")
        self.params = AdamWParams(lr=lr, beta1=betas[0], beta2=betas[1], eps=eps, weight_decay=weight_decay, seed=seed, stochastic=stochastic)
        self.max_norm = max_norm
        dev = params[0].device
        entries: List[Dict] = []
        for k, (p, g) in enumerate(zip(params, grads)):
            n = p.numel()
            e = dict(param=p, grad=g, decay=decay[k] if decay is not None else 1.0)
            if master and p.dtype != torch.float32:
                e["master"] = p.detach().to(torch.float32).contiguous()
            if bits == 32:
                e["exp_avg"], e["exp_avg_sq"] = torch.zeros(n, device=dev), torch.zeros(n, device=dev)
            else:
                blocks = (n + AERO_MOMENT_BLOCK - 1) // AERO_MOMENT_BLOCK
                e["exp_avg"], e["exp_avg_scale"] = torch.zeros(n, dtype=torch.int8, device=dev), torch.zeros(blocks, device=dev)
                e["exp_avg_sq"], e["exp_avg_sq_scale"] = torch.zeros(n, dtype=torch.uint8, device=dev), torch.zeros(blocks, device=dev)
            entries.append(e)
        self.table = TensorTable(entries)
        self.count = torch.zeros(1, dtype=torch.int32, device=dev)   # steps made
        self.norm, self.factor = torch.zeros(1, device=dev), torch.ones(1, device=dev)
        self._workspace = torch.empty(binding.aero_workspace_bytes(binding.OP_GRAD_NORM), dtype=torch.uint8, device=dev)

    def step(self, grad_scale: float = 1.0, lr_factor: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One step on what ``grads`` hold, times ``grad_scale``, clipped to ``max_norm`` if that is positive; ``lr_factor`` f32 [1] on the
        device.  Returns the gradients' norm (f32 [1], before clipping).  Where a gradient is infinite or NaN, nothing changes."""
        binding.aero_grad_norm(self.table, grad_scale, self.max_norm, self.norm, self.factor, self._workspace)
        binding.aero_adamw_step(self.table, self.params, self.count, self.factor, lr_factor)
        return self.norm

    def moments(self, dtype: torch.dtype = torch.float32) -> List[Tuple[torch.Tensor, torch.Tensor]]:
        """Both moments of each parameter as numbers (f32 or bf16), whatever they are held in."""
        n = self.table.n_moments
        avg, sq = (torch.empty(n, dtype=dtype, device=self.count.device) for _ in range(2))
        binding.aero_adamw_moments(self.table, avg, sq)
        sizes = [e["grad"].numel() for e in self.table.entries]
        return [(a.view(e["grad"].shape), s.view(e["grad"].shape))
                for e, a, s in zip(self.table.entries, avg.split(sizes), sq.split(sizes))]

    _HELD = ("master", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")

    def state_dict(self) -> Dict:
        """Copies of what the steps have left besides the parameters."""
        return dict(count=self.count.clone(), tensors=[{k: e[k].clone() for k in self._HELD if e.get(k) is not None} for e in self.table.entries])

    def load_state_dict(self, state: Dict) -> None:
        if len(state["tensors"]) != len(self.table.entries):
            raise AeroError("the state is of another number of tensors")
        for e, s in zip(self.table.entries, state["tensors"]):
            if set(s) != {k for k in self._HELD if e.get(k) is not None}:
                raise AeroError("the state is held in another form")
            for k, x in s.items():
                if x.shape != e[k].shape or x.dtype != e[k].dtype:
                    raise AeroError(f"{k} of the state has another size or type")
        for e, s in zip(self.table.entries, state["tensors"]):
            for k, x in s.items():
                e[k].copy_(x)
        self.count.copy_(state["count"])
