"""The optimizer of PAM models: AdamW over all parameters in a few launches, the
gradients' common norm limited and the states held in 8 or in 32 bits
(``pam.grad_norm``, ``pam.adamw_step``)."""
from __future__ import annotations

import torch

from . import PamError
from . import grad_norm as _grad_norm
from .training import STATE_BLOCK, _adamw, _step_tensors

__all__ = ["AdamW"]


def _check_rates(group) -> None:
    for name in ("lr", "eps", "weight_decay"):
        if not group[name] >= 0:
            raise ValueError(f"{name} must be >= 0, got {group[name]}")
    if not all(0 <= b < 1 for b in group["betas"]):
        raise ValueError(f"betas must be in [0, 1), got {group['betas']}")


def _check_new(some) -> None:
    """(parameter, gradient) pairs whose states are to be made."""
    for p, g in some:
        if p.dtype != torch.float32:
            raise TypeError(f"AdamW takes float32 parameters, got {p.dtype}")
        if not p.is_cuda:
            raise PamError("AdamW takes HIP (cuda) parameters; the PAM library has no CPU path")
        if not p.is_contiguous():
            raise ValueError(f"AdamW takes contiguous parameters, got strides {p.stride()} of shape {tuple(p.shape)}")
        if g.dtype not in (torch.float32, torch.bfloat16) or g.dtype != some[0][1].dtype:
            raise TypeError(f"AdamW takes gradients all float32 or all bfloat16, got {g.dtype}")
        if p.device != some[0][0].device or g.device != p.device:
            raise ValueError(f"parameters of a group are on {some[0][0].device} and {p.device}, a gradient on {g.device}")
    ranges = sorted((p.data_ptr(), p.data_ptr() + 4 * p.numel()) for p, _ in some if p.numel() > 0)
    if any(a[1] > b[0] for a, b in zip(ranges, ranges[1:])):
        raise ValueError("parameters of a group share memory")


class AdamW(torch.optim.Optimizer):
    """AdamW with decoupled weight decay over float32 HIP parameters.

    ``max_norm`` limits the common norm of all gradients of a step (its value:
    ``last_norm``, a tensor).  ``state_bits=8`` keeps the two averages of the
    gradients in a byte a value, and 8 bytes a block of 256, in place of 8
    bytes a value; their rounding is stochastic, by ``seed``.  A parameter
    without a gradient is passed over.  ``step`` counts on the host: inside a
    captured graph use ``pam.adamw_step`` with a step on the device, and for
    bfloat16 copies of the parameters its ``copies``.  A step that is refused
    (parameters not contiguous or of another type or device, rates that are none)
    changes no parameter."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 max_norm: float = None, state_bits: int = 32, seed: int = 0):
        _check_rates(dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits must be 8 or 32, got {state_bits}")
        if max_norm is not None and not max_norm > 0:
            raise ValueError(f"max_norm must be > 0, got {max_norm}")
        self.max_norm, self.state_bits, self.seed = max_norm, state_bits, seed
        self.last_norm = None
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))

    def __getstate__(self):
        return {**super().__getstate__(), "max_norm": self.max_norm, "state_bits": self.state_bits, "seed": self.seed,
                "last_norm": self.last_norm}

    def _state_of(self, p):
        state = self.state[p]
        if not state:
            state["step"] = 0
            if self.state_bits == 32:
                state["avg"], state["sq"] = (torch.zeros_like(p, memory_format=torch.contiguous_format) for _ in range(2))
            else:
                state["avg"], state["sq"] = (torch.zeros(p.shape, dtype=torch.uint8, device=p.device) for _ in range(2))
                state["avg_scale"], state["sq_scale"] = (
                    torch.zeros(-(-p.numel() // STATE_BLOCK), device=p.device) for _ in range(2))
        return state

    def load_state_dict(self, state_dict) -> None:
        """As torch's, but the loaded tensors are copied, and codes stay bytes (torch
        makes every state the parameter's type)."""
        for state in state_dict["state"].values():
            if state and ("avg" not in state or ("avg_scale" in state) != (self.state_bits == 8)):
                raise ValueError(f"the loaded states are not this optimizer's in {self.state_bits} bits")
        super().load_state_dict(state_dict)
        for state in self.state.values():
            for key in ("avg", "sq", "avg_scale", "sq_scale"):
                if key in state:
                    codes = self.state_bits == 8 and not key.endswith("_scale")
                    state[key] = state[key].to(torch.uint8 if codes else torch.float32, copy=True).contiguous()

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a captured step would not count on: use pam.adamw_step with a step on the device")
        # Parameters of one group that have made as many steps go together.  A refused step
        # leaves parameters and states as they were: new states are made, and the first
        # of several calls runs, when every call's tensors and rates are known to do.
        calls, new = {}, {}
        for index, group in enumerate(self.param_groups):
            for p in group["params"]:
                g = p.grad
                if g is None:
                    continue
                if g.is_sparse:
                    raise RuntimeError("AdamW takes dense gradients")
                state = self.state.get(p)
                if state:
                    calls.setdefault((index, state["step"]), []).append((p, g.contiguous(), state))
                else:
                    new.setdefault(index, []).append((p, g.contiguous()))
        if not calls and not new:
            return loss
        if new or len(calls) > 1:
            for group in self.param_groups:
                _check_rates(group)
        for some in new.values():
            _check_new(some)
        for index, some in new.items():
            calls.setdefault((index, 0), []).extend((p, g, self._state_of(p)) for p, g in some)
        ready = []
        for (index, step), some in calls.items():
            params, grads, states = zip(*some)
            scales = [None, None]
            if self.state_bits == 8:
                scales = [[s["avg_scale"] for s in states], [s["sq_scale"] for s in states]]
            packed = _step_tensors(params, grads, [s["avg"] for s in states], [s["sq"] for s in states], *scales, None)
            ready.append((index, step, packed, grads, states))
        norm = None
        if self.max_norm is not None:
            norm = self.last_norm = _grad_norm([g for call in ready for g in call[3]])
        for index, step, packed, _, states in ready:
            group = self.param_groups[index]
            # A seed of its own for each group: tensors are numbered within a call.
            _adamw(packed, step + 1, group["lr"], group["betas"], group["eps"], group["weight_decay"], norm, self.max_norm,
                   self.seed + 0x51ED27 * index)
            for s in states:
                s["step"] = step + 1
        return loss
