"""AdamW on the library's multi-tensor step: nm_adamw (csrc/adamw.hip) takes all tensors of a group in one launch."""
from __future__ import annotations

import torch

from . import api


class NMAdamW(torch.optim.Optimizer):
    """AdamW (decoupled weight decay) for float32 and bfloat16 parameters on the GPU.

    states: "f32", or "q8": e4m3 codes with a power-of-two scale for every 256 elements, rounded stochastically (2 bytes for an element instead of 8).
    master: float32 copies of bfloat16 parameters take the steps; without them a parameter is rounded to nearest after every step, and
    steps below half of its last place are lost.  seed: of the random words of "q8".
    step(grad_scale=...): a factor on the gradients, a number or a float32 tensor on the GPU (unscaling, a clip coefficient).

    A step is not captured in a graph: its number, bias corrections, rates and random words are arguments of the launch, which every replay would repeat.
    """

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2, states: str = "f32", master: bool = False,
                 seed: int = 0):
        if states not in ("f32", "q8"):
            raise ValueError(f'states is "f32" or "q8", got {states!r}')
        if not (lr >= 0 and eps >= 0 and weight_decay >= 0 and all(0 <= b < 1 for b in betas)):
            raise ValueError("lr, eps and weight_decay are not negative, betas lie in [0, 1)")
        self.states, self.master, self.seed = states, master, seed
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))

    def __getstate__(self):
        return {**super().__getstate__(), "states": self.states, "master": self.master, "seed": self.seed}      # (torch's names what it has itself)

    def _state(self, p: torch.Tensor) -> dict:
        s = self.state[p]
        if not s:
            s["step"] = 0
            for k in ("exp_avg", "exp_avg_sq"):
                if self.states == "q8":
                    s[k], s[k + "_scale"] = api.alloc_adamw_state(p.detach(), q8=True)
                else:
                    s[k] = api.alloc_adamw_state(p.detach())
            if self.master and p.dtype != torch.float32:
                s["master"] = p.detach().to(torch.float32, memory_format=torch.preserve_format, copy=True)
        return s

    @torch.no_grad()
    def step(self, closure=None, grad_scale=1.0):
        if torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("NMAdamW.step cannot be captured in a graph: every replay would take the same step number, bias correction and random words")
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        number = 0
        for group in self.param_groups:
            calls = {}                                            # (tensors that joined later are at another step)
            for p in group["params"]:
                number += 1
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise TypeError("NMAdamW takes dense gradients")
                s = self._state(p)
                pair = lambda k: (s[k], s[k + "_scale"]) if k + "_scale" in s else s[k]        # noqa: E731
                calls.setdefault((s["step"] + 1, "master" in s), []).append((p, p.grad, pair("exp_avg"), pair("exp_avg_sq"), s.get("master"), number - 1))
            for (step, master), tensors in calls.items():
                p, g, m, v, w, numbers = map(list, zip(*tensors))
                api.nm_adamw(p, g, m, v, step, lr=group["lr"], betas=group["betas"], eps=group["eps"], weight_decay=group["weight_decay"],
                             masters=w if master else None, grad_scale=grad_scale, seed=self.seed, numbers=numbers)
                for t in p:
                    self.state[t]["step"] = step                  # (once it has been taken: an error leaves the count)
        return loss

    def load_state_dict(self, state_dict):
        """As torch's, but states keep their own types (torch's casts them to their parameter's)."""
        super().load_state_dict(state_dict)
        saved = [k for g in state_dict["param_groups"] for k in g["params"]]
        for k, p in zip(saved, (p for g in self.param_groups for p in g["params"])):
            if k in state_dict["state"]:
                self.state[p] = {name: x.to(p.device, copy=True) if isinstance(x, torch.Tensor) else x for name, x in state_dict["state"][k].items()}
