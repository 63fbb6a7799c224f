"""AdamW over all tensors of a model, 112 of them in a launch (in two with max_norm), with states in 32 or 8 bits.

    opt = AdamW(block.parameters(), lr=1e-3, bits=8, max_norm=1.0)
    loss.backward()
    opt.step()

The arithmetic is ops.adamw's (include/o1d.h, o1d_adamw): decoupled weight decay, steps counted in device memory, one count
for all tensors of a set and type (one that had no gradient for a while is corrected as the others are), and with max_norm the gradients limited to
that norm; a step whose norm is not finite changes nothing.

It is no torch.optim.Optimizer: its sets are in `groups`, and a learning rate that changes is a float32 tensor on the GPU or is
written there.
"""
from __future__ import annotations

import torch

from . import ops


class AdamW:
    """params: tensors, or dicts {"params": tensors} with an lr, betas, eps or weight_decay of their own.  master: keep the
    parameters in float32 beside them (None: those in bfloat16); a parameter that was written since the last step (a loaded
    checkpoint) is no longer its master rounded, and goes on from what was written.  max_norm is of all gradients together, and is for parameters of one
    set and type."""

    def __init__(self, params, lr: float | torch.Tensor = 1e-3, betas: tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, bits: int = 32, master: bool | None = None, max_norm: float | None = None):
        if isinstance(params, torch.Tensor):
            raise TypeError("params are tensors or dicts of them, not one tensor (whose rows would be taken)")
        params = list(params)
        sets = params if params and isinstance(params[0], dict) else [{"params": params}]
        defaults = {"lr": lr, "betas": betas, "eps": eps, "weight_decay": weight_decay}
        self.max_norm, self.groups, seen = max_norm, [], set()
        for given in sets:
            unknown = set(given) - set(defaults) - {"params"}
            if unknown:
                raise ValueError(f"unknown options {sorted(unknown)}")
            kinds: dict = {}
            for p in [given["params"]] if isinstance(given["params"], torch.Tensor) else given["params"]:
                if not isinstance(p, torch.Tensor) or not p.is_leaf:  # (no gradient arrives at a tensor that was computed)
                    raise ValueError(f"parameters must be leaf tensors, got {type(p).__name__}")
                if id(p) in seen:
                    raise ValueError("a parameter is given twice")
                seen.add(id(p))
                kinds.setdefault((p.dtype, p.device), []).append(p)
            for (dtype, _), same in kinds.items():
                keep = dtype is torch.bfloat16 if master is None else master
                self.groups.append({**defaults, **{k: v for k, v in given.items() if k != "params"}, "params": same,
                                    "state": ops.AdamState.zeros(same, bits, keep)})
        if not self.groups:
            raise ValueError("no parameters")
        if max_norm is not None and len(self.groups) > 1:
            raise ValueError("max_norm is for parameters of one set, type and device")

    @torch.no_grad()
    def step(self) -> torch.Tensor | None:
        """One step; with max_norm returns the gradients' norm."""
        norm = None
        for g in self.groups:
            norm = ops.adamw(g["params"], [None if p.grad is None else p.grad.contiguous() for p in g["params"]], g["state"], g["lr"], g["betas"], g["eps"],
                             g["weight_decay"], self.max_norm, follow=True)
        return norm

    def zero_grad(self) -> None:
        for g in self.groups:
            for p in g["params"]:
                p.grad = None

    @property
    def nbytes(self) -> int:
        return sum(g["state"].nbytes for g in self.groups)

    def state_dict(self) -> dict:
        """The options and states (the tensors themselves, not copies), without the parameters."""
        names = [n for n in ops.AdamState.__slots__ if n != "starts"]
        return {"groups": [{**{k: v for k, v in g.items() if k not in ("params", "state")},
                            "state": {n: getattr(g["state"], n) for n in names}} for g in self.groups]}

    @torch.no_grad()
    def load_state_dict(self, held: dict) -> None:
        """Takes over copies of the states, which have to be of these parameters' sizes, and the options, where a captured step finds
        them (but states of other bits, which need a new capture).  The parameters are loaded by
        themselves, before or after: those that are not their masters rounded go on from their own values."""
        if len(held["groups"]) != len(self.groups):
            raise ValueError(f"{len(held['groups'])} sets of states for {len(self.groups)} of parameters")
        made = []
        for g, new in zip(self.groups, held["groups"]):
            device, t = g["state"].m.device, new["state"]
            if list(t["sizes"]) != g["state"].sizes or (t["master"] is None) != (g["state"].master is None):
                raise ValueError(f"the states are of other parameters: {t['sizes']}")
            if isinstance(new.get("lr"), torch.Tensor) and new["lr"].numel() != 1:
                raise ValueError(f"lr must be one value, got {tuple(new['lr'].shape)}")
            steps = t["step"].tolist()
            if len(steps) != 2 or steps[0] < 0 or steps[1] != 0:
                raise ValueError(f"step must be the steps taken and 0, got {steps}")
            made.append(ops.AdamState(t["sizes"], *(None if t[n] is None else t[n].detach().to(device, copy=True)
                                                    for n in ("m", "v", "step", "ms", "vs", "master"))))
        # (into the tensors that there are, where they are of this kind: a captured step reads and writes those)
        for g, new, state in zip(self.groups, held["groups"], made):
            for k, v in new.items():
                if k == "lr" and isinstance(g["lr"], torch.Tensor):
                    g["lr"].copy_(torch.as_tensor(v, dtype=torch.float32).reshape(g["lr"].shape))
                elif k != "state":
                    g[k] = v.detach().to(state.m.device, copy=True) if isinstance(v, torch.Tensor) else v
            if g["state"].m.dtype is not state.m.dtype:
                g["state"] = state
                continue
            for n in ("m", "v", "step", "ms", "vs", "master"):
                if getattr(state, n) is not None:
                    getattr(g["state"], n).copy_(getattr(state, n))
