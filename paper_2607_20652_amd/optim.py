"""AdamW for the parameters of a model, in the library's kernel.

`AdamW(params).step()` updates all parameters of one type in one call of
dpb_adamw_step: fp32 or 8-bit states, optional fp32 masters of bf16
parameters, and decay of matrices only if asked for.  It keeps torch's
step / zero_grad / state_dict manner, but is no torch.optim.Optimizer: a schedule sets .lr.
"""
from __future__ import annotations

from typing import Iterable

import torch

from . import binding as B


def _versions(tensors, master) -> list | None:
    """The parameters' versions, where masters go by them."""
    return None if master is None else [None if t.is_inference() else t._version for t in tensors]


class AdamW:
    """params: tensors with gradients (or (tensor, weight_decay) pairs).

    bits: of the states, 32 or 8; master: fp32 copies of bf16 parameters that
    the steps update (default: whenever parameters are bf16); seed: of the
    rounding of 8-bit states (whose root of the second moment scatters by some 16% around
    what 32 bits hold, 1% high).

    Parameters that were changed since the last step (loaded, say) are taken over into their
    masters by the next one.  It goes by their versions, which writes through .data do not
    change: take_parameters() then does it."""

    def __init__(self, params: Iterable, lr: float = 1e-3, betas: tuple[float, float] = (0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.0, bits: int = 32, master: bool | None = None,
                 seed: int = 0):
        self.lr, self.betas, self.eps, self.bits, self.seed = lr, betas, eps, bits, seed
        self.steps = 0
        pairs = [p if isinstance(p, tuple) else (p, weight_decay) for p in params]
        if len({id(p) for p, _ in pairs}) != len(pairs):
            raise ValueError("a parameter is given twice")
        self.groups = []
        for dtype in (torch.float32, torch.bfloat16):
            mine = [(p, wd) for p, wd in pairs if p.dtype == dtype]
            if mine:
                tensors = [p for p, _ in mine]
                keep = dtype == torch.bfloat16 if master is None else master
                m, v, scales, weights = B.adamw_state(tensors, bits, keep)
                self.groups.append(dict(params=tensors, decay=[float(wd) for _, wd in mine], m=m, v=v, scales=scales,
                                        master=weights, versions=_versions(tensors, weights)))
        if sum(len(g["params"]) for g in self.groups) != len(pairs):
            raise TypeError("parameters have to be float32 or bfloat16")

    @torch.no_grad()
    def step(self, grad_scale: torch.Tensor | None = None):
        """One step from the parameters' gradients, times the device scalar grad_scale; a
        parameter without a gradient is an error, before which nothing is changed."""
        grads = [[p.grad for p in g["params"]] for g in self.groups]
        if any(x is None for mine in grads for x in mine):
            raise ValueError("a parameter has no gradient")
        grads = [[x.contiguous() for x in mine] for mine in grads]
        steps = self.steps + 1
        # the places of two groups' states are the same numbers: their seeds are not
        calls = [B._adamw(g["params"], mine, g["m"], g["v"], g["scales"], g["master"], steps, self.lr, self.betas, self.eps,
                          g["decay"], grad_scale, self.seed + 2 * steps + i)
                 for i, (g, mine) in enumerate(zip(self.groups, grads))]
        for g, call in zip(self.groups, calls):
            if _versions(g["params"], g["master"]) != g["versions"]:
                self._take(g)
            call()
            g["versions"] = _versions(g["params"], g["master"])
        self.steps = steps

    def take_parameters(self):
        """Takes the parameters' present values over into the masters, where they are not
        the masters' own, rounded."""
        for g in self.groups:
            if g["master"] is not None:
                self._take(g)

    @torch.no_grad()
    def _take(self, g):
        at = 0
        for p in g["params"]:
            n = p.numel()
            mine, p = g["master"][at:at + n], p.reshape(-1)
            mine.copy_(torch.where(mine.to(p.dtype) == p, mine, p.float()))
            at += -(-n // B.ADAMW_BLOCK) * B.ADAMW_BLOCK
        g["versions"] = _versions(g["params"], g["master"])

    def zero_grad(self):
        for g in self.groups:
            for p in g["params"]:
                p.grad = None

    def state_dict(self) -> dict:
        return {"steps": self.steps, "groups": [{k: g[k] for k in ("m", "v", "scales", "master")} for g in self.groups]}

    def load_state_dict(self, state: dict):
        if len(state["groups"]) != len(self.groups):
            raise ValueError("the state is of other parameters")
        for g, s in zip(self.groups, state["groups"]):
            for k in ("m", "v", "scales", "master"):
                if (g[k] is None) != (s[k] is None) or (g[k] is not None and g[k].shape != s[k].shape):
                    raise ValueError("the state is of other parameters")
        for g, s in zip(self.groups, state["groups"]):
            for k in ("m", "v", "scales", "master"):
                if g[k] is not None:
                    g[k].copy_(s[k])
        self.steps = int(state["steps"])
