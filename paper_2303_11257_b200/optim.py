"""AdamW over the tensors of a model: one launch of us_adamw a step, and one of us_grad_norm before it where gradients are clipped.

A driver only, as the block drivers are: it owns the states and issues the calls.  With `copies` a step leaves the weights in the matmuls' operands (UnitScaledBiasFFN
takes them as they are: step(X, None, None, G)), so that no cast of the weights opens the next step:

    block = ffn.UnitScaledBiasFFN(T, d, f)
    block.cast_weights(W1, W2)
    opt = optim.AdamW([W1, W2, block.b1, block.b2], [block.dW1, block.dW2, block.db1, block.db2], lr=..., weight_decay=[0.01, 0.01, 0, 0],
                      copies=[block.W1q, block.W2q, None, None], states="8bit", rounding="random", max_norm=1.0)
    for ...:
        block.step(X, None, None, G)
        opt.step()

A step makes no synchronisation, and can be captured into a CUDA graph: the count of steps is kept on the device, as are the gradients' norm and the factor
that clips them.  A schedule that a captured step is to follow goes through lr_factor, a float32 CUDA tensor whose first element multiplies lr.  A step whose gradients'
norm is not finite changes nothing (with max_norm; float("inf") clips nothing).

The tensors are described to the library once, and again whenever one of them is another or lies elsewhere.  That takes about 0.2 ms for 96 tensors, as much as the norm of small ones saves:
keep the gradients' tensors, as the blocks do, and write into them.
"""
from __future__ import annotations

import torch

from . import _binding
from . import lib as L


class AdamW:
    """params: float32 CUDA matrices and vectors, updated in place; grads: their gradients (float32, bfloat16 or float16), the same tensors in every step; copies: None or a
    list of operands (or Nones) of the parameters' shapes; weight_decay: a number or one per tensor; states: "32bit" or "8bit".

    rounding: of states in 8 bits, "nearest" or "random" (up or down with the probabilities that keep the mean, alike in every run).  Take "random" to train with usual betas: to
    the nearest code, a state that a step changes by less than 3 to 6 % does not change at all, so that with beta2 = 0.999 an element whose gradients become ten times smaller than
    its block's others keeps its denominator, and its steps stay many times too small."""

    def __init__(self, params, grads, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, copies=None, states: str = "32bit",
                 max_norm: float | None = None, lr_factor: torch.Tensor | None = None, rounding: str = "nearest"):
        self.params, self.grads = list(params), list(grads)
        if states not in ("32bit", "8bit"):
            raise ValueError("states: 32bit or 8bit")
        if rounding not in ("nearest", "random") or (rounding == "random" and states != "8bit"):
            raise ValueError("rounding of states in 8 bits: nearest or random")
        if not self.params or len(self.grads) != len(self.params) or any(g.shape != p.shape for g, p in zip(self.grads, self.params)):
            raise ValueError("one gradient of the parameter's shape per parameter is wanted")
        if any(p.dtype is not torch.float32 for p in self.params):
            raise ValueError("parameters are float32")
        n, device = len(self.params), self.params[0].device
        self.copies = [None] * n if copies is None else list(copies)
        self.weight_decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        if len(self.copies) != n or len(self.weight_decay) != n:
            raise ValueError("one entry per parameter is wanted")
        self.lr, self.betas, self.eps, self.max_norm, self.states, self.lr_factor = lr, tuple(betas), eps, max_norm, states, lr_factor
        eight, self._rounding = states == "8bit", L.US_ROUND_RANDOM if rounding == "random" else L.US_ROUND_NEAREST
        state = lambda p: torch.zeros(p.shape, dtype=torch.uint8 if eight else torch.float32, device=p.device).view(torch.float8_e4m3fn if eight else torch.float32)
        scale = lambda p: torch.zeros(-(-p.numel() // L.ADAMW_BLOCK), dtype=torch.float32, device=p.device) if eight else None
        self.m, self.v = [state(p) for p in self.params], [state(p) for p in self.params]
        self.m_scale, self.v_scale = [scale(p) for p in self.params], [scale(p) for p in self.params]
        self.count = L.new_adamw_step(0, device)                  # steps made, on the device
        self.norm = torch.zeros(2, dtype=torch.float32, device=device)      # norm of the last step's gradients, and the factor that clipped them
        self.ws = torch.zeros(L.us_grad_norm_workspace_bytes(), dtype=torch.uint8, device=device)
        self._laid_out = None

    def _tensors(self) -> tuple:
        return tuple(t for c in (self.params, self.grads, self.m, self.v, self.m_scale, self.v_scale, self.copies) for t in c if t is not None)

    def _plan(self):
        """The descriptions of all tensors, made anew where one of them, or its decay, is another."""
        tensors, decay = self._tensors(), tuple(self.weight_decay)
        if self._laid_out is None or self._laid_out[0] != decay or not _binding.unchanged(tensors, *self._laid_out[1:3]):
            plan = L.adamw_tensors(self.params, self.grads, self.m, self.v, self.m_scale, self.v_scale, self.copies, weight_decay=self.weight_decay,
                                   rounding=self._rounding)
            self._laid_out = decay, tensors, tuple(t.data_ptr() for t in tensors), plan, L.mats(self.grads)
        return self._laid_out[3:]

    def step(self, stream=None) -> None:
        plan, grads = self._plan()
        if self.max_norm is not None:
            L.us_grad_norm(grads, self.max_norm, self.norm, self.ws, stream)
        L.us_adamw(plan, self.count, self.lr, self.betas, self.eps, self.lr_factor, self.norm[1:] if self.max_norm is not None else None, stream)

    @property
    def launches_per_step(self) -> int:
        """Kernel launches of step() (us_adamw describes 240 tensors to a launch, us_grad_norm 640)."""
        n = sum(p.numel() > 0 for p in self.params)
        return max(1, -(-n // 240)) + (max(1, -(-n // 640)) if self.max_norm is not None else 0)

    def state_dict(self) -> dict:
        """The states' own tensors."""
        return {"states": self.states, "m": self.m, "v": self.v, "m_scale": self.m_scale, "v_scale": self.v_scale, "count": self.count}

    def load_state_dict(self, d: dict) -> None:
        """Takes the values of another optimiser's states over the same parameters."""
        if d["states"] != self.states or [t.numel() for t in d["m"]] != [t.numel() for t in self.m]:
            raise ValueError("states of another kind, or of other parameters")
        for name in ("m", "v", "m_scale", "v_scale"):
            for mine, t in zip(getattr(self, name), d[name]):
                if mine is not None:
                    mine.copy_(t)
        self.count.copy_(d["count"])
