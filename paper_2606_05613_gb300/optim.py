"""AdamW on the resolved direction.

Argument marshalling and bookkeeping only: the norm and the step run in the CUDA
library (bkmoo_grad_norm, bkmoo_adamw).
"""
from __future__ import annotations

import numbers

import torch

from . import native


class AdamW:
    """Holds the moments of `params` (BucketMOO's, registration order) and steps
    them with the flat direction.

    state: "f32", or "e4m3" for 8-bit moments with a scale for every 256
    elements.  master: keep the weights in float32 beside bfloat16 parameters; the
    step goes from these, whatever the parameters have been set to since.
    weight_decay: one number, or one per parameter.  max_norm: clip the
    direction's norm to it; a step whose norm is not finite is skipped on the
    device (the step count moves on).  0 neither clips nor checks.

    Use:
        opt = AdamW(moo.params, lr=3e-4, max_norm=1.0, state="e4m3")
        ...
        opt.step(moo.finish())
    """

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.0, max_norm: float = 0.0, state: str = "f32", master: bool = False,
                 seed: int = 0):
        if state not in ("f32", "e4m3"):
            raise ValueError('state must be "f32" or "e4m3", got %r' % (state,))
        params = list(params)
        decay = weight_decay
        if not isinstance(decay, numbers.Real):
            decay = list(reversed(list(decay)))
        # the flat buffers hold the last registered parameter first
        self.tensors = native.TensorList(reversed(params), decay)
        N, dev = self.tensors.n_elems, torch.device("cuda", self.tensors.device)
        if master and self.tensors.dtype != torch.bfloat16:
            raise ValueError("a master copy goes with bfloat16 parameters")
        self.p = native.bkmoo_adamw_default_params()
        self.p.lr, self.p.eps, self.p.max_norm, self.p.seed = lr, eps, max_norm, seed
        self.p.beta1, self.p.beta2 = betas
        self.p.step = 0
        eight = state == "e4m3"
        self.m, self.v = (torch.zeros(N, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
                          if eight else torch.zeros(N, device=dev) for _ in range(2))
        self.m_scale, self.v_scale = (torch.zeros((N + 255) // 256, device=dev) if eight else None
                                      for _ in range(2))
        self.master = None
        if master:
            self.master = torch.cat([t.detach().reshape(-1) for t in self.tensors.tensors]).float()
        self.norm = torch.zeros((), device=dev)
        self._ws = torch.empty(native.BKMOO_NORM_WS_BYTES, dtype=torch.uint8, device=dev)

    def step(self, direction, lr: "float | None" = None) -> None:
        """One step with the flat direction (float32 or bfloat16).  lr: the rate from
        this step on."""
        before = self.p.step, self.p.lr
        if lr is not None:
            self.p.lr = lr
        self.p.step += 1
        try:
            norm = None
            if self.p.max_norm > 0:
                native.bkmoo_grad_norm(direction, self.norm, ws=self._ws)
                norm = self.norm
            native.bkmoo_adamw(self.tensors, direction, self.m, self.v, params=self.p,
                               master=self.master, m_scale=self.m_scale, v_scale=self.v_scale,
                               grad_norm=norm)
        except Exception:
            self.p.step, self.p.lr = before      # a refused step does not count
            raise
        # autograd does not see the kernel write: a backward pass over what these were fails
        torch.autograd.graph.increment_version(self.tensors.tensors)

    def state_dict(self) -> dict:
        return {"step": self.p.step, "seed": self.p.seed, "m": self.m, "v": self.v, "m_scale": self.m_scale,
                "v_scale": self.v_scale, "master": self.master}

    def load_state_dict(self, d: dict) -> None:
        for name in ("m", "v", "m_scale", "v_scale", "master"):
            mine, other = getattr(self, name), d[name]
            if (mine is None) != (other is None) or \
                    (mine is not None and (mine.dtype != other.dtype or mine.shape != other.shape)):
                raise ValueError("the state's %s does not fit this optimizer" % name)
        for name in ("m", "v", "m_scale", "v_scale", "master"):
            if d[name] is not None:
                getattr(self, name).copy_(d[name])
        self.p.step = int(d["step"])
        self.p.seed = int(d.get("seed", self.p.seed))
