"""AdamW over a model's parameters on the library's operators (ops.adamw_step): one step over all
tensors at once, its averages in 32 or in 8 bits.

    opt = AdamW(model.parameters(), lr=2e-4, bits=8, max_norm=1.0)
    loss.backward(); opt.step(); opt.zero_grad()

Used by residual.train_residual and train.train_encoder.
"""
from __future__ import annotations

import torch

from . import ops


class AdamW:
    """params: tensors, as ops.AdamWState takes them. weight_decay is for matrices; vectors and scalars (biases,
    norms' weights) have none unless decay_vectors. bits: of the averages. master: an fp32 copy of 16-bit parameters is
    what a step updates. max_norm: the gradients' common norm is held to it, and a step whose norm is
    infinite or NaN is left out; `norm` is the last step's, on the device. seed: of the 8-bit
    averages' dither. lr may be set at any time, to a number or an fp32 CUDA tensor of one value (which a
    captured step reads)."""

    def __init__(self, params, lr=2e-4, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, bits=32, master=True,
                 max_norm=None, seed=0, decay_vectors=False):
        self.params = list(params)
        self.state = ops.AdamWState(self.params, bits=bits,
                                    master=master and any(p.dtype is not torch.float32 for p in self.params))
        self.lr, self.betas, self.eps, self.max_norm, self.seed = lr, betas, eps, max_norm, seed
        self.weight_decay = [float(weight_decay) if decay_vectors or p.dim() > 1 else 0.0 for p in self.params]
        self.norm = None

    @torch.no_grad()
    def step(self):
        """One step with the parameters' gradients; parameters without one stay as they are."""
        grads = [p.grad for p in self.params]
        # autograd brings an expanded or transposed gradient now and then
        grads = [g if g is None or g.is_contiguous() else g.contiguous() for g in grads]
        self.norm = ops.adamw_step(self.state, grads, self.lr, self.betas, self.eps, self.weight_decay, self.max_norm,
                                   self.seed)
        return self.norm

    def zero_grad(self):
        for p in self.params:
            p.grad = None

    def _shapes(self):
        return [tuple(p.shape) for p in self.params]

    def state_dict(self):
        """The averages, masters, step count, settings and the parameters' shapes and dtypes; the tensors are the
        optimizer's own."""
        s = self.state
        return {"bits": s.bits, "shapes": self._shapes(), "dtypes": [p.dtype for p in self.params], "m": s.m, "v": s.v,
                "master": s.master, "step": s.step, "lr": self.lr, "betas": self.betas, "eps": self.eps,
                "weight_decay": list(self.weight_decay), "max_norm": self.max_norm, "seed": self.seed}

    @torch.no_grad()
    def load_state_dict(self, d):
        """Takes over what state_dict gave, of an optimizer over tensors of the same shapes in the same order; copies."""
        s = self.state
        if d["bits"] != s.bits or (d["master"] is None) != (s.master is None):
            raise ValueError(f"state: averages in {d['bits']} bits {'without' if d['master'] is None else 'with'} masters, "
                             f"expected {s.bits} bits {'without' if s.master is None else 'with'}")
        pairs = [(s.step, d["step"])] + ([] if s.master is None else [(s.master, d["master"])])
        for mine, theirs in ((s.m, d["m"]), (s.v, d["v"])):
            pairs += [(mine, theirs)] if s.bits == 32 else list(zip(mine, theirs))
        # without shapes, as before they were saved: by the number of tensors and the sum of their sizes
        if [tuple(x) for x in d.get("shapes", self._shapes())] != self._shapes() or len(d["weight_decay"]) != len(self.params) or \
                any(a.shape != b.shape for a, b in pairs):
            raise ValueError("state: made for tensors of other sizes")
        if s.master is not None and any(a is torch.float32 and p.dtype is not a for a, p in zip(d.get("dtypes", []), self.params)):
            raise ValueError("state: made for fp32 tensors, which keep no masters, where these have 16 bits")
        for a, b in pairs:
            a.copy_(b)
        for k in ("betas", "eps", "max_norm", "seed"):
            setattr(self, k, d[k])
        self.weight_decay = list(d["weight_decay"])
        if isinstance(d["lr"], torch.Tensor) and isinstance(self.lr, torch.Tensor):
            self.lr.copy_(d["lr"])  # where a captured step reads it
        else:
            self.lr = d["lr"].to(s.step.device, copy=True) if isinstance(d["lr"], torch.Tensor) else d["lr"]


def of(name, params, lr, weight_decay=0.0, max_norm=None):
    """The optimizer that a training's `optimizer` names: "adam" (torch's), "adamw" or "adamw8" (this
    module's, averages in 32 or 8 bits)."""
    params = list(params)
    if name == "adam":
        if weight_decay or max_norm is not None:
            raise ValueError("weight_decay, max_norm: only with optimizer='adamw' or 'adamw8'")
        return torch.optim.Adam(params, lr=lr)
    if name not in ("adamw", "adamw8"):
        raise ValueError(f"optimizer: {name!r}, expected 'adam', 'adamw' or 'adamw8'")
    return AdamW(params, lr=lr, weight_decay=weight_decay, max_norm=max_norm, bits=8 if name == "adamw8" else 32)
