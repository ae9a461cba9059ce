"""The end of a training step: the norm of all gradients, which clips them, and
the AdamW update of the parameters, over libsppo's calls.

    opt = AdamW(params, {k: out["d" + k] for k in params}, lr=3e-4, max_norm=1.0)
    lay.step({"tokens": tokens, "targets": targets}, params, out)
    opt.step()

bf16 parameters get fp32 masters; the states are fp32 or 8-bit (e4m3 codes under
a power of two for 32 elements).  The update's number counts on the device, and
an update whose gradients hold an infinity or a NaN changes nothing and does not
count, so a step() may be captured into a graph and replayed.  The list of
tensors holds their addresses: gradients are to be written where they were, as a
layer's outputs are, and ones that are allocated anew need another list.  Only
C-ABI calls and torch allocations happen here.
"""
from __future__ import annotations

import torch

from . import sppo as L

_DTYPES = {torch.float32: "f32", torch.bfloat16: "bf16"}


class AdamW:
    def __init__(self, params, grads, lr, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, max_norm=None, state="f32",
                 decay=None, lr_scale=None, seed=0):
        """params, grads: tensors by the same names, of the same sizes,
        contiguous on one device, bf16 or fp32; their memory is what step()
        updates and reads.  decay: whether a name's tensor decays (by default
        those of two dimensions and more); lr_scale: factors of the learning
        rate by name.  seed: of the 8-bit states' rounding."""
        if set(params) != set(grads) or not params:
            raise ValueError("params and grads must have the same names, one at least")
        if state not in ("f32", "e4m3"):
            raise ValueError(f"unknown state {state!r}")
        if max_norm is not None and not max_norm > 0:
            raise ValueError("max_norm must be positive")
        self.betas, self.eps = betas, eps
        self._check()
        device = next(iter(params.values())).device
        for name, p in params.items():
            g = grads[name]
            for t in (p, g):
                if t.dtype not in _DTYPES or not t.is_contiguous() or t.device != device or not t.is_cuda:
                    raise ValueError(f"{name}: parameters and gradients must be contiguous bf16 or fp32 on one device")
            if p.numel() != g.numel():
                raise ValueError(f"{name}: the gradient has another size")
        for name in lr_scale or ():
            if name not in params:
                raise ValueError(f"lr_scale names {name!r}, which is no parameter")
        self.params, self.grads, self.device, self.state = dict(params), dict(grads), device, state
        self.lr, self.max_norm = lr, max_norm
        self.seed = seed
        zeros = lambda n, dt: torch.zeros(n, dtype=dt, device=device)  # noqa: E731
        self.master = {k: p.detach().float() for k, p in self.params.items() if p.dtype == torch.bfloat16}
        sdt = torch.float32 if state == "f32" else torch.uint8
        self.m = {k: zeros(p.numel(), sdt) for k, p in self.params.items()}
        self.v = {k: zeros(p.numel(), sdt) for k, p in self.params.items()}
        self.m_scale, self.v_scale = ({k: zeros(-(-p.numel() // 32), torch.uint8) for k, p in self.params.items()}
                                      if state == "e4m3" else {} for _ in range(2))
        tensors = []
        for k, p in self.params.items():
            wd = weight_decay if (p.dim() >= 2 if decay is None else decay(k)) else 0.0
            tensors.append(L.opt_tensor(p.numel(), self.grads[k], _DTYPES[self.grads[k].dtype], p, _DTYPES[p.dtype],
                                        self.master.get(k), self.m[k], self.v[k], self.m_scale.get(k),
                                        self.v_scale.get(k), (lr_scale or {}).get(k, 1.0), wd))
        self.norm = torch.zeros(2, dtype=torch.float32, device=device)  # of the last step: the norm, the factor
        self.steps = torch.zeros(1, dtype=torch.int64, device=device)   # updates made
        # The table's copy waits for all that was filled before it, so the first step() may be on any stream.
        self.list = L.opt_list(tensors, state, device)
        self.ws_bytes = L.sppo_grad_norm_workspace(self.list)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)

    def step(self, lr=None, stream=None):
        """One update on the stream (the current one of the parameters' device),
        with ``lr`` in the place of the optimizer's: a number, or a device fp32
        tensor of one, which a replayed graph reads anew."""
        lr = self.lr if lr is None else lr
        dev = isinstance(lr, torch.Tensor)
        if dev and (lr.dtype != torch.float32 or lr.numel() != 1 or lr.device != self.device):
            raise ValueError("an lr tensor must be one fp32 on the parameters' device")
        # What the update's call refuses is refused before the norm's call counts the update.
        if not dev and not L.scale_ok(lr, float("inf")):
            raise ValueError("lr must be finite")
        self._check()
        spec = L.adamw(1.0 if dev else lr, *self.betas, self.eps, 0, self.steps, self.norm, lr if dev else None,
                       self.seed)
        with torch.cuda.device(self.device):
            L.sppo_grad_norm(self.list, float("inf") if self.max_norm is None else self.max_norm, self.norm, self.ws,
                             self.ws_bytes, self.steps, stream)
            L.sppo_adamw_step(self.list, spec, stream)

    def _check(self):
        if len(self.betas) != 2 or not all(0.0 <= b < 1.0 for b in self.betas):
            raise ValueError("betas must be two in [0, 1)")
        if not self.eps > 0.0 or not L.scale_ok(self.eps, float("inf")) or L.scale_ok(self.eps, 2.0 ** -126):
            raise ValueError("eps must be positive and a normal fp32 number")

    def state_tensors(self):
        """The tensors that make up the optimizer's state beside the parameters,
        by name: what a checkpoint holds, and what is copied into to go on."""
        out = {"steps": self.steps}
        for kind in ("master", "m", "v", "m_scale", "v_scale"):
            out.update({f"{kind}.{k}": t for k, t in getattr(self, kind).items()})
        return out
