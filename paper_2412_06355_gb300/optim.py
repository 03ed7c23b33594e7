"""AdamW over all parameters in one call of the library (dendsn_adamw_step)."""
from __future__ import annotations

import torch

from . import binding


class AdamW(torch.optim.Optimizer):
    """AdamW whose step is one launch over all tensors (two where it clips; for each 500 tensors).

    params: float32 or bfloat16 parameters on one CUDA device, or groups of them; groups may differ in
    weight_decay, the other options are one for all (a scheduler may change lr). state: m and v as "f32"
    or as "e4m3" codes with scales of 256 elements. max_norm: gradients are scaled down to this norm over
    all parameters (0: not); the last step's norm is in `grad_norm`, a tensor on the device. seed: of the
    random rounding of e4m3 states. A parameter without a gradient stays as it is. A step in a CUDA graph goes on
    with the lr, the weight decays and the gradients' memory that it was captured with; one step has to be made
    before, outside the graph.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, state="f32",
                 max_norm=0.0, seed=0):
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))
        self._options = dict(state=state, max_norm=max_norm, seed=seed)
        self._config()
        self._eight = state == "e4m3"
        ps = self._params()
        kind = binding.E4M3 if self._eight else torch.float32
        like = lambda p, n, dt: torch.zeros(n, dtype=dt, device=p.device)   # noqa: E731
        self._m = [like(p, p.numel(), kind) for p in ps]
        self._v = [like(p, p.numel(), kind) for p in ps]
        self._scales = [like(p, ((p.numel() + 255) // 256, 2), torch.float32) for p in ps] if self._eight else None
        self._step = torch.zeros(1, dtype=torch.int64, device=ps[0].device)
        self._plan, self._of = None, None
        self._captured = []          # plans whose tables CUDA graphs go on using
        self.grad_norm = None

    def _params(self):
        return [p for g in self.param_groups for p in g["params"]]

    def _config(self):
        one = self.param_groups[0]
        for g in self.param_groups:
            for name in ("lr", "betas", "eps"):
                if g[name] != one[name]:
                    raise ValueError(f"{name} has to be the same in all groups")
        return binding.make_adamw_config(float(one["lr"]), one["betas"], one["eps"], **self._options)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        cfg, ps = self._config(), self._params()
        if len(ps) != len(self._m):
            raise ValueError("parameters cannot be added after the first ones")
        decays = [g["weight_decay"] for g in self.param_groups for _ in g["params"]]
        of = ([p.data_ptr() for p in ps], decays)
        if self._plan is None or of != self._of:     # a parameter's memory or a decay was replaced
            self._plan = binding.adamw_plan(cfg, [p.detach() for p in ps], self._m, self._v, self._scales,
                                            weight_decay=decays)
            self._of = of
        grads = [p.grad if p.grad is None or p.grad.is_contiguous() else p.grad.contiguous() for p in ps]
        if torch.cuda.is_current_stream_capturing() and self._plan not in self._captured:
            self._captured.append(self._plan)
        self.grad_norm = binding.adamw_step(cfg, self._plan, grads, self._step)
        return loss

    def state_dict(self):
        groups = [{k: v for k, v in g.items() if k != "params"} for g in self.param_groups]
        return dict(step=self._step, m=self._m, v=self._v, scales=self._scales, param_groups=groups)

    def load_state_dict(self, kept):
        mine = self.state_dict()
        if len(kept["param_groups"]) != len(self.param_groups) or (kept["scales"] is None) != (self._scales is None):
            raise ValueError("the state is of other groups or of another kind of states")
        pairs = [(mine["step"], kept["step"])]
        for name in ("m", "v") + (("scales",) if self._eight else ()):
            if len(mine[name]) != len(kept[name]):
                raise ValueError(f"{name}: {len(kept[name])} tensors for {len(mine[name])} parameters")
            pairs += zip(mine[name], kept[name])
        for to, t in pairs:
            if to.shape != t.shape or to.dtype != t.dtype:
                raise ValueError(f"a state of {list(t.shape)} {t.dtype} for one of {list(to.shape)} {to.dtype}")
        with torch.no_grad():
            for to, t in pairs:
                to.copy_(t)
        for g, k in zip(self.param_groups, kept["param_groups"]):
            g.update(k)
