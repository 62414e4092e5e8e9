"""AdamW over all tensors of a model in one launch (gws_adamw_step), as a torch optimizer."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding


class GaussWSAdamW(torch.optim.Optimizer):
    """AdamW for BF16 weights (a GaussWSLinear's, whose gradient is that of the sampled weight) and FP32 ones (b_i, whose decay is what pulls the bit-width to its target).

        optimizer = GaussWSAdamW(model.parameters(), lr=3e-4, moments=binding.ADAMW_8BIT)
        ...sampler.finish_backward(); optimizer.step(); optimizer.zero_grad(); sampler.advance()

    ``moments`` is ``binding.ADAMW_F32`` (8 bytes per weight) or ``ADAMW_8BIT`` (2 bytes and 1/32).  ``rest`` keeps the 16 bits that a 32-bit weight has below its BF16
    parameter, without which updates smaller than half the spacing of BF16 are lost; :meth:`weight` gives the 32-bit weight.  Parameter groups may differ in lr, betas,
    eps and weight_decay; groups that share the first three are stepped in one launch, and a step is refused for all groups or for none.  All parameters are on one CUDA device; parameters without a gradient are left alone, and a
    step counts for all others.  ``step(grad_scale=t)`` multiplies the gradients by an FP32 one-element tensor.  ``capturable`` keeps the count of steps on the device, so that a
    captured step can be replayed; a learning rate that is to change between replays is an FP32 one-element tensor on the device.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, moments: int = binding.ADAMW_F32, rest: bool = True,
                 capturable: bool = False):
        if moments not in (binding.ADAMW_F32, binding.ADAMW_8BIT):
            raise ValueError("gws: moments is ADAMW_F32 or ADAMW_8BIT")
        self._moments, self._rest, self._capturable = moments, bool(rest), bool(capturable)
        self._state: Optional[binding.AdamWState] = None
        self._count = 0                                   # steps taken; a tensor on the device if they may be captured
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))

    def add_param_group(self, param_group) -> None:
        if self.__dict__.get("_state") is not None:
            raise RuntimeError("gws: all parameter groups are added before the first step")
        super().add_param_group(param_group)
        g = self.param_groups[-1]
        if not isinstance(g["lr"], torch.Tensor) and g["lr"] < 0 or not 0 <= g["betas"][0] < 1 or not 0 <= g["betas"][1] < 1 or g["eps"] < 0 or g["weight_decay"] < 0:
            self.param_groups.pop()
            raise ValueError("gws: lr, eps and weight_decay are not negative, betas in [0, 1)")

    def _all(self):
        return [p for g in self.param_groups for p in g["params"]]

    def _prepare(self) -> binding.AdamWState:
        if self._state is None:
            params = self._all()
            rest = self._rest and any(p.dtype == torch.bfloat16 for p in params)
            self._state = binding.AdamWState([p.numel() for p in params], self._moments, rest=rest, device=params[0].device)
            if self._capturable and not isinstance(self._count, torch.Tensor):
                self._count = torch.full((1,), self._count, dtype=torch.int64, device=params[0].device)
        return self._state

    @torch.no_grad()
    def step(self, closure=None, grad_scale: Optional[torch.Tensor] = None):
        """One step; returns the closure's loss if there is one."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if torch.cuda.is_available() and torch.cuda.is_current_stream_capturing() and (not self._capturable or self._state is None):
            raise RuntimeError("gws: a captured step needs capturable=True and a step before the capture")
        params = self._all()
        grads = [p.grad for p in params]
        if any(g is not None and g.is_sparse for g in grads):
            raise RuntimeError("gws: gradients are dense")
        if all(g is None for g in grads):
            return loss
        state = self._prepare()
        on_device = isinstance(self._count, torch.Tensor)
        count = self._count if on_device else self._count + 1
        decays = [float(g["weight_decay"]) for g in self.param_groups for _ in g["params"]]
        kinds = [(id(g["lr"]) if isinstance(g["lr"], torch.Tensor) else g["lr"], tuple(g["betas"]), g["eps"]) for g in self.param_groups]
        calls = []
        for kind in dict.fromkeys(kinds):
            mine = [k == kind for k, g in zip(kinds, self.param_groups) for _ in g["params"]]
            group = self.param_groups[kinds.index(kind)]
            calls.append((grads if all(mine) else [g if m else None for g, m in zip(grads, mine)],
                          dict(lr=group["lr"], betas=group["betas"], eps=group["eps"], weight_decay=decays, step=count, grad_scale=grad_scale)))
        for some, more in calls[1:]:                      # a step is refused as a whole: what follows the first call, which checks itself, is checked before it
            more["checked"] = binding.adamw_check(params, some, state, **more)
        if on_device:
            count.add_(1)
        begun = False
        try:
            for some, more in calls:
                binding.adamw_step(params, some, state, **more)
                begun = True
        except Exception:                                 # a step that was refused does not count; one that a launch failed in the middle of does
            if on_device and not begun:
                count.sub_(1)
            if begun:
                self._count = count
            raise
        self._count = count
        return loss

    def weight(self, param: torch.Tensor) -> torch.Tensor:
        """The 32-bit weight that a parameter stands for."""
        for i, p in enumerate(self._all()):
            if p is param:
                return self._prepare().weight(i, p)
        raise KeyError("gws: not a parameter of this optimizer")

    def moments(self, param: torch.Tensor):
        """(m, v) of a parameter in FP32, in its shape."""
        for i, p in enumerate(self._all()):
            if p is param:
                state = self._prepare()
                at = state.starts[i]
                return tuple(t[at:at + p.numel()].view(p.shape) for t in state.values())
        raise KeyError("gws: not a parameter of this optimizer")

    def state_dict(self):
        out = super().state_dict()
        s = self._state
        out["gws"] = dict(count=int(self._count), moments=self._moments,
                          state=None if s is None else dict(sizes=list(s.sizes), moments=s.moments, units=s.units, rest=s.rest))
        return out

    @torch.no_grad()
    def load_state_dict(self, state_dict) -> None:
        """Takes over the state of an optimizer over tensors of the same sizes and with moments of the same format.  Count, moments, rest and a learning rate that is a tensor are
        written where they are, so that a captured step goes on from them; its betas, eps and decays stay those of its capture."""
        kept = state_dict.get("gws")
        if kept is None or kept["moments"] != self._moments:
            raise ValueError("gws: the state is of another optimizer or of another format of moments")
        sizes = [p.numel() for p in self._all()]
        s = kept["state"]
        if s is not None and list(s["sizes"]) != sizes:
            raise ValueError("gws: the state is of tensors of other sizes")
        rest = self._rest and any(p.dtype == torch.bfloat16 for p in self._all())
        if s is not None and (s["rest"] is not None) != rest:
            raise ValueError("gws: one of the optimizers keeps the rest of its weights, the other does not")
        rates = [g["lr"] for g in self.param_groups]
        self._check_rates(rates, state_dict["param_groups"])
        super().load_state_dict({k: v for k, v in state_dict.items() if k != "gws"})
        self._take_rates(rates)
        if isinstance(self._count, torch.Tensor):
            self._count.fill_(kept["count"])              # captured steps read it where it is
        else:
            self._count = kept["count"]
        if s is None:
            if self._state is not None:                   # zeros where they are, for captured steps
                for t in (self._state.moments, self._state.units, self._state.rest):
                    if t is not None:
                        t.zero_()
            return
        mine = self._prepare()
        for to, source in ((mine.moments, s["moments"]), (mine.units, s["units"]), (mine.rest, s["rest"])):
            if to is not None:
                to.copy_(source)

    def _check_rates(self, rates, groups) -> None:
        """Whether groups that share a rate's tensor are to take different rates, where a captured step may read it."""
        takes = {}
        for lr, group in zip(rates, groups):
            if isinstance(group["lr"], torch.Tensor) and group["lr"].numel() != 1:
                raise ValueError("gws: a learning rate is one number")
            if isinstance(lr, torch.Tensor) and takes.setdefault(id(lr), float(group["lr"])) != float(group["lr"]) and self._capturable and self._state is not None:
                raise ValueError("gws: groups share a learning rate on the device, of which captured steps may know, and the state has several")

    def _take_rates(self, rates) -> None:
        """The groups' loaded rates: into the tensors that the groups had, which captured steps read where they are; as numbers, or FP32 tensors beside the parameters, otherwise."""
        takes, moved = {}, {}
        for lr, group in zip(rates, self.param_groups):
            loaded = group["lr"]
            if isinstance(lr, torch.Tensor):
                rate = float(loaded)
                if takes.setdefault(id(lr), rate) != rate:
                    lr = torch.full_like(lr, rate)
                group["lr"] = lr.fill_(rate)
            elif isinstance(loaded, torch.Tensor):
                if id(loaded) not in moved:
                    moved[id(loaded)] = loaded.to(device=self._all()[0].device, dtype=torch.float32)
                group["lr"] = moved[id(loaded)]

    def __getstate__(self):
        return {**super().__getstate__(), "_moments": self._moments, "_rest": self._rest, "_capturable": self._capturable, "_state": self._state, "_count": self._count}
