"""AdamW as a torch optimizer: one launch per group and step over all its tensors (ue5m3_adamw), moments in 32 or in 8 bits, float32 master
copies of bfloat16 weights.

Nothing is computed here; states are made, handed over and kept.  Data-parallel replicas that start alike stay alike: the draws that 8-bit
moments are rounded by depend on the seed, the parameter's place, the step and the element only, not on the rank."""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import binding as B


class AdamW(torch.optim.Optimizer):
    """w = w (1 - lr weight_decay) - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps) for contiguous float32 and bfloat16 parameters.

    `state_bits` 32 or 8 (m as E4M3, v as UE5M3, a float32 scale per 256 elements, rounded stochastically: 2 bytes per weight in place of 8).  `eps` is at
    least 2^-126, or 0; with 8 bits at least 2^-50.
    `master_weights`: keep float32 copies of bfloat16 parameters (by default yes: bfloat16 alone loses updates below 2^-9 of a weight).  The copies are
    made at a parameter's first step; call `take_over_weights()` when parameters were changed from outside after that.
    `capturable`: the step is counted on the device, so that a captured `step()` goes on counting when it is replayed; take one step before the
    capture, which makes the states.  Every parameter that has a gradient is then counted as having had one in every step, and lr and the other numbers stay
    those of the capture."""

    def __init__(self, params, lr: float = 1e-3, betas: tuple = (0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 state_bits: int = 32, master_weights: bool = True, capturable: bool = False, seed: int = 0):
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits = {state_bits}: 8 or 32")
        if not lr >= 0 or not weight_decay >= 0 or not (eps >= (2.0 ** -50 if state_bits == 8 else 2.0 ** -126) or (eps == 0 and state_bits == 32)) or not all(0 <= b < 1 for b in betas):
            raise ValueError(f"lr {lr}, betas {betas}, eps {eps}, weight_decay {weight_decay}: out of range")
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                                      master_weights=bool(master_weights), capturable=bool(capturable), seed=int(seed)))

    def _begin(self, p: torch.Tensor, group: dict) -> dict:
        """The state of a parameter before its first step."""
        if p.is_cuda and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("take a step before the capture: a graph that makes the optimizer's states would make them anew at every replay")
        if not p.is_contiguous():
            raise ValueError("parameters have to be contiguous")
        state = self.state[p]
        if group["state_bits"] == 32:
            state["m"], state["v"] = (torch.zeros(p.shape, dtype=torch.float32, device=p.device) for _ in range(2))
        else:
            blocks = -(-p.numel() // B.ADAMW_BLOCK)
            state["m"], state["v"] = (torch.zeros(p.shape, dtype=torch.uint8, device=p.device) for _ in range(2))
            state["m_scale"], state["v_scale"] = (torch.zeros(blocks, dtype=torch.float32, device=p.device) for _ in range(2))
        if group["master_weights"] and p.dtype != torch.float32:
            state["master"] = p.detach().float()
        state["step"] = 0
        return state

    # A capturable group counts on the device: group["clocks"] has a counter per device, of which captured graphs know the address, so it is
    # kept for good.  While group["clocks_behind"] is set the parameters' own numbers are the ones that hold, else the counters are.
    def _read_clocks(self, group: dict) -> None:
        """The parameters' numbers become the counters'."""
        if group.get("clocks_behind"):
            return
        numbers = {device: int(clock[0]) for device, clock in group.get("clocks", {}).items()}
        for p in group["params"]:
            if p.device in numbers and self.state.get(p):
                self.state[p]["step"] = numbers[p.device]

    def _clock(self, group: dict, device: torch.device) -> torch.Tensor:
        """The counter of a capturable group on a device, at the most that one of its parameters has counted."""
        clocks = group.setdefault("clocks", {})
        if device not in clocks or group.get("clocks_behind"):
            if device.type == "cuda" and torch.cuda.is_current_stream_capturing():
                raise RuntimeError("take a step before the capture: it sets the counter on the device")
            if device not in clocks:
                clocks[device] = torch.zeros(B.ADAMW_CLOCK_BYTES // 8, dtype=torch.int64, device=device)
            for other, clock in clocks.items():
                if other == device or group.get("clocks_behind"):
                    clock[0] = max((self.state[p]["step"] for p in group["params"] if p.device == other and self.state.get(p)), default=0)
            group["clocks_behind"] = False
        return clocks[device]

    _notes = ()                                     # steps whose gradient scale the host has not seen yet: (its copy, when that is there, states)

    def _note(self, grad_scale: torch.Tensor) -> list:
        """Notes a step with this gradient scale; returns the list of the states that it counts in."""
        if grad_scale.is_cuda:
            with torch.cuda.device(grad_scale.device):
                value = torch.empty(1, dtype=torch.float32, pin_memory=True).copy_(grad_scale.view(1), non_blocking=True)
                there = torch.cuda.Event()
                there.record()
        else:
            value, there = grad_scale.clone(), None
        states: list = []
        self._notes = (*self._notes, (value, there, states))
        return states

    def _take_back(self) -> None:
        """The noted steps that were left out are not counted."""
        if self._notes and not (torch.cuda.is_available() and torch.cuda.is_current_stream_capturing()):
            notes, self._notes = self._notes, ()
            for value, there, states in notes:
                if there is not None:
                    there.synchronize()
                if not math.isfinite(float(value)):
                    for state in states:
                        state["step"] -= 1

    def __getstate__(self) -> dict:
        self._take_back()
        return super().__getstate__()

    @torch.no_grad()
    def step(self, closure=None, grad_scale: Optional[torch.Tensor] = None):
        """One step.  `grad_scale`: float32 tensor of one value that the gradients are multiplied by (a clipping factor, the inverse of a loss
        scale); where it is not finite the step changes nothing and is not counted.  (Without `capturable` its value is copied to the host and looked at
        when the next step begins, which waits for the copy.)"""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        self._take_back()
        note = None                                 # of what this step counts on the host, should it turn out to be left out
        place = 0                                   # of a parameter among all: the stream of its draws
        for group in self.param_groups:
            if not group["capturable"]:
                if any(p.is_cuda and p.grad is not None for p in group["params"]) and torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("a captured step wants capturable=True: this one would repeat its own number at every replay")
                if group.get("clocks") and not group.get("clocks_behind"):
                    self._read_clocks(group)        # the count goes on on the host
                    group["clocks_behind"] = True
            todo = {}                               # (device, step): parameters
            for p in group["params"]:
                place += 1
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("sparse gradients are not supported")
                state = self.state[p] or self._begin(p, group)
                todo.setdefault((p.device, 0 if group["capturable"] else state["step"] + 1), []).append((p, state, place - 1))
            for (device, step), some in todo.items():
                ps, states, places = zip(*some)
                clock = self._clock(group, device) if group["capturable"] else None
                col = lambda key: [s.get(key) for s in states]
                eight = group["state_bits"] == 8
                master = col("master")
                B.adamw(ps, [p.grad if p.grad.is_contiguous() else p.grad.contiguous() for p in ps], col("m"), col("v"), step, lr=group["lr"],
                        betas=group["betas"], eps=group["eps"], weight_decay=group["weight_decay"],
                        master=master if any(x is not None for x in master) else None, m_scale=col("m_scale") if eight else None,
                        v_scale=col("v_scale") if eight else None, grad_scale=grad_scale, seed=group["seed"], clock=clock, streams=places)
                torch.autograd.graph.increment_version(ps)        # a backward pass that still wants the old weights says so
                for state in states:                              # (a call that was refused is no step)
                    state["step"] += 1
                if grad_scale is not None and clock is None:
                    note = note or self._note(grad_scale)
                    note.extend(states)
        return loss

    @torch.no_grad()
    def take_over_weights(self) -> None:
        """The master copies become what the parameters are now (weights that were loaded after the first step)."""
        for p, state in self.state.items():
            if "master" in state:
                state["master"].copy_(p)

    def state_dict(self) -> dict:
        """As torch's; the number of the step on the device (capturable) comes out as each parameter's."""
        self._take_back()
        for group in self.param_groups:
            self._read_clocks(group)
        d = super().state_dict()
        d["state"] = {i: dict(state) for i, state in d["state"].items()}        # (tensors are the optimizer's own, as in torch)
        for group in d["param_groups"]:
            for key in ("clocks", "clocks_behind"):
                group.pop(key, None)
        return d

    def load_state_dict(self, state_dict: dict) -> None:
        """States keep their own types (torch's way casts them to the parameter's), and tensors that are there are written in place, so that
        captured graphs go on with what was loaded.  `capturable` becomes what was saved, like every number of a group."""
        clocks = [group.get("clocks") for group in self.param_groups]
        old = {p: self.state[p] for group in self.param_groups for p in group["params"] if self.state.get(p)}
        super().load_state_dict({**state_dict, "state": {}})
        self._notes = ()
        saved = [i for group in state_dict["param_groups"] for i in group["params"]]
        for i, p in zip(saved, [p for group in self.param_groups for p in group["params"]]):
            if i not in state_dict["state"]:
                continue
            new = {}
            for key, value in state_dict["state"][i].items():
                if torch.is_tensor(value):
                    there = old.get(p, {}).get(key)
                    if there is not None and there.shape == value.shape and there.dtype == value.dtype:
                        there.copy_(value)
                        value = there
                    else:
                        value = value.detach().to(p.device, copy=True)
                new[key] = value
            self.state[p] = new
        for group, there in zip(self.param_groups, clocks):
            if there:
                group["clocks"], group["clocks_behind"] = there, True
                if group["capturable"]:
                    for device in there:
                        self._clock(group, device)
