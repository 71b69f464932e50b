"""AdamW over many tensors at once on torch CUDA tensors, with moments in 8 bits or in 32.

    optimizer = optim.AdamW(model.parameters(), lr=1e-4, bits=8)
    loss.backward(); optimizer.step(); optimizer.zero_grad()

``AdamW(params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, *, bits=8, seed=0, capturable=False)``
    a torch optimizer; the decay is apart from the gradient.  Parameters are BF16 or FP32, gradients either.  bits: of the moments.  With 8 a block of 128
    elements keeps E4M3 codes of the first moment and of the second's root and a power-of-two scale for each (2.02 bytes an element instead of 8).  Codes, and
    BF16 parameters, are rounded up or down at random so that what a step changes by less than half a distance of codes is not lost: ``seed``, the
    step's number, the parameter's place in the optimizer and the element's in it give the random numbers, so a run can be repeated and no two parameters
    share them.  ``step(grad_scale=None, found_inf=None)``: FP32 tensors of one value; the first multiplies every gradient, and where the second is not zero
    nothing is changed (the step still counts).  With capturable each parameter's steps are counted on the GPU (those of the group in its "step") and lr may be
    a tensor there, so that a captured step can be replayed; a parameter's first step has to be taken before the capture, and without capturable none is captured.
``adamw_(params, grads, exp_avgs, exp_avg_sqs, scales=None, *, step, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, seed=0, grad_scale=None,
found_inf=None, numbers=None)``
    one step over lists of contiguous tensors, changed in place (under torch.no_grad() where they require a gradient), none of them given twice or sharing
    memory with another; all parameters of one type, and all gradients.  The moments are FP32, or float8_e4m3fn with scales uint8 [blocks of 128, 2].  step: its
    number, from 1, or int32 on the GPU, one or one for each parameter; lr: a number, or one FP32 on the GPU.  numbers: one below 2^31 for each parameter, which
    its random numbers go by (None: its place in the list); parameters of one step that come in several calls want different ones.
``moments(exp_avg, exp_avg_sq, scales, dtype=torch.float32)``
    the values of 8-bit moments.

The formulas are those of ``include/mor.h``.
"""
from __future__ import annotations

import torch

from . import fp4  # noqa: F401  (raises if the operators have not been built)
from ._ops import adamw_
from ._ops import adamw_moments as moments

__all__ = ["AdamW", "adamw_", "moments"]


class AdamW(torch.optim.Optimizer):
    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, *, bits=8, seed=0, capturable=False):
        if bits not in (8, 32):
            raise ValueError("bits: 8 or 32 is wanted")
        if not all(0.0 <= b < 1.0 for b in betas):
            raise ValueError("betas: from 0 to below 1 are wanted")
        if not isinstance(lr, torch.Tensor) and not lr >= 0.0 or not eps >= 0.0 or not weight_decay >= 0.0:
            raise ValueError("lr, eps and weight_decay may not be negative")
        if isinstance(lr, torch.Tensor) and not capturable:
            raise ValueError("lr may be a tensor with capturable")
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay, bits=bits, seed=seed, capturable=capturable, step=None))

    def _new_state(self, p, bits):
        if bits == 32:
            return {"exp_avg": torch.zeros_like(p, dtype=torch.float32), "exp_avg_sq": torch.zeros_like(p, dtype=torch.float32)}
        code = dict(dtype=torch.float8_e4m3fn, device=p.device)
        return {"exp_avg": torch.zeros(p.shape, **code), "exp_avg_sq": torch.zeros(p.shape, **code),
                "scales": torch.full(((p.numel() + 127) // 128, 2), 127, dtype=torch.uint8, device=p.device)}

    def load_state_dict(self, state_dict):
        """As torch's, but the moments keep the types they were stored in (torch's brings them to the parameter's)."""
        super().load_state_dict(state_dict)
        stored, ids = state_dict["state"], [i for g in state_dict["param_groups"] for i in g["params"]]
        for i, p in zip(ids, (p for g in self.param_groups for p in g["params"])):
            if i in stored:
                self.state[p] = {k: v.clone().to(p.device) if isinstance(v, torch.Tensor) else v for k, v in stored[i].items()}
        for group in self.param_groups:
            kept = {}
            for p in group["params"]:
                if group["capturable"] and self.state.get(p):
                    state = self.state[p]
                    if not isinstance(state["step"], torch.Tensor) and state["step"] == 0 and group["step"] is not None:
                        state["step"] = int(group["step"])                     # stored when a group's parameters shared its count
                    kept.setdefault((p.device, p.dtype), []).append(state)
            for (device, _), states in kept.items():
                _count_together(states, device)
            if group["step"] is not None and group["params"]:
                group["step"] = group["step"].to(group["params"][0].device)

    @torch.no_grad()
    def step(self, closure=None, *, grad_scale=None, found_inf=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        self._check_capture()
        place = -1
        for group in self.param_groups:
            calls, capturable = {}, group["capturable"]
            for p in group["params"]:
                place += 1
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("sparse gradients are not supported")
                state = self.state[p]
                if not state:
                    state.update(self._new_state(p, group["bits"]))
                    state["step"] = 0
                if not capturable:
                    state["step"] = int(state["step"]) + 1
                calls.setdefault((p.device, p.dtype, p.grad.dtype, 0 if capturable else state["step"]), []).append((p, p.grad.contiguous(), state, place))
            if capturable and calls:
                steps = self._count(group, calls)
            for key, items in calls.items():
                with torch.cuda.device(key[0]):
                    step = key[3]
                    if capturable:
                        step = steps[key] if isinstance(steps[key], torch.Tensor) else torch.stack(steps[key])
                    adamw_([i[0] for i in items], [i[1] for i in items], [i[2]["exp_avg"] for i in items], [i[2]["exp_avg_sq"] for i in items],
                           [i[2]["scales"] for i in items] if group["bits"] == 8 else None, step=step, lr=group["lr"], beta1=group["betas"][0],
                           beta2=group["betas"][1], eps=group["eps"], weight_decay=group["weight_decay"], seed=group["seed"], grad_scale=grad_scale,
                           found_inf=found_inf, numbers=[i[3] for i in items])
        return loss

    def _check_capture(self):
        """A captured step whose number is the host's, or that makes its parameter's moments anew, would not go on from replay to replay."""
        params = ((group, p) for group in self.param_groups for p in group["params"] if p.grad is not None)
        for i, (group, p) in enumerate(params):
            if i == 0 and not (p.is_cuda and torch.cuda.is_current_stream_capturing()):
                return
            if not group["capturable"]:
                raise RuntimeError("a step can be captured with capturable=True only: its number would stay the same in every replay")
            if not isinstance(self.state.get(p, {}).get("step"), torch.Tensor) or group["step"] is None:
                raise RuntimeError("a parameter's first step has to be taken before a capture: every replay would begin with new moments")

    @staticmethod
    def _count(group, calls):
        """One more step on the GPU for the group and for each parameter in `calls`; for each call its parameters' counts, as one tensor where they lie in one."""
        if group["step"] is None:
            group["step"] = torch.zeros((), dtype=torch.int32, device=next(iter(calls))[0])
        steps, more = {}, {group["step"].device: [group["step"]]}
        for key, items in calls.items():
            states = [i[2] for i in items]
            fresh = [s for s in states if not isinstance(s["step"], torch.Tensor)]
            if fresh:
                _count_together(fresh, key[0])
            counts = [s["step"] for s in states]
            whole = counts[0]._base if counts[0]._base is not None else counts[0]
            if whole.numel() != len(counts) or not all(c.data_ptr() == whole.data_ptr() + 4 * i for i, c in enumerate(counts)):
                whole = counts
            steps[key] = whole
            more.setdefault(key[0], []).extend(whole if isinstance(whole, list) else [whole])
        for tensors in more.values():
            torch._foreach_add_(tensors, 1)
        return steps


def _count_together(states, device):
    """The steps of these parameters in one tensor on the GPU, an element each: one operation counts for all of them and a call reads them as they lie."""
    counts = [s["step"] for s in states]
    if any(isinstance(c, torch.Tensor) for c in counts):
        whole = torch.stack([c if isinstance(c, torch.Tensor) else torch.tensor(c, dtype=torch.int32, device=device) for c in counts]).to(torch.int32)
    elif any(counts):
        whole = torch.tensor(counts, dtype=torch.int32, device=device)
    else:
        whole = torch.zeros(len(counts), dtype=torch.int32, device=device)
    for i, s in enumerate(states):
        s["step"] = whole[i]
