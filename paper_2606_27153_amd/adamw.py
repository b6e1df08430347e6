"""AdamW for the parameters that ``Muon`` leaves out -- embedding tables, norms,
biases: many tensors in one launch, with states in 32 bits or in 8.

``adamw_step`` steps lists of tensors; ``AdamW`` is a torch.optim.Optimizer over
it.  A step only enqueues HIP kernels on torch's current stream of the tensors'
device.  What states in 8 bits hold, and how they are rounded, stands in
include/muon_adamw.h.
"""
from __future__ import annotations

import ctypes
import math
from typing import Dict, List, Optional, Sequence, Tuple, Union

import torch

from . import _adamw_lib as AL
from ._lib import MUON_BF16, MUON_F32

_DTYPES = {torch.float32: MUON_F32, torch.bfloat16: MUON_BF16}

State = Tuple[torch.Tensor, ...]


def new_state(param: torch.Tensor, bits: int = 32) -> State:
    """A parameter's state before its first step: ``(exp_avg, exp_avg_sq)`` in fp32,
    of its shape; or, of 8 bits, ``(exp_avg, exp_avg_sq, bases)``: uint8 codes of its
    elements in order, and an int16 pair for every 256 of them."""
    if bits == 32:
        return tuple(torch.zeros(param.shape, dtype=torch.float32, device=param.device) for _ in range(2))
    if bits != 8:
        raise ValueError(f"states of {bits} bits; 32 or 8 are supported")
    n = param.numel()
    code = lambda: torch.zeros(n, dtype=torch.uint8, device=param.device)
    return code(), code(), torch.zeros(-(-n // AL.MUON_ADAMW_BLOCK), 2, dtype=torch.int16, device=param.device)


def _check_state(state: State, n: int, i, device) -> int:
    """The bits of a state for n elements."""
    if not isinstance(state, (tuple, list)) or len(state) not in (2, 3):
        raise TypeError(f"state {i} must be a tuple of 2 tensors (32 bits) or 3 (8 bits)")
    small = len(state) == 3
    dtype = torch.uint8 if small else torch.float32
    for name, t in zip(("exp_avg", "exp_avg_sq"), state):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"state {i}'s {name} must be a tensor, not {type(t).__name__}")
        if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"state {i}'s {name} must be a contiguous {dtype} tensor of {n} elements")
        if t.device != device:
            raise ValueError(f"state {i}'s {name} is on {t.device}, expected {device}")
    if small:
        t, blocks = state[2], -(-n // AL.MUON_ADAMW_BLOCK)
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"state {i}'s bases must be a tensor, not {type(t).__name__}")
        if t.dtype != torch.int16 or t.shape != (blocks, 2) or not t.is_contiguous():
            raise ValueError(f"state {i}'s bases must be a contiguous int16 tensor of shape ({blocks}, 2)")
        if t.device != device:
            raise ValueError(f"state {i}'s bases is on {t.device}, expected {device}")
    return 8 if small else 32


def _one_by_one(params, grads, states, steps):
    """(the library's array of tensors as bytes, the device's index, the states' bits) with
    an exception for the first tensor that does not fit; gradients may be None."""
    device, bits, found, seen = None, None, [], {}
    for i in range(len(params)):
        p, g, s = params[i], grads[i], states[i]
        if not isinstance(p, torch.Tensor):
            raise TypeError(f"param {i} must be a tensor, not {type(p).__name__}")
        if device is None:
            device = p.device
            if not p.is_cuda:
                raise ValueError(f"param {i} is not on a GPU")
        pc = _DTYPES.get(p.dtype)
        if pc is None:
            raise TypeError(f"param {i} has dtype {p.dtype}; use float32 or bfloat16")
        if p.device != device:
            raise ValueError(f"param {i} is on {p.device}, expected {device}")
        if not p.is_contiguous():
            raise ValueError(f"param {i} is not contiguous (stride {p.stride()})")
        b = _check_state(s, p.numel(), i, device)
        for name, t in zip(("param", "exp_avg", "exp_avg_sq", "bases"), (p, *s)):
            first = seen.setdefault(t.data_ptr(), f"{name} {i}") if p.numel() else ""
            if first and first != f"{name} {i}":
                raise ValueError(f"{name} {i} is {first} again")
        if bits is None:
            bits = b
        elif b != bits:
            raise ValueError(f"state {i} has {b} bits, the ones before {bits}")
        if g is None:
            found.append(AL.muon_adamw_tensor(param_dtype=pc, grad_dtype=pc))
            continue
        if not isinstance(g, torch.Tensor):
            raise TypeError(f"grad {i} must be a tensor or None, not {type(g).__name__}")
        gc = _DTYPES.get(g.dtype)
        if gc is None:
            raise TypeError(f"grad {i} has dtype {g.dtype}; use float32 or bfloat16")
        if g.shape != p.shape or g.layout != torch.strided or not g.is_contiguous():
            raise ValueError(f"grad {i} must be contiguous and of param {i}'s shape {tuple(p.shape)}")
        if g.device != device:
            raise ValueError(f"grad {i} is on {g.device}, expected {device}")
        if not -1 << 63 <= steps[i] < 1 << 63:
            raise ValueError(f"step {steps[i]} of param {i} does not fit in 64 bits")
        found.append(AL.muon_adamw_tensor(p.data_ptr(), g.data_ptr(), s[0].data_ptr(), s[1].data_ptr(),
                                          s[2].data_ptr() if b == 8 else None, p.numel(), steps[i], pc, gc))
    return b"".join(map(bytes, found)), device.index, bits


def adamw_step(params: Sequence[torch.Tensor], grads: Sequence[Optional[torch.Tensor]], states: Sequence[State], *,
               step: Union[int, Sequence[int]], lr: float, betas: Tuple[float, float] = (0.9, 0.999),
               eps: float = 1e-8, weight_decay: float = 0.01, seed: int = 0) -> None:
    """One AdamW step of params (fp32 or bf16, contiguous, any shapes) in place, with
    their gradients (fp32 or bf16; None: the tensor is left as it is) and states
    (``new_state``; all of 32 bits or all of 8), which move on too.  ``step`` counts
    from 1 and is one number or one for each tensor; ``seed`` varies the rounding of 8-bit
    states.  All tensors are on one GPU and do not overlap.  As any write in place, a step makes
    autograd refuse a backward pass that would read a param as it was.  A step captured into a graph is
    replayed with the numbers it was captured with."""
    n = len(params)
    if len(grads) != n or len(states) != n:
        raise ValueError(f"{n} params, {len(grads)} grads and {len(states)} states")
    if not n:
        return
    steps = [int(step)] * n if not isinstance(step, (list, tuple)) else [int(s) for s in step]
    if len(steps) != n:
        raise ValueError(f"{len(steps)} steps for {n} params")
    tensors, index, bits = AL.tensors()(params, grads, states, steps) or _one_by_one(params, grads, states, steps)
    opts = AL.muon_adamw_opts(float(lr), float(betas[0]), float(betas[1]), float(eps), float(weight_decay), bits,
                              int(seed) & 0xFFFFFFFF)
    lib = AL.load()
    if index == torch._C._cuda_getDevice():
        AL.check(lib.muon_adamw_step(tensors, n, ctypes.byref(opts), torch._C._cuda_getCurrentRawStream(index)))
    else:
        with torch.cuda.device(index):
            AL.check(lib.muon_adamw_step(tensors, n, ctypes.byref(opts), torch._C._cuda_getCurrentRawStream(index)))
    AL.written(params, grads, states)


def state_values(state: State) -> Tuple[torch.Tensor, torch.Tensor]:
    """The averages ``(exp_avg, exp_avg_sq)`` that a state holds: itself in 32 bits; of
    8 bits the numbers its codes stand for, as bf16 vectors (which holds them exactly)."""
    first = state[0] if isinstance(state, (tuple, list)) and state else None
    if not isinstance(first, torch.Tensor):
        raise TypeError("a state is a tuple of 2 tensors (32 bits) or 3 (8 bits)")
    n, device = first.numel(), first.device
    if _check_state(state, n, "", device) == 32:
        return state[0], state[1]
    if not first.is_cuda:
        raise ValueError("the state is not on a GPU")
    lib = AL.load()
    with torch.cuda.device(device.index):
        m, v = (torch.empty(n, dtype=torch.bfloat16, device=device) for _ in range(2))
        AL.check(lib.muon_adamw_state_values(state[0].data_ptr(), state[1].data_ptr(), state[2].data_ptr(), n,
                                             m.data_ptr(), v.data_ptr(),
                                             torch._C._cuda_getCurrentRawStream(device.index)))
    return m, v


class AdamW(torch.optim.Optimizer):
    """torch.optim-style AdamW over fp32 or bf16 parameters of any shape (contiguous
    ones), for those that ``Muon`` does not step.  Per-parameter state: ``step``, ``exp_avg``,
    ``exp_avg_sq`` and, with ``state_bits=8``, ``bases``.  A parameter without a
    gradient is left as it is."""

    def __init__(self, params, lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, state_bits: int = 32, seed: int = 0):
        if not (math.isfinite(lr) and lr >= 0):
            raise ValueError(f"lr {lr} must be finite and not negative")
        if len(betas) != 2 or not all(0 <= b < 1 for b in betas):
            raise ValueError(f"betas {betas} must be two numbers in [0, 1)")
        if not (math.isfinite(eps) and eps >= 0):
            raise ValueError(f"eps {eps} must be finite and not negative")
        if not (math.isfinite(weight_decay) and weight_decay >= 0):
            raise ValueError(f"weight_decay {weight_decay} must be finite and not negative")
        if state_bits not in (32, 8):
            raise ValueError(f"states of {state_bits} bits; 32 or 8 are supported")
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay,
                                      state_bits=state_bits, seed=seed))

    def load_state_dict(self, state_dict) -> None:
        """As the base class, but the states keep their own types (the base class casts
        them to their parameter's, which codes and fp32 averages of bf16 ones are not)."""
        super().load_state_dict(state_dict)
        ids = [i for g in state_dict["param_groups"] for i in g["params"]]
        ours = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(ids, ours):
            held = state_dict["state"].get(i)
            if held is not None:
                self.state[p] = {k: v.detach().to(p.device, copy=True) if isinstance(v, torch.Tensor) else v
                                 for k, v in held.items()}

    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for index, group in enumerate(self.param_groups):
            per_device: Dict[int, Tuple[List, ...]] = {}
            for p in group["params"]:
                grad = p.grad
                if grad is None:
                    continue
                st = self.state[p]
                if not st:
                    st.update(zip(("exp_avg", "exp_avg_sq", "bases"), new_state(p, group["state_bits"])), step=0)
                params, grads, states, steps, held = per_device.setdefault(p.get_device(), ([], [], [], [], []))
                params.append(p)
                grads.append(grad if grad.layout != torch.strided else grad.contiguous())
                states.append((st["exp_avg"], st["exp_avg_sq"], st["bases"]) if "bases" in st else
                              (st["exp_avg"], st["exp_avg_sq"]))
                steps.append(st["step"] + 1)
                held.append(st)
            for params, grads, states, steps, held in per_device.values():
                # (groups differ in their rounding)
                adamw_step(params, grads, states, step=steps, lr=group["lr"], betas=group["betas"], eps=group["eps"],
                           weight_decay=group["weight_decay"], seed=group["seed"] + index * 0x632BE5AB)
                for st in held:     # (a step that was refused does not count)
                    st["step"] += 1
        return loss
