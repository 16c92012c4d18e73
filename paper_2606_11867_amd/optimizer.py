"""AdamW over the parameters of one rank, through foremoe_adamw_step: every
tensor in one call, first and second moments in 32 or 8 bits, fp32 masters of
bf16 weights, and the gradient accumulators cleared in the same pass (App.
A.4: bf16 weights, gradients accumulated in fp32 over the micro-steps of an
update step).
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple, Union

import torch

from . import _lib
from .api import _dt, _stream, _vec

F32 = torch.float32


class AdamW:
    """Parameters, their gradients and optimizer states of one GPU.

    params, grads: contiguous device tensors, grads[i] with params[i]'s
    elements; all params of one dtype, all grads of one dtype (fp32 or bf16).
    step() reads the gradients from these tensors each time, so they stay in
    place (as PolicyUpdate's dw_gate_up and dw_down do). With zero_grads it
    leaves them zero. A param or grad may be given other memory (.data = ...)
    of the same size and type, and the old memory is released by the next step;
    step() raises where it was given another type.
    weight_decay: one for all, or one per tensor.
    masters: fp32 copies that hold the values of bf16 params; True makes them,
    False does without (every step then rounds to bf16), or a list of tensors.
    state_bits: 32 (fp32 moments) or 8 (a byte each and a scale for every 256
    elements). states: per tensor (m, v), or (m, v, m_scale, v_scale) with 8
    bits, used in place; None starts from zero. step: steps done so far.
    params, grads, masters and states stay the tensors that they are: to load
    others' values, copy_ into them.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *, lr: float = 1e-3,
                 betas: Tuple[float, float] = (0.9, 0.95), eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.0, state_bits: int = 32,
                 masters: Union[bool, Sequence[torch.Tensor]] = True, states: Optional[Sequence[tuple]] = None,
                 step: int = 0, zero_grads: bool = False):
        self.lib = _lib.load()
        self._params, self._grads = tuple(params), tuple(grads)
        n = len(self.params)
        if n == 0:
            raise ValueError("no parameters")
        if len(self.grads) != n:
            raise ValueError("params and grads differ in number")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.lr, self.betas, self.eps = lr, tuple(betas), eps
        self._state_bits, self.n_steps, self.zero_grads = state_bits, int(step), bool(zero_grads)
        self.weight_decay = weight_decay
        dev = self.params[0].device
        self.device = dev
        bf16 = self.params[0].dtype == torch.bfloat16
        # the call's types: a tensor that is given other memory keeps its own
        self._dtypes = self.params[0].dtype, self.grads[0].dtype
        self._pdt, self._gdt = _dt(self.params[0]), _dt(self.grads[0])
        if masters is True:
            masters = [p.detach().to(F32) for p in self.params] if bf16 else None
        elif masters is False:
            masters = None
        elif not bf16:
            raise ValueError("masters go with bf16 parameters")
        # tensors of its own over the same memory: only params and grads can be
        # given other memory from outside
        self._masters = None if masters is None else tuple(t.detach() for t in masters)
        if states is None:
            states = [self._zero_state(p) for p in self.params]
        self._states = tuple(tuple(t.detach() for t in s) for s in states)
        if len(self.states) != n or (self.masters is not None and len(self.masters) != n):
            raise ValueError("masters and states: one per parameter")
        self._fill()

    # The tensors that the call's records were made of. They stay: values are
    # loaded into them (copy_).
    @property
    def params(self) -> Tuple[torch.Tensor, ...]:
        return self._params

    @property
    def grads(self) -> Tuple[torch.Tensor, ...]:
        return self._grads

    @property
    def masters(self) -> Optional[Tuple[torch.Tensor, ...]]:
        return self._masters

    @property
    def states(self) -> Tuple[Tuple[torch.Tensor, ...], ...]:
        return self._states

    @property
    def state_bits(self) -> int:
        return self._state_bits

    @property
    def weight_decay(self) -> List[float]:
        """One per tensor; like lr, betas and eps what the next step uses."""
        return self._weight_decay

    @weight_decay.setter
    def weight_decay(self, value: Union[float, Sequence[float]]) -> None:
        n = len(self.params)
        decay = [float(value)] * n if isinstance(value, (int, float)) else [float(w) for w in value]
        if len(decay) != n:
            raise ValueError("weight_decay: one for all, or one per tensor")
        self._weight_decay = decay

    def _zero_state(self, p: torch.Tensor) -> tuple:
        if self.state_bits == 32:
            return torch.zeros_like(p, dtype=F32), torch.zeros_like(p, dtype=F32)
        blocks = -(-p.numel() // _lib.ADAMW_BLOCK)
        return (torch.zeros(p.shape, dtype=torch.uint8, device=p.device),
                torch.zeros(p.shape, dtype=torch.uint8, device=p.device),
                torch.zeros(blocks, dtype=F32, device=p.device), torch.zeros(blocks, dtype=F32, device=p.device))

    def _fill(self) -> None:
        """The call's records, checked: whole, or those before."""
        dev, (pd, gd) = self.device, self._dtypes
        kinds = (F32, F32) if self.state_bits == 32 else (torch.uint8, torch.uint8, F32, F32)
        none = [None] * (4 - len(kinds))

        def at(t, n, dtype, name, i):
            if t.dtype == dtype and t.numel() == n and t.device == dev and t.is_cuda and t.is_contiguous():
                return t.data_ptr()
            return _vec(t, n, dtype, f"{name}[{i}]", dev)  # says what is wrong

        records = (_lib.AdamWTensor * len(self.params))()
        for i, (p, g, st) in enumerate(zip(self.params, self.grads, self.states)):
            n = p.numel()
            if len(st) != len(kinds):
                raise ValueError(f"states[{i}]: {len(kinds)} tensors expected")
            blocks = -(-n // _lib.ADAMW_BLOCK)
            records[i] = _lib.AdamWTensor(
                at(p, n, pd, "params", i), at(g, n, gd, "grads", i),
                at(self.masters[i], n, F32, "masters", i) if self.masters is not None else None,
                *[at(t, n if j < 2 else blocks, k, "states", i) for j, (t, k) in enumerate(zip(st, kinds))], *none,
                n, self._weight_decay[i])
        self._records = records
        # what the records point to stays allocated as long as they do: other
        # memory is then at another address, which is what step() looks at
        self._held = [t.detach() for t in (*self.params, *self.grads, *(self.masters or ()),
                                           *(t for st in self.states for t in st))]
        self._tensors = self.params + self.grads
        self._at = list(map(torch.Tensor.data_ptr, self._tensors))
        self._decay = list(self._weight_decay)

    def step(self, lr: Optional[float] = None, grad_scale: Optional[torch.Tensor] = None) -> None:
        """One step on the current stream. lr: from now on. grad_scale: a
        device fp32 scalar that every gradient is multiplied by (clipping,
        loss scaling). Captured in a graph, a replay is this step again, with
        this step's number, lr and tensors."""
        if lr is not None:
            self.lr = lr
        # a tensor was given other memory, or a weight decay was changed
        if list(map(torch.Tensor.data_ptr, self._tensors)) != self._at or self._weight_decay != self._decay:
            self._fill()
        _lib.check(self.lib.foremoe_adamw_step(
            self._records, len(self.params), self._pdt, self._gdt, self.state_bits, self.lr, *self.betas, self.eps,
            self.n_steps + 1, _vec(grad_scale, 1, F32, "grad_scale", self.device), self.zero_grads,
            _stream(self.device)), "foremoe_adamw_step")
        self.n_steps += 1
