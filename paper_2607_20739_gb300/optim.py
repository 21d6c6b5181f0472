"""AdamW over many torch CUDA tensors at once, moments in 32 bits or in 8.

    opt = optim.AdamW(params, lr=3e-4, weight_decay=0.1, bits=8, copies=halves)
    opt.step(grads)                       # in place, one launch for up to 240 tensors

Thin layer over pgc_adamw_step (include/pgc.h, which has the formulas and the
8-bit formats).  Parameters are updated in place; their version counters are raised, so that
autograd refuses a backward pass over a graph that kept their older values.
"""

from __future__ import annotations

import ctypes as C
import operator

import numpy as np
import torch

from . import binding as B
from ._tensors import _TYPES, _address, _on, _vector

__all__ = ["AdamW"]

BLOCK = 256            # elements with a common scale, of moments in 8 bits

_dtype_of, _shape_of = operator.attrgetter("dtype"), operator.attrgetter("shape")
_device_of, _is_contiguous, _address_of = torch.Tensor.get_device, torch.Tensor.is_contiguous, torch.Tensor.data_ptr


def _list(name, tensors, params, dtype, shape_of=lambda p: tuple(p.shape)):
    """Refuses what is not a contiguous tensor of that type beside each parameter."""
    tensors = list(tensors)
    if len(tensors) != len(params):
        raise ValueError(f"{name} must have {len(params)} tensors, not {len(tensors)}")
    for i, (t, p) in enumerate(zip(tensors, params)):
        _vector(f"{name}[{i}]", t, dtype, shape_of(p), p.device)
    return tensors


def _refuse_overlaps(tensors):
    """Two tensors that share memory would be written by two threads at once."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors if t.numel())
    if any(end > start for (_, end), (start, _) in zip(spans, spans[1:])):
        raise ValueError("parameters, copies and moments must not share memory")


class AdamW:
    """One step of AdamW over a list of parameters.

    params        float32 or bfloat16 tensors of one type on one device, contiguous
    lr            float, or a float32 tensor of one element on the device (read by every step,
                  a captured one too).  The attribute may be set anew between steps, as betas, eps and weight_decay
    bits          of the moments: 32, or 8 (one byte an element and two scales per 256)
    copies        bfloat16 tensors shaped as the parameters that receive the updated values, or None
    seed          of the chances that 8-bit moments are rounded by
    state         moments and step to go on from, as ``state()`` returns them (the tensors
                  themselves are used); default: zeros
    device_step   the number of steps is kept on the device, so that a captured step
                  counts itself when it is replayed; without it a step under capture is refused.  Rates that
                  are floats are those of the capture in every replay
    """

    def __init__(self, params, *, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, bits=32, copies=None, seed=0,
                 state=None, device_step=False):
        self.params = list(params)
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        self._check_params()
        self.device = self.params[0].device if self.params else None
        self.lr, self.betas, self.eps, self.weight_decay, self.bits, self.seed = lr, betas, eps, weight_decay, bits, seed
        self.copies = None if copies is None else _list("copies", copies, self.params, torch.bfloat16)
        self._moments(state)
        t = 0 if state is None else int(state["t"])
        if t < 0:
            raise ValueError("the number of steps must not be negative")
        self._device_step = torch.full((), t, dtype=torch.int64, device=self.device) if device_step and self.params else None
        self._t = t
        self._table = (B.AdamWTensor * len(self.params))()
        # the column of the gradients' addresses
        self._grads = np.frombuffer(self._table, dtype=np.int64).reshape(-1, C.sizeof(B.AdamWTensor) // 8)[
            :, B.AdamWTensor.grad.offset // 8] if self.params else None
        self._fill()

    def _check_params(self):
        for i, p in enumerate(self.params):
            if not isinstance(p, torch.Tensor):
                raise TypeError(f"params[{i}] must be a torch tensor")
            if not p.is_cuda:
                raise ValueError(f"params[{i}] must be a CUDA tensor")
            if p.dtype not in _TYPES or p.dtype != self.params[0].dtype:
                raise ValueError("parameters must be float32 or bfloat16, all of one type")
            _vector(f"params[{i}]", p, p.dtype, tuple(p.shape), self.params[0].device)

    def _fill(self):
        """The table of all tensors but the gradients, from where they lie now."""
        copies = self.copies or []
        moments = [t for group in (self.m, self.v, self.m_scale or [], self.v_scale or []) for t in group]
        _refuse_overlaps(self.params + copies + moments)
        for i, p in enumerate(self.params):
            e = self._table[i]
            e.param, e.m, e.v, e.n = p.data_ptr(), self.m[i].data_ptr(), self.v[i].data_ptr(), p.numel()
            e.copy = copies[i].data_ptr() if copies else None
            if self.bits == 8:
                e.m_scale, e.v_scale = self.m_scale[i].data_ptr(), self.v_scale[i].data_ptr()
        self._shapes = [p.shape for p in self.params]
        self._devices = [p.get_device() for p in self.params]
        given = self.params + copies
        self._at = list(map(_address_of, given))
        # inference tensors have no version
        self._versioned = [t for t in given if not t.is_inference()]

    def _moved(self):
        """Parameters or copies whose data has been exchanged (``p.data = ...``): looked at anew."""
        self._check_params()
        for i, (p, shape) in enumerate(zip(self.params, self._shapes)):
            _vector(f"params[{i}]", p, p.dtype, shape, self.device)
        if self.copies is not None:
            self.copies = _list("copies", self.copies, self.params, torch.bfloat16)
        self._fill()

    def _moments(self, state):
        blocks = lambda p: (-(-p.numel() // BLOCK),)  # noqa: E731
        m_type, v_type = (torch.float32, torch.float32) if self.bits == 32 else (torch.float8_e4m3fn, torch.uint8)
        if state is None:
            self.m = tuple(torch.zeros(p.shape, dtype=m_type, device=p.device) for p in self.params)
            self.v = tuple(torch.zeros(p.shape, dtype=v_type, device=p.device) for p in self.params)
        else:
            self.m = tuple(_list("m", state["m"], self.params, m_type))
            self.v = tuple(_list("v", state["v"], self.params, v_type))
        self.m_scale = self.v_scale = None
        if self.bits == 8 and state is None:
            self.m_scale, self.v_scale = ([torch.zeros(blocks(p), dtype=torch.float32, device=p.device)
                                           for p in self.params] for _ in range(2))
        elif self.bits == 8:
            self.m_scale, self.v_scale = (_list(name, state[name], self.params, torch.float32, blocks)
                                          for name in ("m_scale", "v_scale"))

    @property
    def t(self) -> int:
        """Steps made (read from the device, and waited for, with device_step)."""
        return int(self._device_step.item()) if self._device_step is not None else self._t

    def state(self):
        """What ``state`` takes: the step and the moments (the tensors themselves)."""
        s = {"t": self.t, "m": list(self.m), "v": list(self.v)}
        if self.bits == 8:
            s["m_scale"], s["v_scale"] = list(self.m_scale), list(self.v_scale)
        return s

    def _addresses(self, grads):
        """The gradients' type and addresses, 0 for None; refuses what does not go with the parameters."""
        # A step of few elements lasts as long as this: five passes of C over the list (0.28 us a tensor), and the
        # loop that finds what is wrong only where something is.
        try:
            kinds = set(map(_dtype_of, grads))
            if len(kinds) == 1 and kinds <= _TYPES.keys() and list(map(_device_of, grads)) == self._devices and \
                    list(map(_shape_of, grads)) == self._shapes and all(map(_is_contiguous, grads)):
                return kinds.pop(), np.fromiter(map(_address_of, grads), np.int64, len(grads))
        except (TypeError, AttributeError):
            pass
        dtype = next((g.dtype for g in grads if isinstance(g, torch.Tensor)), torch.float32)
        if dtype not in _TYPES:
            raise ValueError("gradients must be float32 or bfloat16")
        for i, (g, shape) in enumerate(zip(grads, self._shapes)):
            if g is not None:
                _vector(f"grads[{i}]", g, dtype, shape, self.device)
        return dtype, [0 if g is None else g.data_ptr() for g in grads]

    def step(self, grads, *, grad_scale=None, stream=None):
        """One step.  grads: a tensor shaped as each parameter (float32 or bfloat16, one type), or None for a
        parameter that stays as it is.  grad_scale: factor of the gradients, a float32 tensor
        of one element on the device."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError(f"grads must have {len(self.params)} tensors, not {len(grads)}")
        dtype, addresses = self._addresses(grads)
        device = self.device
        lr_at = None
        if isinstance(self.lr, torch.Tensor):
            _vector("lr", self.lr, torch.float32, tuple(self.lr.shape), device)
            if self.lr.numel() != 1:
                raise ValueError("lr must have one element")
            lr_at = self.lr
        if grad_scale is not None:
            _vector("grad_scale", grad_scale, torch.float32, tuple(grad_scale.shape), device)
            if grad_scale.numel() != 1:
                raise ValueError("grad_scale must have one element")
        if not self.params:
            return
        if list(map(_address_of, self.params + (self.copies or []))) != self._at:
            self._moved()
        self._grads[:] = addresses

        def call(st):
            if self._device_step is not None:
                self._device_step.add_(1)
            elif torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a step that is captured needs device_step: replays would all be the same step")
            a = B.AdamW(0.0 if lr_at is not None else self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay,
                        self._t + 1, _address(self._device_step), _address(lr_at), _address(grad_scale),
                        self.seed & 0xffffffff, _TYPES[self.params[0].dtype], _TYPES[dtype], self.bits)
            B._check(B.lib.pgc_adamw_step(a, self._table, len(self._table), st), "pgc_adamw_step")
        kept = ()
        if stream is not None:
            kept = [self.params, self.m, self.v, self.m_scale or [], self.v_scale or [], self.copies or [], grads,
                    [lr_at, grad_scale, self._device_step]]
            kept = [t for group in kept for t in group]
        _on(device, stream, kept, call)
        self._t += 1
        torch.autograd.graph.increment_version(self._versioned)
