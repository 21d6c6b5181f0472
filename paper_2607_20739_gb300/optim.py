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
import sys

import numpy as np
import torch

from . import binding as B
from ._tensors import _TYPES, _address, _on, _vector

__all__ = ["AdamW"]

BLOCK = 256            # elements with a common scale, of moments in 8 bits

_dtype_of, _shape_of = operator.attrgetter("dtype"), operator.attrgetter("shape")
_device_of, _is_contiguous, _address_of = torch.Tensor.get_device, torch.Tensor.is_contiguous, torch.Tensor.data_ptr
# References that a tensor in a tuple has while they are counted, if it is in no other place.
_ALONE = max(map(sys.getrefcount, (torch.empty(0),)))

try:
    from torch._C._dynamo.guards import TensorGuards as _Guards
except ImportError:
    _Guards = None


def _guard(tensors):
    """A check(*tensors) that tensors have the shapes, strides, types and devices that these have, in one call of C."""
    return _Guards(*tensors, dynamic_dims_sizes=None, dynamic_dims_strides=None).check


def _guards_tell():
    """Whether torch has that check, and it tells what it is for."""
    try:
        t = torch.empty(4, 4)
        check = _guard([t])
        others = t[:2], t.t(), t.view(torch.int32), t.view(2, 8)
        return check(t) and check(torch.empty(4, 4)) and not any(check(o) for o in others)
    except Exception:                       # it is not a documented part of torch
        return False


if not _guards_tell():
    def _guard(tensors):  # noqa: F811
        return lambda *_: False


class _Layout:
    """Contiguous tensors of these shapes and types: with their addresses, what a table of them is right for."""

    def __init__(self, shapes, types):
        self._shapes, self._types, self._check, self._met = shapes, types, None, False

    def has(self, tensors):
        """As many tensors, laid out so.  What the check refuses may do all the same (it is stricter)."""
        if self._check is not None and self._check(*tensors):
            return True
        if list(map(_shape_of, tensors)) != self._shapes or list(map(_dtype_of, tensors)) != self._types or \
                not all(map(_is_contiguous, tensors)):
            return False
        if self._met:                       # the check costs more to make than a look
            self._check = _guard(tensors)
        self._met = True
        return True


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
    seed          of the chances that 8-bit moments are rounded by, which go by it, the step, a tensor's place in the list
                  and an element's in the tensor: optimizers of one seed draw the same ones
    state         moments and step to go on from, as ``state()`` returns them (the tensors
                  themselves are used); default: zeros
    device_step   the number of steps is kept on the device, so that a captured step
                  counts itself when it is replayed; without it a step under capture is refused.  Rates that
                  are floats, and the places of all tensors, are those of the capture in every replay

    All parameters decay alike; those that should not (norms, biases) are another optimizer's, with a seed of its own.
    Data of parameters, copies and moments may be exchanged between steps (``t.data = ...``, off the GPU and back
    for instance): the next step finds it, or refuses what does not go together.
    """

    def __init__(self, params, *, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, bits=32, copies=None, seed=0,
                 state=None, device_step=False):
        self.params = list(params)
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        self._check_params()
        self.device = self.params[0].device if self.params else None
        self.lr, self.betas, self.eps, self.weight_decay, self._bits, self.seed = lr, betas, eps, weight_decay, bits, seed
        self.copies = None if copies is None else _list("copies", copies, self.params, torch.bfloat16)
        self._moments = self._zeros() if state is None else self._given_moments(state)
        self._which = () if state is None else None         # who gave the moments may have them
        t = 0 if state is None else int(state["t"])
        if t < 0:
            raise ValueError("the number of steps must not be negative")
        self._next = None
        if device_step and self.params:
            with torch.inference_mode(False):
                # the number of the next step: raised behind a step that was taken
                self._next = torch.full((), t + 1, dtype=torch.int64, device=self.device)
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
        copies, moments, n = self.copies or [], self._moments, len(self.params)
        given = [*self.params, *copies]
        _refuse_overlaps([*given, *moments])
        self._given_at, self._kept_at = list(map(_address_of, given)), list(map(_address_of, moments))
        for i, p in enumerate(self.params):
            e = self._table[i]
            e.param, e.n, e.copy = self._given_at[i], p.numel(), self._given_at[n + i] if copies else None
            e.m, e.v = self._kept_at[i], self._kept_at[n + i]
            if self.bits == 8:
                e.m_scale, e.v_scale = self._kept_at[2 * n + i], self._kept_at[3 * n + i]
        # all of them have been checked
        self._shapes, self._gradients = list(map(_shape_of, self.params)), None
        self._given = _Layout(self._shapes * (len(given) // n if n else 0), [t.dtype for t in given[::n or 1] for _ in range(n)])
        self._kept = _Layout([shape(p) for _, _, shape in self._formats() for p in self.params],
                             [dtype for _, dtype, _ in self._formats() for _ in range(n)])
        self._watch(self._which)
        self._devices = list(map(_device_of, self.params))
        # inference tensors have no version
        self._versioned = [t for t in given if not t.is_inference()]

    def _watch(self, which):
        """The moments that the next steps look for where the table has them: all (None), or those numbers."""
        self._which = which
        self._watched = self._moments if which is None else tuple(self._moments[i] for i in which)
        self._at = self._given_at + (self._kept_at if which is None else [self._kept_at[i] for i in which])

    def _look(self):
        """Data of parameters, copies or moments that has been exchanged (``t.data = ...``) is looked over, and the table
        made anew.  Moments that nobody else has a reference to can move with their storage only: one of each is enough, and
        none where the storage was never anybody else's.  (A look is 0.06 to 0.1 us a tensor: 577 parameters 243 us a step; while
        somebody keeps their moments 430, with 8 bits 590.)"""
        given = [*self.params, *(self.copies or ())]
        if list(map(_address_of, (*given, *self._watched))) != self._at or not self._given.has(given) or \
                (self._which is None and not self._kept.has(self._moments)):
            if len(self.params) != len(self._table):
                raise ValueError(f"there must be {len(self._table)} parameters, not {len(self.params)}")
            self._check_params()
            if self.params[0].device != self.device:
                raise ValueError(f"params[0] is on {self.params[0].device}, not on {self.device}")
            if self.copies is not None:
                self.copies = _list("copies", self.copies, self.params, torch.bfloat16)
            self._given_moments(self._groups())
            self._fill()
        if self._which is None and max(map(sys.getrefcount, self._moments)) <= _ALONE:
            starts = [at - t.storage_offset() * t.element_size() for at, t in zip(self._kept_at, self._moments)]
            self._watch(list({start: i for i, start in enumerate(starts)}.values()))

    def _show(self):
        """Whoever has the moments may exchange their data."""
        if self._which is not None:
            self._watch(None)
        return self._groups()

    def _formats(self):
        """Of the groups of moments: name, type, shape beside a parameter."""
        same, blocks = (lambda p: tuple(p.shape)), (lambda p: (-(-p.numel() // BLOCK),))
        if self.bits == 32:
            return ("m", torch.float32, same), ("v", torch.float32, same)
        return (("m", torch.float8_e4m3fn, same), ("v", torch.uint8, same), ("m_scale", torch.float32, blocks),
                ("v_scale", torch.float32, blocks))

    def _zeros(self):
        with torch.inference_mode(False):
            return tuple(torch.zeros(shape(p), dtype=dtype, device=p.device) for _, dtype, shape in self._formats() for p in self.params)

    def _given_moments(self, groups):
        return tuple(t for name, dtype, shape in self._formats() for t in _list(name, groups[name], self.params, dtype, shape))

    def _groups(self):
        n = len(self._table)
        return {name: list(self._moments[i * n:(i + 1) * n]) for i, (name, _, _) in enumerate(self._formats())}

    @property
    def bits(self) -> int:
        """Of the moments."""
        return self._bits

    @property
    def m(self):
        """First moments, of each parameter."""
        return tuple(self._show()["m"])

    @property
    def v(self):
        """Second moments."""
        return tuple(self._show()["v"])

    @property
    def m_scale(self):
        """With 8 bits, the scales of the first moments' blocks."""
        return self._show().get("m_scale")

    @property
    def v_scale(self):
        return self._show().get("v_scale")

    @property
    def t(self) -> int:
        """Steps made (read from the device, and waited for, with device_step)."""
        return int(self._next.item()) - 1 if self._next is not None else self._t

    def state(self):
        """What ``state`` takes: the step and the moments (the tensors themselves)."""
        return {"t": self.t, **self._show()}

    def _addresses(self, grads):
        """The gradients' type and addresses, 0 for None; refuses what does not go with the parameters."""
        # A step of few elements lasts as long as this: gradients laid out as the last step's are looked at twice (0.1 us a
        # tensor), others five times, and one by one only where something is wrong.
        if self._gradients is not None and self._gradients(*grads):
            return self._gradient_type, np.fromiter(map(_address_of, grads), np.int64, len(grads))
        try:
            kinds = set(map(_dtype_of, grads))
            if len(kinds) == 1 and kinds <= _TYPES.keys() and list(map(_device_of, grads)) == self._devices and \
                    list(map(_shape_of, grads)) == self._shapes and all(map(_is_contiguous, grads)):
                self._gradients, self._gradient_type = _guard(grads), kinds.pop()
                return self._gradient_type, np.fromiter(map(_address_of, grads), np.int64, len(grads))
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
        if self.params:
            self._look()
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
        self._grads[:] = addresses

        def call(st):
            if self._next is None and torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a step that is captured needs device_step: replays would all be the same step")
            a = B.AdamW(0.0 if lr_at is not None else self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay,
                        self._t + 1, _address(self._next), _address(lr_at), _address(grad_scale),
                        self.seed & 0xffffffff, _TYPES[self.params[0].dtype], _TYPES[dtype], self.bits)
            B._check(B.lib.pgc_adamw_step(a, self._table, len(self._table), st), "pgc_adamw_step")
            if self._next is not None:
                self._next.add_(1)
        kept = ()
        if stream is not None:
            kept = [*self.params, *self._moments, *(self.copies or []), *grads, lr_at, grad_scale, self._next]
        _on(device, stream, kept, call)
        self._t += 1
        torch.autograd.graph.increment_version(self._versioned)
