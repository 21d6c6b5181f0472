"""Tokens to their experts and back, for torch CUDA tensors.

A router's choice (``losses.balance_loss``) is sorted by expert; the tokens'
rows are copied in that order, so that the experts' products are made over
consecutive rows, and what the experts made of them is added at the tokens:

    r = experts.route(choice, n)              # choice int32 [tokens, k]
    rows = experts.spread(x, r)               # expert e: rows[r.offsets[e]:r.offsets[e + 1]]
    y = experts.join(made, r, weight)         # sum over k of weight times row

    dmade, dweight = experts.join_grad(dy, made, r, weight)
    dx = experts.spread_grad(drows, r)

Thin layer over the calls of include/pgc.h, as ``losses``; nothing here is
recorded by autograd.  Rows are float32 or bfloat16, their elements contiguous (any
row pitch); ``out`` is a tensor for the result that shares no element with the arguments; ``stream`` as
in ``losses``.
"""

from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B
from ._tensors import _TYPES, _address, _bytes, _matrix, _on, _vector

__all__ = ["Routes", "route", "spread", "spread_grad", "join", "join_grad"]


class Routes(NamedTuple):
    """Slots (token times k plus place in its choice) sorted by expert."""
    tokens: int
    k: int
    experts: int
    place: torch.Tensor      # int32 [tokens, k]: the row of each slot, -1 without an expert
    slot: torch.Tensor       # int32 [tokens * k]: the slot of each row, -1 behind the last
    offsets: torch.Tensor    # int32 [experts + 1]: first row of each expert, and the end


def route(choice, experts, *, stream=None):
    """Sorts the slots of choice (int32 [tokens, k]; entries outside [0, experts) hold nothing) by expert,
    in their order within one."""
    if not isinstance(choice, torch.Tensor):
        raise TypeError("choice must be a torch tensor")
    if not choice.is_cuda:
        raise ValueError("choice must be a CUDA tensor")
    if choice.dim() != 2:
        raise ValueError("choice must be [tokens, k]")
    tokens, k = choice.shape
    device = choice.device
    _vector("choice", choice, torch.int32, (tokens, k), device)
    if not 1 <= experts <= 1024:            # before it is cut to 32 bits
        raise B.PGCError(B.EINVAL if experts < 1 else B.ENOTSUP, "pgc_route")
    size = _bytes("pgc_route_workspace", tokens, k, experts)

    def call(st):
        place = torch.empty((tokens, k), dtype=torch.int32, device=device)
        slot = torch.empty(tokens * k, dtype=torch.int32, device=device)
        offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
        ws = torch.empty(size, dtype=torch.uint8, device=device)
        B._check(B.lib.pgc_route(tokens, k, experts, choice.data_ptr(), place.data_ptr(), slot.data_ptr(),
                                 offsets.data_ptr(), ws.data_ptr(), size, st), "pgc_route")
        return Routes(tokens, k, experts, place, slot, offsets)
    return _on(device, stream, (choice,), call)


def _rows(name, t, routes, count=None, like=None):
    """(rows, width, pitch) of a tensor of rows that goes with the routes."""
    rows, d, ld = _matrix(name, t, "elements")
    _vector("place", routes.place, torch.int32, (routes.tokens, routes.k), t.device)
    if count is not None and rows != count:
        raise ValueError(f"{name} must have {count} rows, not {rows}")
    if like is not None and (t.dtype != like.dtype or t.device != like.device or d != like.shape[1]):
        raise ValueError(f"{name} must have the type, device and width of the other rows")
    return rows, d, ld


def _share(a, b):
    """Whether two matrices of rows have an element in common."""
    (rows_a, d, ld_a), (rows_b, _, ld_b), size = _matrix("out", a), _matrix("rows", b), a.element_size()
    if not rows_a or not rows_b:
        return False
    start_a, start_b = a.data_ptr(), b.data_ptr()
    if start_a + ((rows_a - 1) * ld_a + d) * size <= start_b or start_b + ((rows_b - 1) * ld_b + d) * size <= start_a:
        return False
    if rows_a < 2 and rows_b < 2 or rows_a > 1 and rows_b > 1 and ld_a != ld_b:
        return True
    pitch = ld_a if rows_a > 1 else ld_b
    # columns beside one another in rows of a common pitch
    apart = (start_b - start_a) % (pitch * size)
    return not d * size <= apart <= (pitch - d) * size


def _same(a, b):
    """Whether the rows of two matrices are the same memory."""
    return a is not None and a.data_ptr() == b.data_ptr() and a.stride() == b.stride()


def _result(out, rows, routes, like, *inputs):
    """The tensor for `rows` rows and its pitch; made anew unless given, then apart from the inputs."""
    if out is None:
        d = like.shape[1]
        return torch.empty((rows, d), dtype=like.dtype, device=like.device), d
    ld = _rows("out", out, routes, rows, like)[2]
    if any(_share(out, t) for t in inputs):
        raise ValueError("out must not share memory with the other rows")
    return out, ld


def spread(x, routes, *, out=None, stream=None):
    """rows[place[t, j]] = x[t], [tokens * k, width].  Rows behind the last expert's are
    not written.  An out of fewer rows cuts those behind off."""
    _, d, ld = _rows("x", x, routes, routes.tokens)
    rows = routes.tokens * routes.k if out is None else _rows("out", out, routes, None, x)[0]

    def call(st):
        result, ldo = _result(out, rows, routes, x, x)
        B._check(B.lib.pgc_spread(_TYPES[x.dtype], routes.tokens, routes.k, d, x.data_ptr(), ld, routes.place.data_ptr(),
                                  rows, result.data_ptr(), ldo, st), "pgc_spread")
        return result
    return _on(x.device, stream, (x, routes.place, out), call)


def join(rows, routes, weight=None, *, out=None, stream=None):
    """y[t] = sum over j of weight[t, j] rows[place[t, j]]; weight float32 [tokens, k], ones if not given."""
    n, d, ld = _rows("rows", rows, routes)
    if weight is not None:
        _vector("weight", weight, torch.float32, (routes.tokens, routes.k), rows.device)

    def call(st):
        result, ldo = _result(out, routes.tokens, routes, rows, rows)
        B._check(B.lib.pgc_join(_TYPES[rows.dtype], routes.tokens, routes.k, d, rows.data_ptr(), ld, n,
                                routes.place.data_ptr(), _address(weight), result.data_ptr(), ldo, st), "pgc_join")
        return result
    return _on(rows.device, stream, (rows, routes.place, weight, out), call)


def spread_grad(drows, routes, *, out=None, stream=None):
    """Gradient of ``spread``: dx[t] = sum over j of drows[place[t, j]]."""
    return join(drows, routes, out=out, stream=stream)


def join_grad(dy, rows, routes, weight, *, out=None, stream=None):
    """Gradient of ``join`` for the derivative dy [tokens, width]: (drows, dweight).  Rows
    behind the last expert's are not written.  out may be rows itself."""
    n, d, ld = _rows("rows", rows, routes)
    _, _, ldy = _rows("dy", dy, routes, routes.tokens, rows)
    _vector("weight", weight, torch.float32, (routes.tokens, routes.k), rows.device)

    def call(st):
        drows, ldo = _result(out, n, routes, rows, dy, *(() if _same(out, rows) else (rows,)))
        dweight = torch.empty((routes.tokens, routes.k), dtype=torch.float32, device=rows.device)
        B._check(B.lib.pgc_join_grad(_TYPES[rows.dtype], routes.tokens, routes.k, d, dy.data_ptr(), ldy, rows.data_ptr(), ld,
                                     n, routes.place.data_ptr(), weight.data_ptr(), drows.data_ptr(), ldo,
                                     dweight.data_ptr(), st), "pgc_join_grad")
        return drows, dweight
    return _on(rows.device, stream, (dy, rows, routes.place, weight, out), call)
