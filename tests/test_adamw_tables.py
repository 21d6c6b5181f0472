"""What optim.AdamW hands to the library, without a GPU: tensors of the host,
and in the library's place a step in numpy that goes by the table's addresses."""

import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")


def array(address, n, kind=C.c_float):
    return np.ctypeslib.as_array((kind * n).from_address(address))


@pytest.fixture(params=["torch's check", "lists"])
def optim(libpgc, monkeypatch, request):
    """optim.AdamW on the host; the calls that were made in optim.calls, as (step, sizes).  Also where torch
    has no check of layouts in one call."""
    from paper_2607_20739_gb300 import optim
    if request.param == "lists":
        monkeypatch.setattr(optim, "_guard", lambda tensors: lambda *_: False)
    calls, made, library = [], [], libpgc.lib.pgc_adamw_step
    begin = optim.AdamW.__init__

    def watched(self, *args, **kw):
        begin(self, *args, **kw)
        made.append(self)

    def extents():
        """Where an optimizer's tensors lie now."""
        for o in made:
            n = len(o.params)
            for t in zip(o.params, o._moments[:n], o._moments[n:]):
                assert all(x.is_contiguous() and x.dtype == torch.float32 and x.shape == t[0].shape for x in t)
                yield (*(x.data_ptr() for x in t), t[0].numel())

    def step(s, table, count, stream):
        code = library(s, table, 0, stream)                      # what it says of the rates
        if code:
            return code
        t = int(array(s.step_at, 1, C.c_int64)[0]) if s.step_at else s.step
        lr = array(s.lr_at, 1)[0] if s.lr_at else s.lr
        for e in table:
            if not e.grad or not e.n:
                continue
            assert (e.param, e.m, e.v, e.n) in extents()          # before anything is written
            assert s.bits == 32 and s.param_dtype == s.grad_dtype == libpgc.F32
            p, g, m, v = (array(a, e.n) for a in (e.param, e.grad, e.m, e.v))
            m[:] = s.beta1 * m + (1 - s.beta1) * g
            v[:] = s.beta2 * v + (1 - s.beta2) * g * g
            p[:] = p * (1 - lr * s.weight_decay) - lr * (m / (1 - s.beta1 ** t)) / (np.sqrt(v / (1 - s.beta2 ** t)) + s.eps)
        calls.append((int(t), [e.n for e in table]))
        return libpgc.OK
    monkeypatch.setattr(libpgc.lib, "pgc_adamw_step", step)
    monkeypatch.setattr(optim.AdamW, "__init__", watched)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(optim, "_on", lambda device, stream, tensors, call: call(None))
    monkeypatch.setattr(optim, "calls", calls, raising=False)
    return optim


def tensors(*shapes, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g) for s in shapes]


SHAPES = [(5, 5), (300,), (4, 7)]


def pair(optim, **kw):
    """Two optimizers of equal parameters, and gradients."""
    params = tensors(*SHAPES)
    other = [p.clone() for p in params]
    return params, other, optim.AdamW(params, **kw), optim.AdamW(other, **kw), tensors(*SHAPES, seed=1)


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("holds", ["a state", "a given state", "nothing"])
def test_exchanged_moments(optim, holds):
    """Moments whose data is moved off and back, between any two steps; where they lay nothing is written."""
    params, other, a, b, grads = pair(optim)
    if holds == "a given state":
        a = optim.AdamW(params, state={"t": 0, "m": [torch.zeros_like(p) for p in params], "v": [torch.zeros_like(p) for p in params]})
    kept = a.state() if holds == "a state" else None
    for _ in range(3):
        a.step(grads)
        b.step(grads)
        old = [t.data for t in a.m + a.v]
        before = [t.clone() for t in old]
        for t in (kept["m"] + kept["v"] if kept else a.m + a.v):
            t.data = t.data.clone()
        a.step(grads)
        b.step(grads)
        assert same(params, other) and same(a.m + a.v, b.m + b.v)
        assert same(old, before)
        del old


def test_moments_of_other_values(optim):
    """The next step goes on from what the moments hold, wherever that lies."""
    params, other, a, b, grads = pair(optim)
    a.step(grads)
    b.step(grads)
    for t, u in zip(a.m + a.v, b.m + b.v):
        t.data = t.data * 0.5
        u.mul_(0.5)
    a.step(grads)
    b.step(grads)
    assert same(params, other) and same(a.m + a.v, b.m + b.v)


def test_parameters_exchanged_before_the_moments_are_looked_at(optim):
    params, other, a, b, grads = pair(optim)
    a.step(grads)
    b.step(grads)
    old = [p.data for p in params]
    before = [p.clone() for p in old]
    for p in params:
        p.data = p.data.clone()
    a.state(), a.m
    a.step(grads)
    b.step(grads)
    assert same(params, other) and same(old, before)


@pytest.mark.parametrize("change", [lambda t: t.t(), lambda t: t[:3], lambda t: t.reshape(-1)[:20].view(4, 5), lambda t: t.view(torch.int32),
                                    lambda t: t.view(-1), lambda t: t.reshape(-1)[::2], lambda t: t.bfloat16(), lambda t: torch.zeros(5, 4)])
@pytest.mark.parametrize("which", ["param", "m", "v"])
def test_another_layout_is_refused(optim, change, which):
    """At the same address too; with gradients of the old shape or the new."""
    params, other, a, b, grads = pair(optim)
    a.step(grads)
    b.step(grads)
    t = {"param": params, "m": a.m, "v": a.v}[which][0]
    data = t.data
    t.data = change(data)
    before = data.clone(), [p.clone() for p in params]
    for g in (grads, [t.data.float(), *grads[1:]]):
        with pytest.raises(ValueError):
            a.step(g)
    assert torch.equal(data, before[0]) and same(params[1:], before[1][1:]) and a.t == 1
    t.data = data
    a.step(grads)
    b.step(grads)
    assert same(params, other) and same(a.m + a.v, b.m + b.v)


def test_parameters_and_moments_of_another_shape(optim):
    """Exchanged together they go on."""
    params, other, a, b, grads = pair(optim)
    a.step(grads)
    b.step(grads)
    for t in (params[1], a.m[1], a.v[1]):
        t.data = t.data[:200]
    grads[1] = grads[1][:200]
    a.step(grads)
    b.step([grads[0], torch.cat([grads[1], torch.zeros(100)]), grads[2]])
    assert optim.calls[-2][1] == [25, 200, 28]
    assert torch.equal(params[1], other[1][:200]) and torch.equal(a.m[1], b.m[1][:200])


def test_a_freed_storage_is_refused(optim):
    """Storage that was given back through a tensor that shares it."""
    flat = torch.zeros(64)
    params = tensors((8,), (9,))
    a = optim.AdamW(params, state={"t": 0, "m": [flat[:8], flat[16:25]], "v": [flat[32:40], flat[48:57]]})
    grads = tensors((8,), (9,), seed=1)
    a.step(grads)
    a.step(grads)
    flat.untyped_storage().resize_(0)
    with pytest.raises(Exception):
        a.step(grads)
    assert a.t == 2


def test_a_storage_that_moved(optim):
    """Moments that only the optimizer has, in a storage that somebody else makes larger: it lies elsewhere then."""
    flat = torch.zeros(64)
    params = tensors((8,), (9,))
    other = [p.clone() for p in params]
    a = optim.AdamW(params, state={"t": 0, "m": [flat[:8], flat[16:25]], "v": [flat[32:40], flat[48:57]]})
    b, grads = optim.AdamW(other), tensors((8,), (9,), seed=1)
    for n in (0, 1 << 20, 0, 1 << 26):
        if n:
            flat.untyped_storage().resize_(4 * n)
        a.step(grads)
        b.step(grads)
    assert same(params, other) and same(a.m + a.v, b.m + b.v)


def test_the_number_of_parameters_stays(optim):
    params, other, a, b, grads = pair(optim)
    a.step(grads)
    a.params.pop()
    with pytest.raises(ValueError, match="3 parameters"):
        a.step(grads[:2])
    a.params.pop()
    with pytest.raises(ValueError, match="3 parameters"):
        a.step(grads[:1])
    assert a.t == 1


@pytest.mark.parametrize("device_step", [False, True])
def test_a_refused_step_does_not_count(optim, device_step):
    """Whoever refuses it: the library the rates, the checks of tensors the rest."""
    from paper_2607_20739_gb300 import PGCError
    params, other, a, b, grads = pair(optim, device_step=device_step, betas=(0.9, 0.99))
    a.step(grads)
    b.step(grads)
    before = [p.clone() for p in params]
    for name, bad in (("lr", float("nan")), ("eps", -1.0), ("betas", (0.9, 1.0)), ("weight_decay", float("inf"))):
        good = getattr(a, name)
        setattr(a, name, bad)
        with pytest.raises(PGCError):
            a.step(grads)
        setattr(a, name, good)
    for bad in (grads[:2], [grads[0].double(), *grads[1:]], [None, grads[0], grads[2]]):
        with pytest.raises(ValueError):
            a.step(bad)
    assert a.t == a.state()["t"] == 1 and same(params, before)
    for _ in range(2):
        a.step(grads)
        b.step(grads)
    assert a.t == b.t == 3 and same(params, other) and [t for t, _ in optim.calls] == [1, 1, 2, 2, 3, 3]


def test_made_in_inference_mode(optim):
    """What the optimizer makes for itself may be changed outside of it."""
    params, grads = tensors(*SHAPES), tensors(*SHAPES, seed=1)
    other = [p.clone() for p in params]
    with torch.inference_mode():
        a = optim.AdamW(params, device_step=True)
        a.step(grads)
    b = optim.AdamW(other)
    b.step(grads)
    for t, u in zip(a.m + a.v, b.m + b.v):
        t.mul_(0.5)
        u.mul_(0.5)
    a.step(grads)
    b.step(grads)
    assert a.t == 2 and same(params, other)


def test_bits_stay(optim):
    """Those of the moments that were made: a step would read them as others'."""
    params, other, a, b, grads = pair(optim)
    with pytest.raises(AttributeError):
        a.bits = 8
    with pytest.raises(AttributeError):
        a.m = b.m
    assert a.bits == 32
    a.step(grads)
    b.step(grads)
    assert same(params, other)


def test_gradients_of_another_layout(optim):
    """Gradients may change their type, objects and places between steps, not their shapes or strides."""
    params, other, a, b, grads = pair(optim)
    for _ in range(3):
        a.step(grads)
        b.step([g.clone() for g in grads])
    for bad in (grads[0].t(), grads[0][:3], grads[0].view(-1), grads[0].double(), grads[0].bfloat16(), torch.zeros(5, 10)[:, ::2], 3.0):
        with pytest.raises((ValueError, TypeError)):
            a.step([bad, *grads[1:]])
        data, good = grads[0].data, isinstance(bad, torch.Tensor)
        if good:
            grads[0].data = bad
            with pytest.raises(ValueError):
                a.step(grads)
            grads[0].data = data
    for p in params + grads:
        p.requires_grad_(True)
    with torch.no_grad():
        a.step(grads)
    b.step([g.detach() for g in grads])
    for g in (grads, [None, *grads[1:]], grads):
        a.step(g)
        b.step(g)
    twice = [grads[0], grads[1], grads[0][:4, :].reshape(-1)[:1].expand(4, 7).contiguous()]
    a.step(twice)
    b.step(twice)
    assert a.t == b.t and same(params, other) and same(a.m + a.v, b.m + b.v)
