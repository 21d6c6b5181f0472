"""AdamW's state between steps on a GPU: data that is exchanged, steps that are refused."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def optim(cuda):
    from paper_2607_20739_gb300 import optim
    return optim


def pair(torch, optim, bits, sizes=((16, 16), (700,), (3, 1000)), **kw):
    """Two optimizers of equal parameters, and gradients."""
    r = np.random.default_rng(0)
    params, grads = ([torch.from_numpy(r.standard_normal(s).astype(np.float32)).cuda() for s in sizes] for _ in range(2))
    other = [p.clone() for p in params]
    return params, other, optim.AdamW(params, bits=bits, seed=5, **kw), optim.AdamW(other, bits=bits, seed=5, **kw), grads


def moments(o):
    return [*o.m, *o.v, *(o.m_scale or ()), *(o.v_scale or ())]


def same(torch, a, b):
    return all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a, b))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("holds", [False, True])
def test_moments_moved_off_and_back(cuda, optim, bits, holds):
    """To the host and back to another place; what lies at the old one is somebody else's by then."""
    torch = cuda
    params, other, a, b, grads = pair(torch, optim, bits)
    kept = moments(a) if holds else None
    for _ in range(2):
        a.step(grads)
        b.step(grads)
        old = [t.data for t in moments(a)]
        for t in kept or moments(a):
            t.data = t.data.cpu()
        for t in old:
            t.view(torch.uint8).fill_(7)
        for t in kept or moments(a):
            t.data = t.data.cuda()
        a.step(grads)
        b.step(grads)
        assert same(torch, params, other) and same(torch, moments(a), moments(b))
        assert all((t.view(torch.uint8) == 7).all() for t in old)


@pytest.mark.parametrize("bits", [32, 8])
def test_layouts_at_the_same_address(cuda, optim, bits):
    torch = cuda
    params, other, a, b, grads = pair(torch, optim, bits)
    a.step(grads)
    b.step(grads)
    for t in [params[0], *moments(a)[::3]]:
        data = t.data
        for change in (data.t() if data.dim() == 2 else data[::2], data[:1], data.view(torch.int16), data.view(-1)[:data.numel() // 2]):
            if change.shape == data.shape and change.dtype == data.dtype and change.is_contiguous():
                continue
            t.data = change
            with pytest.raises(ValueError):
                a.step(grads)
        t.data = data
    assert same(torch, params, other) and same(torch, moments(a), moments(b)) and a.t == 1
    a.step(grads)
    b.step(grads)
    assert same(torch, params, other) and same(torch, moments(a), moments(b))


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_on_the_host_are_refused(cuda, optim, bits):
    torch = cuda
    params, other, a, b, grads = pair(torch, optim, bits)
    a.step(grads)
    b.step(grads)
    for i in range(len(moments(a))):
        t = moments(a)[i]
        data, t.data = t.data, t.data.cpu()
        with pytest.raises(ValueError):
            a.step(grads)
        t.data = data
    a.step(grads)
    b.step(grads)
    assert same(torch, params, other) and a.t == 2


@pytest.mark.parametrize("device_step", [False, True])
def test_a_refused_step_does_not_count(cuda, optim, device_step):
    """Nor does it leave anything else behind: captured and replayed steps go on as if it had not been."""
    torch = cuda
    from paper_2607_20739_gb300 import PGCError
    params, other, a, b, grads = pair(torch, optim, 8, device_step=device_step)
    a.step(grads)
    b.step(grads)
    a.lr = float("nan")
    with pytest.raises(PGCError):
        a.step(grads)
    a.lr, a.eps = b.lr, -1.0
    with pytest.raises(PGCError):
        a.step(grads)
    a.eps = b.eps
    assert a.t == 1
    if device_step:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            a.step(grads)
        graph.replay()
        graph.replay()
    else:
        a.step(grads)
        a.step(grads)
    b.step(grads)
    b.step(grads)
    assert a.t == b.t == 3
    assert same(torch, params, other) and same(torch, moments(a), moments(b))
