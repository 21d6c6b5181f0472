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


def values(torch, o):
    """(m, v) of an optimizer's only tensor in 64 bits."""
    from oracle import training_oracle as O
    if o.bits == 32:
        return o.m[0].double(), o.v[0].double()
    of_v = torch.from_numpy(O.decode_v(np.arange(256))).cuda()[o.v[0].long()]
    return o.m[0].double() * o.m_scale[0].double().repeat_interleave(256), of_v * o.v_scale[0].double().repeat_interleave(256)


@pytest.mark.parametrize("beta2,steps", [(0.9, 300), (0.999, 6000)])
def test_noise_of_second_moments(cuda, optim, beta2, steps):
    """The spread of an 8-bit v about the one of 32 bits, for normal gradients.

    A rounding between codes a step s apart (relative to v: 1/32 to 1/16 for the large elements of a block, 1/16 to 1/8 for
    those below 2^-8 of the largest) at a place f between them has variance f (1 - f) s^2, and steps keep it as 1 / (1 - beta2^2).
      beta2 = 0.9: f is anywhere, f (1 - f) at most 1/4 and 1/6 in the mean:
        s / 2 / 0.436 at most 0.072, and 0.4 s / 0.436 at least 0.029.
      beta2 = 0.999: v starts on a code and moves by 0.001 |g^2 / v - 1|, 0.968 in the mean, so f (1 - f) s^2 is that times s:
        sqrt(0.000968 s / 0.002) between 0.123 and 0.174, up to f^2, 0.001 / s or 3 % of it.
    Twice that (0.999: sqrt 2) for the small ones.  A tenth for the scatter of g^2 about v."""
    torch = cuda
    n = 1 << 16
    p, q = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    a, b = (optim.AdamW([t], betas=(0.9, beta2), bits=bits, seed=3) for t, bits in ((p, 8), (q, 32)))
    small = torch.arange(n, device="cuda") % 2 == 1
    size = torch.where(small, 2.0 ** -6, 1.0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(steps):
        g = torch.randn(n, generator=gen, device="cuda") * size
        a.step([g])
        b.step([g])
    ratio = values(torch, a)[1] / values(torch, b)[1]
    lo, hi, more = (0.029, 0.072, 2.0) if beta2 == 0.9 else (0.123, 0.174, 2.0 ** 0.5)
    for on, f in ((~small, 1.0), (small, more)):
        mean, noise = float(ratio[on].mean()), float(ratio[on].std())
        assert 0.9 * f * lo < noise < 1.1 * f * hi, noise
        assert abs(mean - 1) < 6 * f * hi / (n / 2) ** 0.5 + 0.002


def test_parameters_of_8_bits_go_with_those_of_32(cuda, optim):
    """Of 200 steps, elements up to 2^9 smaller than their block's largest.  A rounding of m (half a step, 1/16 of |m| at most,
    which is 0.229 of sqrt(v) in the root mean square) stays for ten steps: 200^0.5 times 10 times 0.0143 lr is 0.0020.  The
    noise of v, 0.144 at most, is half of that in a step of 0.229 lr: 0.0033 even if it kept its sign in all 200.  Together 0.37 of
    the 0.0145 that 200 steps of noise move a parameter."""
    torch = cuda
    n = 1 << 16
    r = np.random.default_rng(5)
    size = torch.from_numpy(2.0 ** r.integers(-3, 7, n)).float().cuda()
    p, q = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    a, b = (optim.AdamW([t], betas=(0.9, 0.9), bits=bits, seed=3, weight_decay=0.0) for t, bits in ((p, 8), (q, 32)))
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(200):
        g = torch.randn(n, generator=gen, device="cuda") * size
        a.step([g])
        b.step([g])
    moved, apart = float(q.square().mean().sqrt()), float((p - q).square().mean().sqrt())
    assert apart < 0.4 * moved and float((p * q).sum()) > 0


def test_small_second_moments_are_raised(cuda, optim):
    """Below the lowest code, 1.25 2^-19 of the scale, a positive v is that code's; the next step goes by it."""
    torch = cuda
    from oracle import training_oracle as O
    n = 1024
    p = torch.zeros(n, device="cuda")
    g = torch.full((n,), 2.0 ** -14, device="cuda")
    g[::256] = 1.0
    g[5::256] = 0.0
    opt = optim.AdamW([p], bits=8, lr=1e-3, betas=(0.9, 0.999), eps=1e-12, weight_decay=0.0)
    opt.step([g])
    scale = float(opt.v_scale[0][0])
    v = values(torch, opt)[1]
    low = 1.25 * 2.0 ** -19 * scale
    assert low == float(O.decode_v(1)) * scale and 0.001 * 2.0 ** -28 < low
    tiny = torch.ones(n, dtype=torch.bool, device="cuda")
    tiny[::256] = tiny[5::256] = False
    assert (v[tiny] == low).all() and (v[5::256] == 0).all()
    before = p.clone()
    opt.step([g])
    # m' is between 0.9 and 1.1 of 0.19 g (its rounding) and v' almost the raised one: a step of m' / 0.19 / sqrt(v' / 0.001999)
    moved = (before - p).double()[tiny]
    want = 1e-3 * 2.0 ** -14 / np.sqrt((0.999 * low + 0.001 * 2.0 ** -28) / 0.001999)
    assert want < 0.5e-3 and ((moved > 0.85 * want) & (moved < 1.15 * want)).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32")])
def test_every_element_of_large_tensors(cuda, optim, bits, ptype, gtype):
    """All of a list's elements: equal to the step over pieces of it that are tensors of their own (8 bits, whose chances go by tensor and
    element: the parameters after one step), and the moments of 32 bits within their roundings of 64."""
    torch = cuda
    ptype, gtype = getattr(torch, ptype), getattr(torch, gtype)
    sizes, piece = [5_000_003, 1, 777, 9_000_000, 4_000_001, 300], 256 * 1237
    gen = torch.Generator(device="cuda").manual_seed(2)
    params = [(torch.randn(n + 1, generator=gen, device="cuda") * 0.05).to(ptype)[i == 4:][:n] for i, n in enumerate(sizes)]
    grads = [(torch.randn(n + 1, generator=gen, device="cuda") * 1e-3).to(gtype)[i == 4:][:n] for i, n in enumerate(sizes)]
    other = [p.clone() for p in params]
    cut = lambda ts: [t[i:i + piece] for t in ts for i in range(0, t.numel(), piece)]  # noqa: E731
    kw = dict(lr=1e-2, betas=(0.9, 0.95), weight_decay=0.1, bits=bits, seed=11)
    a, b = optim.AdamW(params, **kw), optim.AdamW(cut(other), **kw)
    for t in range(1 if bits == 8 else 2):
        a.step(grads)
        b.step(cut(grads))
        assert all(torch.equal(p, q) for p, q in zip(params, other))
        if bits == 8:
            continue
        for x, y in ((a.m, b.m), (a.v, b.v)):
            assert all(torch.equal(p, q) for p, q in zip(cut(x), y))
        for m, v, g in zip(a.m, a.v, grads):
            if t:
                continue
            g, u = g.double(), 2.0 ** -24
            assert ((m.double() - 0.1 * g).abs() <= 4 * u * 0.1 * g.abs() + 1e-44).all()
            assert ((v.double() - 0.05 * g * g).abs() <= 7 * u * 0.05 * g * g + 1e-44).all()
