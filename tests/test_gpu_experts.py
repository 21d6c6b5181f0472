"""Tokens to their experts and back against the 64-bit oracle.

Copies and whole numbers are equal.  u = 2^-24, h half a step of the rows' type: a sum of k
products adds at most (k + 1) u of their magnitudes, one of d products as
many as its chain is long (d / 32 + 64 at most, or d), and the result is rounded once."""

import numpy as np
import pytest

from oracle import training_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def experts(cuda):
    from paper_2607_20739_gb300 import experts
    return experts


def on_host(x):
    return x.double().cpu().numpy()


def choices(T, k, E, seed=0, empty=0.1):
    """Distinct experts a token, some favoured, some slots empty (-1, or beyond the experts)."""
    r = np.random.default_rng([seed, T, k, E])
    likes = r.standard_normal(E) + r.standard_normal((T, E))
    c = np.argsort(-likes, axis=1)[:, :k].astype(np.int32)
    if k > E:
        c = np.concatenate([c, r.integers(0, E, (T, k - E)).astype(np.int32)], 1)
    off = r.random((T, k)) < empty
    c[off] = np.where(r.random((T, k)) < 0.5, -1, E)[off]
    return c


def check_routes(r, choice, E):
    place, slot, offsets = O.route(choice, E)
    assert (r.place.cpu().numpy() == place).all()
    assert (r.slot.cpu().numpy() == slot).all()
    assert (r.offsets.cpu().numpy() == offsets).all()


@pytest.mark.parametrize("T,k,E", [(0, 1, 4), (1, 1, 1), (1, 8, 64), (2, 3, 1), (7, 3, 5), (31, 1, 8), (32, 1, 8), (33, 2, 40), (100, 64, 64),
                                   (100, 10, 6), (511, 2, 8), (1000, 4, 16), (2048, 8, 128), (2049, 8, 129), (5000, 8, 256), (4097, 4, 1024),
                                   (16384, 1, 7), (40000, 8, 384), (70000, 2, 1024)])
@pytest.mark.parametrize("empty", [0.0, 0.2])
def test_route(cuda, experts, T, k, E, empty):
    torch = cuda
    c = choices(T, k, E, empty=empty)
    check_routes(experts.route(torch.from_numpy(c).cuda(), E), c, E)


@pytest.mark.parametrize("T", [3, 1000, 60000])
def test_route_of_one_expert_or_none(cuda, experts, T):
    torch = cuda
    for value in (0, 9, -1, 10, 2 ** 31 - 1, -2 ** 31):
        c = np.full((T, 2), value, np.int32)
        check_routes(experts.route(torch.from_numpy(c).cuda(), 10), c, 10)


def place_of(torch, T, k, N, seed=0, empty=0.15):
    """Places of T k slots among N rows, all different; some outside."""
    r = np.random.default_rng([seed, T, k, N])
    order = r.permutation(max(N, T * k))[:T * k].astype(np.int32).reshape(T, k)
    order[r.random((T, k)) < empty] = -1
    order[r.random((T, k)) < 0.02] = 2 ** 31 - 1
    return order


def rows(torch, dtype, n, d, pad=0, shift=0, seed=0):
    r = np.random.default_rng([seed, n, d])
    store = torch.full((shift + n * (d + pad) + 3,), float("nan"), dtype=dtype, device="cuda")
    x = store.as_strided((n, d), (d + pad, 1), shift)
    x.copy_(torch.from_numpy(r.standard_normal((n, d)).astype(np.float32)))
    return x


def routes_of(torch, experts, place):
    T, k = place.shape
    return experts.Routes(T, k, 0, torch.from_numpy(place).cuda(), None, None)


WIDTHS = [1, 2, 3, 4, 7, 8, 9, 31, 64, 100, 255, 256, 257, 512, 1000, 1001, 2048, 2050, 4099, 8192, 20000]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,k,pad,shift", [(1, 1, 0, 0), (13, 8, 0, 0), (37, 3, 0, 1), (9, 64, 8, 0), (21, 5, 3, 2)])
def test_moves(cuda, experts, d, dtype, T, k, pad, shift):
    torch = cuda
    dtype = getattr(torch, dtype)
    h = torch.finfo(dtype).eps / 2
    for cut in (0, 3):
        N = max(1, T * k - cut)
        place = place_of(torch, T, k, N, seed=d)
        r = routes_of(torch, experts, place)
        x, dy, e = (rows(torch, dtype, n, d, pad, shift, seed) for seed, n in ((1, T), (2, T), (3, N)))
        w = torch.from_numpy(np.random.default_rng(d).standard_normal((T, k)).astype(np.float32)).cuda()
        xs, dys, es, ws = on_host(x), on_host(dy), on_host(e), on_host(w)
        on = (place >= 0) & (place < N)

        store = torch.full((shift + N * (d + pad) + 9,), 7.0, dtype=dtype, device="cuda")
        out = store.as_strided((N, d), (d + pad, 1), shift)
        assert experts.spread(x, r, out=out) is out
        want = np.full((N, d), 7.0)
        for t, j in np.argwhere(on):
            want[place[t, j]] = xs[t]
        assert (on_host(out) == want).all()
        out.fill_(7.0)
        assert (store == 7.0).all()                      # nothing beside the rows

        y, size = O.join(es, place, ws)
        got = on_host(experts.join(e, r, w))
        assert (np.abs(got - y) <= U * (k + 1) * size * (1 + h) + h * np.abs(y)).all()
        y, size = O.join(es, place)
        dx = experts.spread_grad(e, r, out=torch.empty_like(x))
        assert (np.abs(on_host(dx) - y) <= U * (k + 1) * size * (1 + h) + h * np.abs(y)).all()

        drows, dweight = experts.join_grad(dy, e, r, w, out=out)
        assert drows is out
        want, dw, size = O.join_grad(dys, es, place, ws)
        full = np.full((N, d), 7.0)
        for i, g in want.items():
            full[i] = g
        got = on_host(drows)
        assert (np.abs(got - full) <= (h + (2 * U if h > U else 0)) * np.abs(full)).all()
        chain = min(d, d / 32 + 64) + 1
        assert (np.abs(on_host(dweight) - dw) <= U * chain * size).all()
        assert (on_host(dweight)[~on] == 0).all()
        out.fill_(7.0)
        assert (store == 7.0).all()
        # in place of the experts' rows
        again, dweight2 = experts.join_grad(dy, e, r, w, out=e)
        assert again is e and torch.equal(dweight, dweight2)
        hit = sorted(want)
        assert (on_host(e)[hit] == got[hit]).all()


@pytest.mark.parametrize("T,k,E,d", [(1000, 8, 64, 256), (4000, 2, 8, 1024), (70000, 1, 16, 64), (300, 6, 256, 1001)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_there_and_back(cuda, experts, T, k, E, d, dtype):
    """Through route: weights that sum to 1 bring every token's own row back, up to roundings."""
    torch = cuda
    dtype = getattr(torch, dtype)
    c = choices(T, k, E, empty=0.0)
    r = experts.route(torch.from_numpy(c).cuda(), E)
    x = rows(torch, dtype, T, d)
    e = experts.spread(x, r)
    assert e.shape == (T * k, d)
    assert torch.equal(e, x[(r.slot // k).long()])
    y = experts.join(e, r, torch.full((T, k), 1.0 / k, device="cuda"))
    h = torch.finfo(dtype).eps / 2
    assert ((y.double() - x.double()).abs() <= (h + (k + 3) * U) * x.double().abs() * (1 + h)).all()


def test_special_values(cuda, experts):
    """Infinities and NaN stay in their rows; a row that no slot has is not read."""
    torch = cuda
    place = np.array([[0, 2], [1, -1]], np.int32)
    r = routes_of(torch, experts, place)
    e = torch.ones(4, 33, device="cuda")
    e[3] = float("nan")
    e[2, 5] = float("inf")
    w = torch.tensor([[1.0, 2.0], [3.0, float("nan")]], device="cuda")
    y = experts.join(e, r, w)
    assert y[0, 5] == float("inf") and torch.isfinite(y[0, :5]).all() and (y[1] == 3).all()
    drows, dw = experts.join_grad(torch.ones(2, 33, device="cuda"), e, r, w, out=torch.full_like(e, 9.0))
    assert (drows[0] == 1).all() and (drows[2] == 2).all() and (drows[1] == 3).all() and (drows[3] == 9).all()
    assert dw.tolist() == [[33.0, float("inf")], [33.0, 0.0]]


def test_no_tokens(cuda, experts):
    torch = cuda
    r = experts.route(torch.zeros(0, 4, dtype=torch.int32, device="cuda"), 8)
    x = torch.zeros(0, 16, device="cuda")
    assert (r.offsets == 0).all()
    e = experts.spread(x, r)
    assert e.shape == (0, 16) and experts.join(e, r).shape == (0, 16)
    # no rows at all: every token gets zeros
    r = routes_of(torch, experts, np.zeros((5, 2), np.int32))
    assert (experts.join(torch.zeros(0, 16, device="cuda"), r) == 0).all()
    drows, dw = experts.join_grad(torch.ones(5, 16, device="cuda"), torch.zeros(0, 16, device="cuda"), r, torch.ones(5, 2, device="cuda"))
    assert drows.shape == (0, 16) and (dw == 0).all()


def test_refusals(cuda, experts):
    torch = cuda
    c = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    r = experts.route(c, 8)
    x = torch.zeros(4, 16, device="cuda")
    e = torch.zeros(8, 16, device="cuda")
    w = torch.zeros(4, 2, device="cuda")
    for call in (lambda: experts.route(c.long(), 8), lambda: experts.route(c[:, 0], 8), lambda: experts.route(c.t(), 8),
                 lambda: experts.spread(x[:3], r), lambda: experts.spread(x.half(), r), lambda: experts.spread(x.t(), r),
                 lambda: experts.spread(x, r, out=e[:, :8]), lambda: experts.spread(x, r, out=e.bfloat16()),
                 lambda: experts.join(e, r, w[:3]), lambda: experts.join(e, r, w.double()), lambda: experts.join(e, r, out=x[:3]),
                 lambda: experts.join_grad(x[:, :8], e, r, w), lambda: experts.join_grad(x.bfloat16(), e, r, w),
                 lambda: experts.join_grad(x, e, r, w, out=e[:4])):
        with pytest.raises(ValueError):
            call()
    from paper_2607_20739_gb300 import PGCError
    with pytest.raises(PGCError):
        experts.route(c, 0)
    with pytest.raises(PGCError):
        experts.route(c, 1025)


def test_results_apart_from_the_rows(cuda, experts):
    """An out that shares elements with the arguments is refused; columns of one tensor beside one another are not."""
    torch = cuda
    T, k, d = 40, 1, 24
    c = torch.arange(T, device="cuda", dtype=torch.int32).flip(0)[:, None].contiguous()
    r = experts.route(c, T)
    w = torch.full((T, k), 2.0, device="cuda")
    wide = torch.randn(T, 3 * d + 1, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        buf = wide.to(dtype)
        x, y, z = buf[:, :d], buf[:, d:2 * d], buf[:, 2 * d:3 * d]
        for call in (lambda: experts.spread(x, r, out=x), lambda: experts.spread(x, r, out=buf[:, d - 1:2 * d - 1]),
                     lambda: experts.spread(y, r, out=buf[:, 1:d + 1]), lambda: experts.join(x, r, w, out=x),
                     lambda: experts.join(x[:5], r, w, out=buf[:, d // 2:d // 2 + d]),
                     lambda: experts.join_grad(x, y, r, w, out=x), lambda: experts.join_grad(x, y, r, w, out=buf[:, d + 1:2 * d + 1]),
                     lambda: experts.spread(buf.view(-1)[:T * d].view(T, d), r, out=y), lambda: experts.join_grad(x, x, r, w, out=x)):
            with pytest.raises(ValueError, match="share"):
                call()
        torch.cuda.synchronize()
        assert torch.equal(buf, wide.to(dtype))
        want = x.clone()
        experts.spread(x, r, out=y)
        assert torch.equal(y, want.flip(0)) and torch.equal(x, want)
        experts.join(y, r, w, out=z)
        assert torch.equal(z, 2 * want) and torch.equal(x, want)
        dx = experts.join_grad(x, y, r, w, out=z)[0]
        assert torch.equal(dx, 2 * want.flip(0)) and torch.equal(x, want) and torch.equal(y, want.flip(0))
        one = experts.route(c[:1] * 0, 1)
        assert torch.equal(experts.spread(x[3:4], one, out=x[4:5]), x[3:4])     # two rows of one tensor
        with pytest.raises(ValueError, match="share"):
            experts.spread(x[3:4], one, out=buf[3:4, d - 1:2 * d - 1])
        few = experts.route(c[:1] * 0, 1)
        assert torch.equal(experts.spread(x[3:4], few, out=z[2:6])[:1], x[3:4])   # a row and columns beside it
        with pytest.raises(ValueError, match="share"):
            experts.spread(x[3:4], few, out=buf[2:6, 1:d + 1])


def test_streams_and_graphs(cuda, experts):
    torch = cuda
    T, k, E, d = 3000, 8, 64, 130
    cs = [torch.from_numpy(choices(T, k, E, seed=s)).cuda() for s in (1, 2)]
    x = rows(torch, torch.bfloat16, T, d)
    w = torch.rand(T, k, device="cuda")

    def all_of(c):
        r = experts.route(c, E)
        e = experts.spread(x, r, out=torch.zeros(T * k, d, dtype=x.dtype, device="cuda"))
        y = experts.join(e, r, w)
        return [r.place, r.slot, r.offsets, e, y] + list(experts.join_grad(x, e, r, w, out=torch.zeros_like(e)))
    want = [all_of(c) for c in cs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = experts.route(cs[0], E, stream=side)
    y = experts.join(experts.spread(x, r, stream=side), r, w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(y, want[0][4])
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in cs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(all_of(c))
        graphs.append(graph)
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert all(torch.equal(p, q) for p, q in zip(got, ref))


def test_rows_beyond_32_bits(cuda, experts):
    """More than 2^31 elements of rows."""
    torch = cuda
    T, k, d = 33000, 2, 40000
    r = np.random.default_rng(0)
    place = r.permutation(T * k).astype(np.int32).reshape(T, k)
    routes = routes_of(torch, experts, place)
    x = torch.randn(T, d, device="cuda").bfloat16()
    e = experts.spread(x, routes)
    at = torch.from_numpy(place).cuda().long()
    for t in range(0, T, 4096):
        for j in range(k):
            assert torch.equal(e[at[t:t + 4096, j]], x[t:t + 4096])
    w = torch.tensor([[0.5, 0.5]], device="cuda").repeat(T, 1)
    assert torch.equal(experts.join(e, routes, w), x)
    drows, dw = experts.join_grad(x, e, routes, w, out=e)
    for t in range(0, T, 4096):
        assert torch.equal(drows[at[t:t + 4096, 1]], x[t:t + 4096] * 0.5)
    want = x[-1].double().square().sum()
    assert abs(float(dw[-1, 0]) - float(want)) <= U * (d / 32 + 65) * float(want)
    del x, e, drows
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,k,E", [(2048, 1, 16), (2049, 1, 16), (256, 8, 9), (257, 8, 9), (70000, 4, 31), (300000, 1, 33), (65536, 5, 1024)])
def test_route_of_sorted_and_blocked_choices(cuda, experts, T, k, E):
    """Choices that keep one expert in long runs: CTAs that hold only a few of the experts."""
    torch = cuda
    c = (np.arange(T * k) * E // (T * k)).astype(np.int32).reshape(T, k)
    for choice in (c, c[::-1].copy(), np.where(c % 3 == 1, -5, c).astype(np.int32)):
        check_routes(experts.route(torch.from_numpy(choice).cuda(), E), choice, E)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("k,d,pad,shift", [(1, 8, 0, 0), (2, 30, 0, 0), (3, 33, 0, 0), (3, 33, 3, 1), (5, 100, 4, 2), (9, 257, 0, 0), (8, 260, 0, 4), (4, 513, 1, 0)])
def test_moves_of_many_tokens(cuda, experts, dtype, k, d, pad, shift):
    """A token per warp."""
    torch = cuda
    dtype, T = getattr(torch, dtype), 5003
    h = torch.finfo(dtype).eps / 2
    N = T * k - 5
    place = place_of(torch, T, k, N, seed=d)
    r = routes_of(torch, experts, place)
    x, dy, e = (rows(torch, dtype, n, d, pad, shift, seed) for seed, n in ((1, T), (2, T), (3, N)))
    w = torch.from_numpy(np.random.default_rng(d).standard_normal((T, k)).astype(np.float32)).cuda()
    on = torch.from_numpy((place >= 0) & (place < N)).cuda()
    at = torch.from_numpy(np.where((place >= 0) & (place < N), place, 0)).cuda().long()
    token = torch.arange(T, device="cuda")[:, None].expand(T, k)
    out = torch.full((N, d), 7.0, dtype=dtype, device="cuda")
    experts.spread(x, r, out=out)
    want = torch.full((N, d), 7.0, dtype=dtype, device="cuda")
    want[at[on]] = x[token[on]]
    assert torch.equal(out, want)
    terms = e.double()[at] * w.double()[:, :, None] * on[:, :, None]
    y, size = terms.sum(1), terms.abs().sum(1)
    assert ((experts.join(e, r, w).double() - y).abs() <= U * (k + 1) * size * (1 + h) + h * y.abs()).all()
    drows, dweight = experts.join_grad(dy, e, r, w, out=torch.full((N, d), 7.0, dtype=dtype, device="cuda"))
    full = torch.full((N, d), 7.0, dtype=torch.float64, device="cuda")
    full[at[on]] = (w.double()[:, :, None] * dy.double()[:, None, :])[on]
    assert ((drows.double() - full).abs() <= (h + (2 * U if h > U else 0)) * full.abs()).all()
    terms = e.double()[at] * dy.double()[:, None, :] * on[:, :, None]
    chain = min(d, d / 32 + 64) + 1
    assert ((dweight.double() - terms.sum(2)).abs() <= U * chain * terms.abs().sum(2)).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,k,d", [(5000, 1, 2002), (5000, 2, 1030), (5100, 2, 769), (300, 2, 5001), (40, 1, 9000), (5000, 3, 1031), (5000, 5, 650),
                                   (5000, 6, 331), (200, 6, 4098), (5000, 7, 100)])
def test_moves_of_each_number_of_rows(cuda, experts, dtype, T, k, d):
    """The kernels' numbers of rows at once, with rows that are longer than a step of theirs and end inside one."""
    torch = cuda
    dtype = getattr(torch, dtype)
    r = routes_of(torch, experts, place_of(torch, T, k, T * k, seed=d))
    e, dy = rows(torch, dtype, T * k, d, seed=1), rows(torch, dtype, T, d, seed=2)
    w = torch.rand(T, k, device="cuda") + 0.5
    y = experts.join(e, r, w)
    de, dw = experts.join_grad(dy, e, r, w, out=torch.zeros_like(e))
    # on the host, where an index out of range is an error
    e, dy, w, y, de, dw, place = (t.double().cpu() if t.is_floating_point() else t.long().cpu() for t in (e, dy, w, y, de, dw, r.place))
    on = (place >= 0) & (place < T * k)
    taken = e[torch.where(on, place, 0)] * on[..., None]                         # [T, k, d]
    want = (taken * w[..., None]).sum(1)
    size = (taken.abs() * w[..., None]).sum(1)
    half = torch.finfo(dtype).eps / 2
    # k roundings of products and sums, then that of the result
    assert ((y - want).abs() <= (k + 1) * 2.0 ** -24 * size + half * want.abs() * (1 + 1e-6) + 1e-38).all()
    prod = taken * dy[:, None]
    # every sum of d terms in one order or another
    assert ((dw - prod.sum(2)).abs() <= (d + 2) * 2.0 ** -24 * prod.abs().sum(2) + 1e-38).all()
    want = torch.zeros_like(e)
    want[place[on]] = (w[..., None] * dy[:, None])[on]
    assert ((de - want).abs() <= (2.0 ** -24 + half) * want.abs() * (1 + 1e-6) + 1e-38).all()
