"""Token scores against the 64-bit oracle.

Tolerances as in test_gpu_row_losses (u = 2^-24, D a class's distance from the
row's maximum over tau, rS the relative error of a sum of exponentials, eL that of L):
  W = sum e z / sum e, the mean of D under p: a term e z has e's error (4 D + 4) u and z's
    3 u, and the two sums their chains of additions, so
    eW = u (sum p D (4 D + 7) + W (chain + 2)) + W rS, and H = L + W: eL + eW + u |H|;
  q of a class: (x - m) / tau - L: 3 u D + eL + u |q|;
  gradient -p (a + b (q + H)) / tau + [v = y] a / tau: p's relative error, that of q + H
    times b p, 6 u of the magnitudes of its parts, then half a step of the output's type.
Where x leaves the range of u-accurate p (below 2^-126) both are 0 to 1e-37."""

import numpy as np
import pytest

from oracle import training_oracle as O
from test_gpu_row_losses import SIZES, U, half_step, make, on_host, rows_and_bounds

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def losses(cuda):
    from paper_2607_20739_gb300 import losses
    return losses


def bounds(x, y, tau):
    """(q, H, errors of q [rows, classes], of H, relative error of p)"""
    xs = on_host(x)
    q = O.log_probabilities(xs, tau)
    H = O.entropy(q)
    with np.errstate(all="ignore"):
        D = np.where(np.isfinite(xs), (xs.max(1, keepdims=True) - xs) / tau, 0.0)
        p = np.exp(q)
    V = xs.shape[1]
    L = -q.max(1)
    chain = min(V, 128 + V / 256)
    rS = U * ((4 * D * p).sum(1) + 4 + chain)
    eL = rS + 2 * U * np.abs(L)
    W = (p * D).sum(1)
    eW = U * ((p * D * (4 * D + 7)).sum(1) + W * (chain + 2)) + W * rS
    eH = eL + eW + U * np.abs(H)
    with np.errstate(all="ignore"):
        eq = U * (3 * D + np.where(np.isfinite(q), np.abs(q), 0.0)) + eL[:, None]
    ep = U * (4 * D + 12 + np.abs(L)[:, None]) + eL[:, None]
    return q, H, eq, eH, ep


def check_scores(torch, r, x, y, k, tau):
    q, H, eq, eH, _ = bounds(x, y, tau)
    T = len(q)
    ys = y.cpu().numpy() if y is not None else np.zeros(T, np.int32)
    on = ys >= 0
    if y is None:
        assert r["logp"] is None
    else:
        at = np.clip(ys, 0, q.shape[1] - 1)
        want, tol = q[np.arange(T), at], eq[np.arange(T), at]
        got = on_host(r["logp"])
        assert (got[~on] == 0).all()
        with np.errstate(invalid="ignore"):
            assert ((np.abs(got - want) <= tol) | (got == want) | ~on).all()
    got = on_host(r["entropy"])
    assert (got[~on] == 0).all() and (np.abs(got - H)[on] <= eH[on]).all(), (np.abs(got - H) / eH).max()
    want = O.top(on_host(x), k)
    want[~on] = -1
    top = r["top"].cpu().numpy()
    assert top.shape == (T, k) and (top == want).all()
    got = on_host(r["top_logp"])
    assert (got[want < 0] == -np.inf).all()
    t, j = np.nonzero(want >= 0)
    c = want[t, j]
    # (x - m) / tau of a class at -3.40e38 with tau = 0.8 is -4.25e38: -inf in single precision
    with np.errstate(over="ignore", invalid="ignore"):
        assert ((np.abs(got[t, j] - q[t, c]) <= eq[t, c]) | (got[t, j] == q[t, c].astype(np.float32))).all()
    st = on_host(r["stats"])
    assert (st[~on] == 0).all() and (st[on, 0] == on_host(x).max(1)[on]).all()


def check_gradient(torch, got, x, y, a, b, tau, stats=None):
    q, H, eq, eH, ep = bounds(x, y, tau)
    ys = y.cpu().numpy() if y is not None else np.zeros(len(q), np.int32)
    want = O.scores_gradient(on_host(x), None if y is None else ys, a, b, tau)
    with np.errstate(all="ignore"):
        p = np.exp(q)
        inner = np.where(p > 0, q + H[:, None], 0.0)
        error = np.where(p > 0, eq + eH[:, None], 0.0)
        size = np.abs(a)[:, None] + np.abs(b)[:, None] * (np.where(p > 0, np.abs(q), 0.0) + H[:, None])
        tol = p * (ep * np.abs(a[:, None] + b[:, None] * inner) + np.abs(b)[:, None] * error + 6 * U * size)
    if y is not None:
        t = np.flatnonzero(ys >= 0)
        tol[t, ys[t]] += 4 * U * np.abs(a[t])
    h = half_step(torch, got.dtype)
    tol = (tol / tau + h * np.abs(want)) * (1 + h) + 1e-37
    g = on_host(got)
    off = (ys < 0) | ((a == 0) & (b == 0))
    assert (g[off] == 0).all()
    err = np.abs(g - want)
    assert (err <= tol).all(), (np.argwhere(~(err <= tol))[:5], np.nanmax(err / tol))


def derivatives(torch, T, seed=1):
    r = np.random.default_rng([seed, T])
    a, b = (r.standard_normal(T).astype(np.float32) for _ in range(2))
    a[T // 2] = 0
    b[T // 3] = 0
    return a.astype(np.float64), b.astype(np.float64), torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda()


@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tau,k", [(1.0, 5), (0.7, 20)])
def test_sizes(cuda, losses, T, V, dtype, tau, k):
    torch = cuda
    _, x, y = make(torch, getattr(torch, dtype), T, V, masked=range(2, T, 5))
    r = losses.token_scores(x, y, k, tau)
    check_scores(torch, r, x, y, k, tau)
    a, b, da, db = derivatives(torch, T)
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, tau)
    assert g.dtype == x.dtype and g.is_contiguous()
    check_gradient(torch, g, x, y, a, b, tau)


@pytest.mark.parametrize("k", [0, 1, 2, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("T,V", [(3, 7), (2, 40), (3, 100), (2, 700), (3, 5001), (1, 70001)])
def test_numbers_of_alternatives(cuda, losses, k, T, V):
    torch = cuda
    for dtype in (torch.float32, torch.bfloat16):
        _, x, _ = make(torch, dtype, T, V, seed=k, shift=1)
        check_scores(torch, losses.token_scores(x, None, k), x, None, k, 1.0)


@pytest.mark.parametrize("T", [1, 2, 7, 40, 80, 160, 320, 700, 3000])
def test_numbers_of_rows(cuda, losses, T):
    """Few rows are shared by several CTAs, many are queued."""
    torch = cuda
    for V in (9000, 33000):
        if T * V > 30_000_000:
            continue
        _, x, y = make(torch, torch.bfloat16, T, V, masked=[T // 2])
        r = losses.token_scores(x, y, 3)
        check_scores(torch, r, x, y, 3, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V,pad,shift,out_pad,out_shift", [
    (7, 1000, 0, 1, 0, 1), (7, 1000, 8, 0, 0, 0), (7, 1001, 0, 3, 0, 3), (7, 1001, 5, 2, 2, 1), (5, 33, 1, 5, 3, 0),
    (9, 100, 0, 1, 0, 1), (9, 100, 1, 0, 0, 0), (9, 300, 2, 0, 4, 2), (5, 20003, 0, 1, 0, 1), (5, 20003, 6, 3, 1, 2),
    (4, 70001, 0, 7, 0, 7), (4, 70001, 0, 7, 0, 0), (3, 5, 0, 1, 0, 2)])
def test_pitches_and_alignments(cuda, losses, dtype, T, V, pad, shift, out_pad, out_shift):
    torch = cuda
    dtype = getattr(torch, dtype)
    _, x, y = make(torch, dtype, T, V, pad=pad, shift=shift, masked=[1])
    r = losses.token_scores(x, y, 4)
    check_scores(torch, r, x, y, 4, 1.0)
    a, b, da, db = derivatives(torch, T)
    outs = torch.full((out_shift + T * (V + out_pad) + 40,), 7.0, dtype=dtype, device="cuda")
    out = outs.as_strided((T, V), (V + out_pad, 1), out_shift)
    before = x.clone()
    assert losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, out=out) is out
    check_gradient(torch, out, x, y, a, b, 1.0)
    assert torch.equal(before, x)
    gaps = outs.clone()
    gaps.as_strided((T, V), (V + out_pad, 1), out_shift).fill_(7.0)
    assert (gaps == 7.0).all()
    # in place
    inside = losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, out=x)
    assert inside is x and torch.equal(x, out)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [5, 100, 700, 3001, 40000, 131072])
def test_masked_classes(cuda, losses, dtype, V):
    """Masked by -inf, by the type's lowest value, by -1e30 and -1e9: a class that has no part adds
    nothing; by -inf it is no alternative either."""
    torch = cuda
    dtype = getattr(torch, dtype)
    for value in (float("-inf"), float(torch.finfo(dtype).min), -1e30, -1e9):
        _, x, y = make(torch, dtype, 6, V)
        hide = torch.arange(V, device="cuda") % 3 != 1
        x[:3, hide] = value
        x[3, :] = value
        x[3, 2] = 1.5                                      # one class left: no entropy, the derivative 0
        y[:3] = 1
        y[3] = 2
        r = losses.token_scores(x, y, 3, 0.8)
        if value != float("-inf"):
            assert (r["top"][3] == torch.tensor([2, 0, 1], device="cuda")).all()
        check_scores(torch, r, x, y, 3, 0.8)
        a, b, da, db = derivatives(torch, 6)
        g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, 0.8)
        check_gradient(torch, g, x, y, a, b, 0.8)
        assert (g[:3, hide] == 0).all() and torch.isfinite(g).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [64, 1000, 20000])
def test_rows_without_a_distribution(cuda, losses, dtype, V):
    torch = cuda
    dtype = getattr(torch, dtype)
    _, x, y = make(torch, dtype, 5, V)
    x[0] = float("-inf")
    x[1, V // 2] = float("nan")
    x[2, 3] = float("inf")
    y[3] = V                                               # no class
    r = losses.token_scores(x, y, 2)
    assert torch.isnan(r["logp"][:4]).all() and torch.isfinite(r["logp"][4])
    assert torch.isnan(r["entropy"][:3]).all() and torch.isfinite(r["entropy"][3:]).all()
    assert (r["top"][0] == -1).all() and (r["top_logp"][0] == float("-inf")).all()
    assert r["top"][2, 0] == 3 and torch.isnan(r["top_logp"][1:3]).all()
    rest = x[1].float().clone()
    rest[V // 2] = float("-inf")
    assert (r["top"][1].cpu().numpy() == O.top(rest[None].double().cpu().numpy(), 2)[0]).all()
    one = torch.ones(5, device="cuda")
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], one, one)
    assert torch.isnan(g[:4]).all() and torch.isfinite(g[4]).all()
    # an entropy alone asks nothing of the target
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], one * 0, one)
    assert torch.isnan(g[:3]).all() and torch.isfinite(g[3:]).all()
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], one * 0, one * 0)
    assert (g == 0).all()
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], one * float("nan"), one * 0)
    assert torch.isnan(g).all()
    y[:] = -1
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], one * float("nan"), one)
    assert (g == 0).all()
    r = losses.token_scores(x, y, 2)
    assert (r["logp"] == 0).all() and (r["entropy"] == 0).all() and (r["stats"] == 0).all() and (r["top"] == -1).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [50, 900, 5000, 100003])
@pytest.mark.parametrize("k", [1, 20, 64])
def test_equal_logits(cuda, losses, dtype, V, k):
    """Ties to the lower class: all equal, two values, zeros of both signs, the largest ones last."""
    torch = cuda
    dtype = getattr(torch, dtype)
    x = torch.zeros(5, V, dtype=dtype, device="cuda")
    x[1, ::2] = 1.0
    x[2, 1::2] = -0.0
    x[3] = torch.arange(V, device="cuda").to(dtype)        # rising: every new one is an alternative
    x[4] = -torch.arange(V, device="cuda").to(dtype)
    check_scores(torch, losses.token_scores(x, None, k), x, None, k, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shift", [0.0, 300.0, -300.0, 3e8, -3e8])
def test_far_from_zero(cuda, losses, dtype, shift):
    torch = cuda
    dtype = getattr(torch, dtype)
    for V in (80, 3000, 40000):
        r_, x, y = make(torch, dtype, 4, V)
        x.copy_((x.float() * (1 if abs(shift) < 1e3 else 1e7) + shift).to(dtype))
        for tau in (1.0,) if abs(shift) < 1e3 else (1.0, 1e7):
            r = losses.token_scores(x, y, 6, tau)
            check_scores(torch, r, x, y, 6, tau)
            a, b, da, db = derivatives(torch, 4)
            g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, tau)
            check_gradient(torch, g, x, y, a, b, tau)


def test_agrees_with_the_log_probability(cuda, losses):
    """The same statistics as token_logprob's serve its gradient; one of the two derivatives alone."""
    torch = cuda
    _, x, y = make(torch, torch.float32, 20, 3001, masked=[4])
    r = losses.token_scores(x, y, 2)
    logp, stats = losses.token_logprob(x, y)
    _, _, _, _, elogp, _ = rows_and_bounds(x, y, 1.0)
    assert (np.abs(on_host(logp) - on_host(r["logp"])) <= 2 * elogp).all()
    a, b, da, db = derivatives(torch, 20)
    none = np.zeros(20)
    check_gradient(torch, losses.token_logprob_grad(x, y, r["stats"], da), x, y, a, none, 1.0)
    check_gradient(torch, losses.token_scores_grad(x, y, r["stats"], dlogp=da), x, y, a, none, 1.0)
    check_gradient(torch, losses.token_scores_grad(x, y, r["stats"], r["entropy"], dentropy=db), x, y, none, b, 1.0)
    free = losses.token_scores(x, None, 2)
    check_gradient(torch, losses.token_scores_grad(x, None, free["stats"], free["entropy"], dentropy=db), x, None, none, b, 1.0)


def test_no_rows(cuda, losses):
    torch = cuda
    x, y = torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    r = losses.token_scores(x, y, 3)
    assert r["top"].shape == (0, 3) and r["logp"].shape == (0,)
    assert losses.token_scores_grad(x, y, r["stats"], r["entropy"], r["logp"], r["logp"]).shape == (0, 10)


def test_streams_and_graphs(cuda, losses):
    """Calls on another stream, and captured: two graphs replayed at once have nothing in common; the same
    call gives the same bits."""
    torch = cuda
    _, x, y = make(torch, torch.bfloat16, 40, 50001, masked=[3])
    a, b, da, db = derivatives(torch, 40)

    def both(x):
        r = losses.token_scores(x, y, 7)
        return [r["logp"], r["entropy"], r["top"], r["top_logp"], losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db)]
    want, want2 = both(x), both(x + 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = losses.token_scores(x, y, 7, stream=side)
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(r["top"], want[2]) and torch.equal(g, want[4])
    x2 = x + 1
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for inp in (x, x2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(both(inp))
        graphs.append(graph)
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, (want, want2)):
        for p, q in zip(got, ref):
            assert torch.equal(p, q)


def test_classes_beyond_32_bits_of_bytes(cuda, losses):
    """Rows whose elements lie beyond 2^31 from the first one's."""
    torch = cuda
    T, V, ld = 3, 70001, 1 << 30
    store = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((T, V), (ld, 1))
    _, small, y = make(torch, torch.bfloat16, T, V)
    x.copy_(small)
    r = losses.token_scores(x, y, 4)
    check_scores(torch, r, small, y, 4, 1.0)
    a, b, da, db = derivatives(torch, T)
    g = losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, out=x)
    check_gradient(torch, g, small, y, a, b, 1.0)
    del store, x, g
    torch.cuda.empty_cache()


def some_rows(torch, r, x, y, rows):
    at = torch.tensor(rows, device="cuda")
    part = {k: None if v is None else v[at] for k, v in r.items()}
    return part, x[at], None if y is None else y[at]


@pytest.mark.parametrize("dtype,V", [("bfloat16", 2500), ("bfloat16", 9000), ("bfloat16", 33001), ("float32", 1200), ("float32", 9001), ("float32", 17000)])
@pytest.mark.parametrize("k", [0, 1, 20, 32, 33, 64])
def test_many_longer_rows(cuda, losses, dtype, V, k):
    """So many rows that a warp takes one of up to 72 KB: against the oracle here and there, special rows among them, and
    against the calls on fewer rows everywhere."""
    torch = cuda
    dtype, T = getattr(torch, dtype), 5200
    g = torch.Generator(device="cuda").manual_seed(V + k)
    x = torch.empty(T, V, dtype=dtype, device="cuda")
    for t in range(0, T, 400):
        x[t:t + 400] = torch.randn((400, V), generator=g, device="cuda") * 2
    y = torch.randint(V, (T,), generator=g, device="cuda").to(torch.int32)
    y[5::7] = -1
    x[10] = 0.0                                              # all equal
    x[11, 3:] = float("-inf")                                # fewer than most k left
    x[12] = float(torch.finfo(dtype).min)                    # masked by a number
    x[12, V // 2:V // 2 + 9] = 1.5
    x[13] = torch.linspace(-3, 9, V, device="cuda").to(dtype)     # rising
    x[14, ::2] = 5.0                                         # many of the largest
    y[10:15] = 4
    y[11] = 2
    r = losses.token_scores(x, y, k)
    part, xs, ys = some_rows(torch, r, x, y, list(range(0, 40)) + [2600, T - 2, T - 1])
    check_scores(torch, part, xs, ys, k, 1.0)
    for t in range(0, T, 1300):
        few = losses.token_scores(x[t:t + 1300], y[t:t + 1300], k)
        assert torch.equal(few["top"], r["top"][t:t + 1300])
        # both within the bound of logp and entropy, here 1e-4 of a few units at most
        for name in ("logp", "entropy", "top_logp"):
            a, b = few[name], r[name][t:t + 1300]
            assert ((a - b).abs() <= 1e-4 * (1 + b.abs()) * (1 + V ** 0.5 * 1e-2))[torch.isfinite(b)].all() and \
                torch.equal(torch.isfinite(a), torch.isfinite(b))
    if k in (0, 20):
        a, b = (torch.randn(T, generator=g, device="cuda") for _ in range(2))
        d = losses.token_scores_grad(x, y, r["stats"], r["entropy"], a, b)
        rows = list(range(0, 25)) + [T - 2, T - 1]
        at = torch.tensor(rows, device="cuda")
        check_gradient(torch, d[at], x[at], y[at], on_host(a[at]), on_host(b[at]), 1.0)
        assert (d[y < 0] == 0).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [3, 17, 64, 100, 129, 200, 256, 301, 511, 512])
@pytest.mark.parametrize("k", [1, 9, 64])
def test_short_rows(cuda, losses, dtype, V, k):
    """Several rows to a warp: the last warp is not full; special rows among them."""
    torch = cuda
    dtype = getattr(torch, dtype)
    _, x, y = make(torch, dtype, 203, V, masked=range(2, 203, 5))
    x[0] = 1.0
    x[1, V // 2:] = float("-inf")
    y[1] = 0
    x[3] = float(torch.finfo(dtype).min)
    x[3, V - 1] = 2.0
    y[3] = V - 1
    x[4, ::2] = 0.0
    x[4, 1::2] = -0.0
    y[4] = V - 1
    r = losses.token_scores(x, y, k, 0.9)
    check_scores(torch, r, x, y, k, 0.9)
    a, b, da, db = derivatives(torch, 203)
    check_gradient(torch, losses.token_scores_grad(x, y, r["stats"], r["entropy"], da, db, 0.9), x, y, a, b, 0.9)
    x[5, V // 2] = float("nan")
    x[6, V // 2] = float("inf")
    y[5:7] = 0
    r = losses.token_scores(x, y, k)
    assert torch.isnan(r["logp"][5:7]).all() and torch.isnan(r["entropy"][5:7]).all()
    assert r["top"][6, 0] == V // 2 and V // 2 not in r["top"][5].tolist()
    assert torch.isfinite(r["logp"][7:]).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [258, 300, 520, 700, 1024, 1025, 2040])
@pytest.mark.parametrize("k", [12, 13, 16, 17, 21, 48, 64])
def test_bounds_of_a_warps_row(cuda, losses, dtype, V, k):
    """Rows that a warp takes, where the parts that its lanes know the largest of are few, equal, empty or uneven."""
    torch = cuda
    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(V * 100 + k)
    x = torch.randn(14, V, generator=g, device="cuda") * 3
    x[0] -= 100
    for row, left in ((1, k - 1), (2, k), (3, k + 1)):
        some = torch.randperm(V, generator=g, device="cuda")[left:]
        x[row, some] = float("-inf")
    x[4] = -2.5
    x[5] = torch.arange(V, device="cuda") / 8
    x[6] = -torch.arange(V, device="cuda") / 8
    x[7] = torch.randn(V, generator=g, device="cuda") * 1e-38
    x[8, :64] += 50                               # the largest side by side
    x[9, ::32] += 50
    x[10, ::256] += 50
    x[11] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.5, float(torch.finfo(dtype).min), -1e30)
    x[11, torch.randperm(V, generator=g, device="cuda")[:k // 2]] = 1.0
    x[12] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.5, 0.0, -0.0)
    x[13, :V // 2] = float("-inf")
    x = x.to(dtype)
    check_scores(torch, losses.token_scores(x, None, k), x, None, k, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V,shift", [(12, 600, 1), (12, 1000, 3), (12, 2000, 0), (12, 2031, 5), (12, 9001, 1), (170, 9001, 3), (12, 40001, 7), (320, 40001, 2),
                                       (5000, 6001, 1)])
@pytest.mark.parametrize("k", [1, 5, 20, 64])
def test_many_equal_ones_reach_the_bound(cuda, losses, dtype, T, V, shift, k):
    """Fewer than k above the equal ones: they are the lowest classes among these, wherever they lie."""
    torch = cuda
    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(V + k)
    store = torch.empty(T * V + shift, dtype=dtype, device="cuda")
    x = store[shift:].view(T, V)
    lowest = float(torch.finfo(dtype).min)
    values = torch.randn(12, V, generator=g, device="cuda").to(dtype)
    perm = torch.randperm(V, generator=g, device="cuda")
    for row, (left, mask) in enumerate([(k - 1, lowest), (k // 2, -1e9), (0, 0.0), (max(k - 2, 0), -3.0), (k, lowest), (k + 1, -1e30)]):
        values[row, perm[left:]] = mask
    values[6] = 0.0
    values[6, V // 2:] = 1.0                      # nothing above, in the upper half
    values[7] = -1.0
    values[7, V // 3::2] = 4.0
    values[7, perm[:k // 3]] = 5.0
    values[8] = 2.0
    values[8, :V - V // 4] = -values[8, :V - V // 4]
    values[9] = (perm % 3).to(dtype)
    values[10] = lowest
    values[10, V - k // 2:] = 1.0                  # at the very end
    values[11, perm[k // 2:]] = float("-inf")
    x.copy_(values.repeat(-(-T // 12), 1)[:T])
    some = torch.cat([torch.arange(12), torch.arange(T - 12, T)]).unique().cuda()
    r = losses.token_scores(x, None, k)
    if k < 2:                                     # the last row has no class left
        none = some[some % 12 == 11]
        assert r["entropy"][none].isnan().all() and (r["top"][none] == -1).all()
        some = some[some % 12 != 11]
    got = {name: v[some] for name, v in r.items() if v is not None}
    got["logp"] = None
    check_scores(torch, got, x[some], None, k, 1.0)
    reps = r["top"][:T // 12 * 12].view(-1, 12, k)
    assert (reps == reps[:1]).all()
