"""Losses on rows of logits where rows are split, many to a CTA, masked or far
from zero, against the 64-bit oracle (bounds: test_gpu_row_losses.py)."""

import numpy as np
import pytest

from oracle import row_losses_oracle as O
from test_gpu_row_losses import (U, check_gradient, check_policy, check_preference, losses, make, offsets_of,  # noqa: F401
                                 on_host, rows_and_bounds)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V", [(1, 4104), (5, 9001), (1, 32768), (30, 32771), (60, 20000), (100, 9000), (130, 65537),
                                 (2, 50001), (9, 100003), (3, 262147)])
def test_rows_split_over_clusters(cuda, losses, dtype, T, V):
    """Rows shared by the CTAs of a cluster, which exchange their parts: many
    launches behind one another, beside a stream that keeps SMs busy."""
    torch = cuda
    r, x, y = make(torch, getattr(torch, dtype), T, V, seed=17, masked=range(1, T, 7))
    noise = torch.zeros(1 << 22, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    logp, stats = losses.token_logprob(x, y)
    want, m, L, p, elogp, ep = rows_and_bounds(x, y, 1.0)
    assert (np.abs(on_host(logp) - want) <= elogp).all()
    old = logp - 0.1
    adv = torch.from_numpy(r.standard_normal(T).astype(np.float32)).cuda()
    pol = losses.policy_loss(x, y, old, adv)
    check_policy(torch, pol, x, y, old, adv, None, {})
    same = torch.ones((), dtype=torch.bool, device="cuda")
    for _ in range(30):
        with torch.cuda.stream(side):
            noise.add_(1.0)
        again = losses.token_logprob(x, y)
        twice = losses.policy_loss(x, y, old, adv)
        same &= (again[0] == logp).all() & (again[1] == stats).all() & (twice["dlogits"] == pol["dlogits"]).all()
        same &= (twice["logp"] == pol["logp"]).all() & (twice["loss"] == pol["loss"])
    assert bool(same)


def test_longest_row(cuda, losses):
    """A row of 2^31 - 1 classes, all masked by the lowest value, so that every
    pass goes element by element (bf16: 4.3 GB, written in place)."""
    torch = cuda
    V = (1 << 31) - 1
    low = float(torch.finfo(torch.bfloat16).min)
    x = torch.full((1, V), low, dtype=torch.bfloat16, device="cuda")
    y = torch.tensor([V - 1], dtype=torch.int32, device="cuda")
    logp, stats = losses.token_logprob(x, y)
    # equal terms: sums of ones below 2^24 per thread are exact, their total is rounded, log within 2 u
    assert float(logp) == pytest.approx(-np.log(V), rel=4 * U)
    one = torch.ones(1, device="cuda")
    p = torch.tensor(-1.0 / V).bfloat16()           # 2^-31 (1 + 2^-31): one bf16 value, its neighbours 2^-8 away
    d = losses.token_logprob_grad(x, y, stats, one, out=x)
    assert (d[0, :V - 1] == p.cuda()).all() and float(d[0, V - 1]) == 1.0
    x.fill_(low)
    pol = losses.policy_loss(x, y, logp, -one, out=x)
    assert torch.equal(pol["logp"], logp) and float(pol["loss"]) == 1.0
    assert (x[0, :V - 1] == p.cuda()).all() and float(x[0, V - 1]) == 1.0


MASKS = [-1e4, -1e9, -5e9, -1e10, -1e20, -1e30, -1e37, "lowest"]


def masked_rows(torch, dtype, V, seed):
    """A row for every mask value and place of the masked classes: a prefix, a suffix, all but ten, the last one
    alone, every second (by -inf and the value in turn), and all of them."""
    places = 6
    r, x, y = make(torch, dtype, places * len(MASKS), V, seed=seed)
    for i, value in enumerate(MASKS):
        value = float(torch.finfo(dtype).min) if value == "lowest" else value
        rows = range(places * i, places * (i + 1))
        x[rows[0], :V // 2] = value
        x[rows[1], V // 5:] = value
        keep = x[rows[2], V // 3:V // 3 + 10].clone()
        x[rows[2]] = value
        x[rows[2], V // 3:V // 3 + 10] = keep
        x[rows[3], V - 1] = value
        x[rows[4], 1::2] = value
        x[rows[4], 1::4] = -float("inf")
        x[rows[5]] = value
        for row, at in zip(rows, (V - 1, 0, V // 3 + 4, V // 7, V // 4 * 2, 3)):
            y[row] = at
    return r, x, y


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [100, 500, 600, 1000, 1001, 9001, 20003, 50001, 70001, 131073])
def test_masks_of_any_value(cuda, losses, dtype, V):
    """Classes masked by large negative numbers count for nothing, whatever the number, the temperature and the
    order in which a thread meets them.  (Elements of probability 0 are exact, so the bounds are those of the rest.)"""
    torch = cuda
    r, x, y = masked_rows(torch, getattr(torch, dtype), V, 29)
    T = len(y)
    copies = 4                                      # enough rows that none is split over a cluster, and a few to a CTA
    many, ymany = x.repeat(copies, 1), y.repeat(copies)
    off, off_d = offsets_of(torch, [T // 2, T - T // 2])
    one = torch.ones(T, device="cuda")
    for tau in (0.6, 0.7, 1.0, 1.3, 10.0):
        logp, stats = losses.token_logprob(x, y, tau)
        want, m, L, p, elogp, ep = rows_and_bounds(x, y, tau)
        assert (np.abs(on_host(logp) - want) <= elogp).all(), tau
        assert (np.abs(on_host(stats)[:, 1] - L) <= elogp).all()
        d = losses.token_logprob_grad(x, y, stats, one, tau)
        check_gradient(torch, d, x, y, np.ones(T), tau, p, ep, 0.0)
        again, _ = losses.token_logprob(many, ymany, tau)
        assert (np.abs(on_host(again).reshape(copies, T) - want) <= elogp).all()
        old = torch.from_numpy((want - 0.1).astype(np.float32)).cuda()
        pol = losses.policy_loss(x, y, old, one, temperature=tau)
        check_policy(torch, pol, x, y, old, one, None, dict(temperature=tau))
        all_of_them = losses.policy_loss(many, ymany, old.repeat(copies), one.repeat(copies), temperature=tau, scale=copies)
        parts = all_of_them["dlogits"].view(copies, T, V)
        assert (parts[1:] == parts[0]).all()
        few = dict(pol, logp=all_of_them["logp"][:T], dlogits=parts[0])
        check_policy(torch, few, x, y, old, one, None, dict(temperature=tau))
        kw = dict(beta=0.01, average=True, temperature=tau)
        check_preference(torch, losses.preference_loss(x, y, off_d, **kw), x, y, off, None, kw)


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("average", [False, True])
def test_preference_of_well_separated_pairs(cuda, losses, smoothing, average):
    """The slope of the sigmoid loss keeps its digits where it is small: relative to e sig(h) + (1 - e) sig(-h), the
    sum of its two terms, exp is good to 4 u, and one sum, one quotient and the products with e, beta, scale, 1 /
    pairs and 1 / rows add 7 u at most; h moves it by sig'(h) beta times the error of the gap, which is that of
    the scores, its own rounding and, through h = beta gap, two more."""
    torch = cuda
    wanted = [-40.0, -20.0, -10.0, -5.0, -1.0, 0.3, 2.2, 5.0, 10.0, 12.0, 15.0, 17.0, 20.0, 40.0]
    beta, pairs, rows = float(np.float32(0.1)), len(wanted), 3
    T, V = 2 * pairs * rows, 1000
    r, x, y = make(torch, torch.float32, T, V, seed=41)
    off, off_d = offsets_of(torch, [rows] * (2 * pairs))
    _, _, _, p, elogp, ep = rows_and_bounds(x, y, 1.0)
    kw = dict(beta=beta, smoothing=float(np.float32(smoothing)), average=average)
    scores = O.preference(on_host(x), y.cpu().numpy(), off, **kw)[1]
    ref = np.zeros((pairs, 2))
    ref[:, 1] = scores[:, 1] + 0.25
    ref[:, 0] = scores[:, 0] - np.array(wanted) / beta + 0.25
    ref = torch.from_numpy(ref.astype(np.float32)).cuda()
    loss, scores, coef = O.preference(on_host(x), y.cpu().numpy(), off, ref.cpu().numpy(), **kw)
    gap = (scores[:, 0] - scores[:, 1]) - (on_host(ref)[:, 0] - on_host(ref)[:, 1])
    h = beta * gap
    assert np.abs(h - wanted).max() < 1e-4
    share = 1.0 / rows if average else 1.0
    egap = (elogp.reshape(pairs, -1).sum(1) + 2 * U * np.abs(scores).sum(1)) * share + 3 * U * np.abs(gap)
    near, far = 1 / (1 + np.exp(-h)), 1 / (1 + np.exp(h))
    e = kw["smoothing"]
    ecoef = beta * share / pairs * (1.01 * beta * near * far * egap + 11 * U * (e * near + (1 - e) * far))
    res = losses.preference_loss(x, y, off_d, ref, **kw)
    check_gradient(torch, res["dlogits"], x, y, coef, 1.0, p, ep, np.repeat(ecoef, 2 * rows))
    value = (1 - e) * np.logaddexp(0, -h) + e * np.logaddexp(0, h)
    eloss = np.mean(np.abs(e * near - (1 - e) * far) * beta * egap + 12 * U * value)
    assert abs(float(res["loss"]) - loss) <= eloss


@pytest.mark.parametrize("V", [8, 1000, 20003, 70001])
def test_policy_near_its_reference(cuda, losses, V):
    """KL and its slope keep their digits where policy and reference nearly agree.  Both are functions of u = ref -
    logp, so they are taken at the log probabilities that the call returned: u is one rounding off (none, where
    small), which moves exp(u) - u - 1 by at most (2 + |u|) u of itself and exp(u) - 1 by (1 + |u|) u; exp(u) - 1
    is good to 2 u; its distance to u to 9 u at |u| = 1/2 and better beyond, the series below to 6 u; weights,
    coefficients and sums add 4 roundings."""
    torch = cuda
    T = 6
    r, x, y = make(torch, torch.float32, T, V, seed=43, spread=1.0)
    _, _, _, p, _, ep = rows_and_bounds(x, y, 1.0)
    logp, _ = losses.token_logprob(x, y)
    nothing = torch.zeros(T, device="cuda")
    for size in (1e-5, 1e-4, 3e-4, 1e-3, 1e-2, 0.1, 0.3, 0.49, 0.51, 1.0, 3.0, 20.0):
        for sign in (1, -1):
            ref = logp + torch.from_numpy((sign * size * r.uniform(0.9, 1.0, T)).astype(np.float32)).cuda()
            res = losses.policy_loss(x, y, logp, nothing, ref, kl=1.0)
            u = on_host(ref) - on_host(res["logp"])
            assert (np.sign(u) == sign).all()
            kl = np.where(np.abs(u) < 1e-2, u * u * (1 / 2 + u / 6 * (1 + u / 4 * (1 + u / 5 * (1 + u / 6)))), np.expm1(u) - u)
            tol = U * ((15 + np.abs(u)) * kl).mean()
            assert abs(float(res["terms"][1]) - kl.mean()) <= tol, (size, sign)
            assert abs(float(res["loss"]) - kl.mean()) <= tol + 2 * U * kl.mean()
            coef = -np.expm1(u) / T
            check_gradient(torch, res["dlogits"], x, y, coef, 1.0, p, ep, U * (7 + np.abs(u)) * np.abs(coef))


@pytest.mark.parametrize("kind", ["sigmoid", "hinge"])
@pytest.mark.parametrize("beta", [1e-3, 1e-30, 1e-38])
def test_preference_of_small_beta_and_margin(cuda, losses, kind, beta):
    """h = beta gap - margin where margin / beta passes the range of a float: h is -margin to a rounding, and
    everything is the function of it (4 u of exp, 4 more roundings)."""
    torch = cuda
    _, x, y = make(torch, torch.float32, 8, 50, seed=3)
    off = torch.arange(9, dtype=torch.int32, device="cuda")
    margin = 30.0
    res = losses.preference_loss(x, y, off, kind=kind, beta=beta, margin=margin, smoothing=0.25)
    loss = O.preference(on_host(x), y.cpu().numpy(), np.arange(9), beta=float(np.float32(beta)), kind=kind, margin=margin,
                        smoothing=0.25)[0]
    # beta gap (below 0.03) has the scores' error, 100 u at most here, times beta
    assert float(res["loss"]) == pytest.approx(loss, rel=16 * U)
    assert res["dlogits"].isfinite().all()


def gradient_and_bound(torch, dtype, x, y, coef, p, ep, ecoef):
    """coef ([v = y] - p) in double and check_gradient's bound, on the GPU (temperature 1, every row with a target)."""
    ys = y.cpu().numpy()
    want = O.logits_gradient(on_host(x), ys, coef)
    one = np.zeros_like(p)
    one[np.arange(len(ys)), ys] = 1.0
    h = torch.finfo(dtype).eps / 2
    k, ek = np.abs(coef)[:, None], ecoef[:, None]
    tol = ((k + ek) * (p * ep + 4 * U * (one + p)) + ek * np.abs(one - p) + h * np.abs(want)) * (1 + h) + 1e-37
    return torch.from_numpy(want).cuda(), torch.from_numpy(tol).cuda()


MANY = [("bfloat16", 1001, 9000), ("bfloat16", 6144, 8000), ("bfloat16", 6152, 6000), ("bfloat16", 16385, 3000),
        ("bfloat16", 18432, 2500), ("bfloat16", 18441, 2500), ("bfloat16", 32769, 1500), ("bfloat16", 56320, 1000),
        ("bfloat16", 56329, 700), ("bfloat16", 65537, 700), ("bfloat16", 75776, 500), ("bfloat16", 75785, 500),
        ("bfloat16", 100003, 500), ("bfloat16", 106496, 400), ("bfloat16", 106505, 400), ("bfloat16", 131073, 400),
        ("float32", 1001, 9000), ("float32", 9001, 3000), ("float32", 20003, 1200), ("float32", 36001, 600),
        ("float32", 50001, 400), ("float32", 53248, 400), ("float32", 53253, 400)]


@pytest.mark.parametrize("dtype,V,T", MANY)
def test_policy_of_many_rows(cuda, losses, dtype, V, T):
    """Several rows to a CTA, one behind the other: 37 kinds of rows in turn, at every place in a 16-byte piece, so
    that no row stands where one of its kind stood before; some without a target (alone, and more in a run than
    there are CTAs), some clipped, some worked out element by element.  Every row against the oracle's row of its
    kind; the same bits whatever the output's place."""
    torch = cuda
    kinds = 37
    dtype = getattr(torch, dtype)
    pad = V % 3
    r, x, y = make(torch, dtype, kinds, V, seed=51, pad=pad, shift=1)
    x[5] = float(torch.finfo(dtype).min)
    x[9, V // 2:] = -1e10
    x[11] += 3e4
    x[12] = -1e30
    y[9] = V // 3
    logp, _, _, p, elogp, ep = rows_and_bounds(x, y, 1.0)
    old = (logp - np.where(r.random(kinds) < 0.3, 0.5, 0.1)).astype(np.float32)
    ref = (logp + 0.3 * r.standard_normal(kinds)).astype(np.float32)
    adv = r.standard_normal(kinds).astype(np.float32)
    kl = float(np.float32(0.1))
    one = [O.policy(on_host(x[j:j + 1]), y[j:j + 1].cpu().numpy(), old[j:j + 1], adv[j:j + 1], ref[j:j + 1],
                    reduction="sum", kl=kl) for j in range(kinds)]
    terms, coef = np.array([o[1] for o in one]), np.array([o[3][0] for o in one])
    # the ratio: logp's error and the difference's rounding in the exponent, 4 u of expf and the product; KL: by its derivative
    A, ratio, u = np.abs(adv), np.exp(logp - old), ref - logp
    er, eu = elogp + U * (np.abs(logp - old) + 6), elogp + U * np.abs(u)
    ekl = np.abs(np.expm1(u)) * eu + eu ** 2 + 16 * U * terms[:, 1]
    ecoef = A * ratio * er + kl * np.exp(u) * eu + 8 * U * (A * ratio + kl * np.abs(np.expm1(u)))
    want, tol = gradient_and_bound(torch, dtype, x, y, coef, p, ep, ecoef)

    kind = torch.arange(T, device="cuda") % kinds
    store = torch.zeros(3 + T * (V + pad) + 8, dtype=dtype, device="cuda")
    many = store.as_strided((T, V), (V + pad, 1), 3)
    for t in range(0, T, kinds):
        many[t:t + kinds] = x[:min(kinds, T - t)]
    target = y[kind].contiguous()
    off = np.zeros(T, bool)
    off[r.integers(kinds, T, T // 9)] = True
    off[T // 2:T // 2 + min(600, T // 3)] = True
    off = torch.from_numpy(off).cuda()
    target[off] = -1
    args = [target] + [torch.from_numpy(v).cuda()[kind].contiguous() for v in (old, adv, ref)]
    kw = dict(reduction="sum", kl=0.1)
    res = losses.policy_loss(many, *args, **kw)
    assert (res["dlogits"][off] == 0).all() and (res["logp"][off] == 0).all()
    on = torch.nonzero(~off)[:, 0]
    for rows in on.split(256):
        k = kind[rows]
        assert ((res["logp"][rows].double() - torch.from_numpy(logp).cuda()[k]).abs() <= torch.from_numpy(elogp).cuda()[k]).all()
        assert ((res["dlogits"][rows].double() - want[k]).abs() <= tol[k]).all()
    # the sums: every kind's terms as often as it occurs
    times = np.bincount(kind[on].cpu().numpy(), minlength=kinds)
    total, got = times @ terms, on_host(res["terms"])
    assert abs(got[0] - total[0]) <= times @ (A * (ratio * er + 4 * U * (ratio + 1)))
    assert abs(got[1] - total[1]) <= times @ ekl
    assert got[2] == total[2] and total[2] > 0
    # other places for the gradient
    outs = torch.full((2 + T * (V + 1) + 40,), 7.0, dtype=dtype, device="cuda")
    out = outs.as_strided((T, V), (V + 1, 1), 2)
    again = losses.policy_loss(many, *args, out=out, **kw)
    assert torch.equal(out, res["dlogits"]) and all(torch.equal(again[k], res[k]) for k in ("loss", "terms", "logp"))
    out.fill_(7.0)
    assert (outs == 7.0).all()
    alone = losses.policy_loss(many, *args, grad=False, **kw)
    assert all(torch.equal(alone[k], res[k]) for k in ("loss", "terms", "logp"))
    losses.policy_loss(many, *args, out=many, **kw)
    assert torch.equal(many, res["dlogits"])


def test_outputs_keep_nothing_else(cuda, losses):
    """A loss or a score that is kept, or saved, holds its own bytes and neither the workspace's nor another's."""
    torch = cuda
    _, x, y = make(torch, torch.float32, 40, 600)
    f = torch.zeros(40, device="cuda")
    off = torch.arange(0, 41, 10, dtype=torch.int32, device="cuda")
    logp, stats = losses.token_logprob(x, y)
    outs = [logp, stats, losses.token_logprob_grad(x, y, stats, f)]
    for res in (losses.preference_loss(x, y, off), losses.balance_loss(x[:, :16], 2),
                losses.policy_loss(x, y, f, f, f, kl=0.1, offsets=off, reduction="sequences")):
        outs += res.values()
    assert all(t.is_contiguous() and t.untyped_storage().nbytes() == t.numel() * t.element_size() for t in outs)
    assert len({t.untyped_storage().data_ptr() for t in outs}) == len(outs)


@pytest.mark.parametrize("V", [50, 9001, 40000])
def test_targets_that_are_none_where_nothing_is_asked(cuda, losses, V):
    """A target that is no class makes the gradients NaN that depend on it; a row outside every sequence, or of
    derivative 0, takes no part whatever its target."""
    torch = cuda
    _, x, y = make(torch, torch.float32, 8, V, seed=6)
    y[0] = y[5] = y[7] = V
    off = torch.tensor([1, 3, 5], dtype=torch.int32, device="cuda")
    res = losses.preference_loss(x, y, off)
    assert res["loss"].isfinite() and res["dlogits"].isfinite().all() and (res["dlogits"][[0, 5, 6, 7]] == 0).all()
    f = torch.zeros(8, device="cuda")
    pol = losses.policy_loss(x, y, f - 5, f + 1, offsets=off, reduction="sequences")
    assert pol["loss"].isfinite() and (pol["dlogits"][[0, 5, 6, 7]] == 0).all()
    _, stats = losses.token_logprob(x, y)
    one = f + 1
    one[[0, 3]] = 0
    d = losses.token_logprob_grad(x, y, stats, one)
    assert (d[[0, 3]] == 0).all() and d[[5, 7]].isnan().all() and d[[1, 2, 4, 6]].isfinite().all()
