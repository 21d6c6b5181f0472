"""The losses on rows of logits against the 64-bit oracle.

Tolerances, u = 2^-24 (fp32 rounding), h = half a step of the gradient's type
(2^-24 fp32, 2^-8 bf16), z = x / tau, D = distance of a row's z from its maximum:
  exp((x - m) / tau): the argument is rounded at most four times (subtraction,
    1 / tau, log2 e, product) and ex2 is good to 2 u, so its relative error is
    at most (4 D + 4) u; a sum of positive terms inherits the mean of that under
    p plus its chain of additions (128 + V / 256 at most here);
  logp = (x_y - m) / tau - L: 3 u D_y + the error of L (that of the sum, 2 u |L|) + u |logp|;
  gradient k ([v = y] - p) / tau: p's relative error as above with L's, 8 u for
    the products, k's own relative error, then h.
A score adds its rows' errors; a loss those of its scores through its derivative."""

import numpy as np
import pytest

from oracle import row_losses_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LOWEST = float(np.finfo(np.float32).min)


@pytest.fixture(scope="module")
def losses(cuda):
    from paper_2607_20739_gb300 import losses
    return losses


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def make(torch, dtype, T, V, seed=0, pad=0, shift=0, spread=2.0, masked=()):
    """Logits [T, V] of row pitch V + pad whose first element lies `shift` elements into its storage."""
    r = np.random.default_rng([seed, T, V])
    store = torch.full((shift + T * (V + pad) + 3,), float("nan"), dtype=dtype, device="cuda")
    x = store.as_strided((T, V), (V + pad, 1), shift)
    x.copy_(torch.from_numpy((r.standard_normal((T, V)) * spread).astype(np.float32)))
    y = r.integers(0, V, T).astype(np.int32)
    y[list(masked)] = -1
    return r, x, torch.from_numpy(y).cuda()


def on_host(x):
    return x.double().cpu().numpy()


def rows_and_bounds(x, y, tau):
    """Oracle rows, and the error allowed to each logp and to the relative error of each p."""
    xs, ys = on_host(x), y.cpu().numpy()
    logp, m, L, p = O.rows(xs, ys, tau)
    with np.errstate(all="ignore"):
        D = np.where(np.isfinite(xs), (m[:, None] - xs) / tau, 0.0)
    V = xs.shape[1]
    eL = U * ((4 * D * p).sum(1) + 4 + min(V, 128 + V / 256) + 2 * np.abs(L))
    Dy = D[np.arange(len(ys)), np.clip(ys, 0, V - 1)]
    elogp = eL + U * (3 * np.abs(Dy) + np.abs(np.nan_to_num(logp, neginf=0.0)) + 1)
    ep = U * (4 * D + 12 + np.abs(L)[:, None]) + eL[:, None]
    return logp, m, L, p, elogp, ep


def check_gradient(torch, got, x, y, coef, tau, p, ep, ecoef, headroom=None):
    """got against coef ([v = y] - p) / tau; ecoef: absolute error allowed to coef."""
    ys = y.cpu().numpy()
    want = O.logits_gradient(on_host(x), ys, coef, tau)
    one = np.zeros_like(p)
    valid = (ys >= 0) & (ys < p.shape[1])
    one[valid, ys[valid]] = 1.0
    h = half_step(torch, got.dtype)
    k, ek = np.abs(coef)[:, None] / tau, np.broadcast_to(ecoef, coef.shape)[:, None] / tau
    tol = (k + ek) * (p * ep + 4 * U * (one + p)) + ek * np.abs(one - p) + h * np.abs(want)
    tol = tol * (1 + h) + 1e-37
    g = on_host(got)
    assert np.isfinite(want).all()
    assert (g[ys < 0] == 0).all()
    err = np.abs(g - want)
    assert (err <= tol).all(), (np.argwhere(err > tol)[:5], (err / tol).max())


SIZES = [(1, 1), (3, 2), (5, 7), (4, 8), (9, 33), (70, 100), (300, 10), (31, 16), (66, 17), (37, 64), (5, 65), (35, 128), (18, 129),
         (17, 255), (17, 256), (9, 257), (9, 258), (11, 511), (11, 512), (6, 513), (6, 514), (33, 1000), (6, 4095), (5, 4096), (4, 4097), (3, 8191),
         (3, 12345), (5, 32768), (3, 50001), (2, 131072), (1, 262147)]


@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_token_logprob(cuda, losses, T, V, dtype, tau):
    torch = cuda
    dtype = getattr(torch, dtype)
    _, x, y = make(torch, dtype, T, V, masked=range(2, T, 5))
    logp, stats = losses.token_logprob(x, y, tau)
    want, m, L, p, elogp, ep = rows_and_bounds(x, y, tau)
    assert (np.abs(on_host(logp) - want) <= elogp).all()
    st = on_host(stats)
    assert (st[:, 0] == m).all()
    assert (np.abs(st[:, 1] - L) <= elogp).all()
    coef = np.random.default_rng(1).standard_normal(T).astype(np.float32)
    coef[T // 2] = 0
    d = losses.token_logprob_grad(x, y, stats, torch.from_numpy(coef).cuda(), tau)
    assert d.dtype == dtype and d.is_contiguous()
    check_gradient(torch, d, x, y, coef.astype(np.float64), tau, p, ep, 0.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V,pad,shift,out_pad,out_shift", [
    (7, 1000, 0, 1, 0, 1), (7, 1000, 8, 0, 0, 0), (7, 1001, 0, 3, 0, 3), (7, 1001, 5, 2, 2, 1), (5, 33, 1, 5, 3, 0),
    (9, 100, 0, 1, 0, 1), (9, 100, 1, 0, 0, 0), (9, 100, 2, 2, 0, 1), (9, 300, 2, 0, 4, 2), (9, 300, 0, 1, 0, 0), (9, 60, 0, 0, 1, 0),
    (5, 20003, 0, 1, 0, 1), (5, 20003, 6, 3, 1, 2), (4, 70001, 0, 7, 0, 7), (4, 70001, 0, 7, 0, 0), (3, 5, 0, 1, 0, 2)])
def test_pitches_and_alignments(cuda, losses, dtype, T, V, pad, shift, out_pad, out_shift):
    torch = cuda
    dtype = getattr(torch, dtype)
    r, x, y = make(torch, dtype, T, V, pad=pad, shift=shift, masked=[1])
    _, out, _ = make(torch, dtype, T, V, pad=out_pad, shift=out_shift)
    outs = torch.full((out_shift + T * (V + out_pad) + 40,), 7.0, dtype=dtype, device="cuda")
    out = outs.as_strided((T, V), (V + out_pad, 1), out_shift)
    logp, stats = losses.token_logprob(x, y)
    want, m, L, p, elogp, ep = rows_and_bounds(x, y, 1.0)
    assert (np.abs(on_host(logp) - want) <= elogp).all()
    coef = r.standard_normal(T).astype(np.float32)
    assert losses.token_logprob_grad(x, y, stats, torch.from_numpy(coef).cuda(), out=out) is out
    check_gradient(torch, out, x, y, coef.astype(np.float64), 1.0, p, ep, 0.0)
    # policy form into the same place, and nothing beside the rows is touched
    old = logp - 0.1
    adv = torch.from_numpy(coef).cuda()
    before = x.clone()
    res = losses.policy_loss(x, y, old, adv, out=out, reduction="sum")
    check_policy(torch, res, x, y, old, adv, None, dict(reduction="sum"))
    assert torch.equal(before, x)
    gaps = outs.clone()
    gaps.as_strided((T, V), (V + out_pad, 1), out_shift).fill_(7.0)
    assert (gaps == 7.0).all()
    # in place
    inside = losses.policy_loss(x, y, old, adv, out=x, reduction="sum")
    assert inside["dlogits"] is x and torch.equal(x, out) and inside["loss"] == res["loss"]


def test_masked_logits_and_values(cuda, losses):
    torch = cuda
    for V in (64, 120, 400, 600, 6000, 40000):
        _, x, y = make(torch, torch.float32, 8, V, seed=2)
        y[:] = torch.arange(8, dtype=torch.int32) * (V // 9)
        x[0, 1:] = -float("inf")                    # one class left, the target
        x[1, :V // 2] = LOWEST                      # masked by the lowest value
        x[2, :] = LOWEST                            # all of them
        x[3, int(y[3])] = -float("inf")             # the target itself masked
        y[4] = -1
        x[4, :] = float("nan")                      # NaN where nothing is read
        x[5, :] = -float("inf")                     # no class left
        x[6, 3] = float("nan")
        x[7, :] += 3e4                              # far from zero
        logp, stats = losses.token_logprob(x, y)
        lp = logp.cpu().numpy()
        # one class: the sum is 2^r with r the residue of the rounded exponent of the maximum, |r| <= u |m c| here
        # below 2^-19; ex2 gives it within 2 u and its logarithm takes r ln 2 back with at most u more: 3 u
        assert abs(lp[0]) <= 3 * U
        assert lp[2] == pytest.approx(-np.log(V), rel=4 * U) and lp[3] == -np.inf and lp[4] == 0
        assert np.isnan(lp[5]) and np.isnan(lp[6])
        sel = [0, 1, 2, 7]
        want, _, _, p, elogp, ep = rows_and_bounds(x[sel], y[sel], 1.0)
        assert (np.abs(lp[sel] - want) <= elogp).all()
        one = torch.ones(8, device="cuda")
        d = losses.token_logprob_grad(x, y, stats, one)
        check_gradient(torch, d[sel], x[sel], y[sel], np.ones(4), 1.0, p, ep, 0.0)
        assert (d[4] == 0).all() and d[5].isnan().any() and d[6].isnan().any()
        # the same rows through the fused forms: every value of a row with a distribution is that of the split form
        one[5:7] = 0
        y2 = y.clone()
        y2[5:7] = -1
        pol = losses.policy_loss(x, y2, logp.nan_to_num(neginf=0.0), -one, reduction="sum")
        ratio = torch.ones(8, device="cuda")
        ratio[3] = 0
        ref = losses.token_logprob_grad(x, y2, stats, ratio)
        torch.testing.assert_close(pol["dlogits"], ref, rtol=64 * U, atol=1e-30)
        assert pol["logp"][3] == -float("inf")
        # advantage -1: max(r, q) a row, r = 1 in four rows, r = 0 and q = 0.8 in the masked target's
        assert float(pol["loss"]) == pytest.approx(4.8, rel=16 * U)


@pytest.mark.parametrize("tau", [1e-38, 1e-30, 1e30])
def test_far_temperatures(cuda, losses, tau):
    """So cold that one class is left, so hot that all are alike."""
    torch = cuda
    for V in (40, 7000):
        _, x, y = make(torch, torch.float32, 3, V, seed=4)
        top = x.argmax(1).to(torch.int32)
        y[0] = top[0]
        logp, stats = losses.token_logprob(x, y, tau)
        one = torch.ones(3, device="cuda")
        d = losses.token_logprob_grad(x, y, stats, one, tau)
        pol = losses.policy_loss(x, y, logp.nan_to_num(neginf=0.0), -one, reduction="sum", temperature=tau)
        assert torch.equal(pol["logp"], logp)
        if tau > 1:
            assert torch.allclose(logp, torch.full_like(logp, -float(np.log(V))), rtol=4 * U)
        else:
            assert logp[0] == 0 and (logp[1:] < -1e20).all()
            assert (d[0] == 0).all()


def offsets_of(torch, lens, first=0):
    off = np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)
    return off, torch.from_numpy(off).cuda()


def check_preference(torch, res, x, y, off, ref, kw):
    tau = kw.get("temperature", 1.0)
    okw = {("tau" if k == "temperature" else k): v for k, v in kw.items()}
    okw["beta"] = float(np.float32(kw.get("beta", 0.1)))
    for k in ("margin", "smoothing", "scale"):
        if k in kw:
            okw[k] = float(np.float32(kw[k]))
    ys = y.cpu().numpy()
    loss, scores, coef = O.preference(on_host(x), ys, off, None if ref is None else ref.cpu().numpy(), **okw)
    _, _, _, p, elogp, ep = rows_and_bounds(x, y, tau)
    pairs = len(scores)
    escore = np.zeros((pairs, 2))
    for i in range(pairs):
        for j in range(2):
            t = [t for t in range(off[2 * i + j], off[2 * i + j + 1]) if ys[t] >= 0]
            escore[i, j] = sum(elogp[q] for q in t) / (max(len(t), 1) if kw.get("average") else 1)
    got = on_host(res["logp"])
    assert (np.abs(got - scores) <= escore + U * np.abs(scores)).all()
    egap = escore.sum(1)
    beta, scale = okw["beta"], abs(okw.get("scale", 1.0))
    # |f'| <= beta for sigmoid and hinge; squared: |f'| = 2 |gap + ...|, f'' = 2; sigmoid f'' <= beta^2 / 4
    top = np.abs(coef).max() if len(coef) else 0.0
    if kw.get("kind", "sigmoid") == "squared":
        slope, bend = 2 * (np.abs(scores[:, 0] - scores[:, 1]) + (0 if ref is None else np.abs(on_host(ref)).sum(1)) +
                           0.5 / beta + abs(okw.get("margin", 0.0)) / beta), 2.0
    else:
        slope, bend = beta, beta * beta / 4
    eloss = scale * np.mean(slope * egap + bend * egap ** 2) if pairs else 0.0
    assert abs(float(res["loss"]) - loss) <= eloss + 2 * U * abs(loss)
    if res["dlogits"] is None:
        return
    ecoef = np.zeros(len(ys))
    for i in range(pairs):
        for j in range(2):
            lo, hi = off[2 * i + j], off[2 * i + j + 1]
            share = max((ys[lo:hi] >= 0).sum(), 1) if kw.get("average") else 1
            ecoef[lo:hi] = scale * bend * egap[i] / pairs / share + 2 * U * np.abs(coef[lo:hi])
    assert top > 0 or not pairs
    check_gradient(torch, res["dlogits"], x, y, coef, tau, p, ep, ecoef)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V,lens,kw", [
    (1000, [3, 5, 1, 1], dict()),
    (100, [1, 0, 4, 2, 0, 0], dict(kind="hinge", smoothing=0.25, margin=0.5, temperature=1.3)),
    (33, [40, 70, 9, 30], dict(kind="squared", average=True, beta=0.5, scale=3.0)),
    (4097, [2, 3], dict(smoothing=0.1, average=True, temperature=0.6)),
    (20003, [3, 2, 1, 4], dict(margin=0.2, scale=0.5)),
    (131072, [2, 1], dict(beta=0.7)),
    (300, [1] * 600, dict(kind="sigmoid", beta=1.0)),
    (10, [1, 0, 2, 3] * 700, dict(average=True, smoothing=0.2)),
    (10, [130, 127, 128, 129], dict(scale=2.0)),
    (64, [700, 900], dict(average=True))])
@pytest.mark.parametrize("ref", [True, False])
def test_preference(cuda, losses, dtype, V, lens, kw, ref):
    torch = cuda
    first, behind = 2, 3
    T = first + sum(lens) + behind
    r, x, y = make(torch, getattr(torch, dtype), T, V, masked=range(3, T, 7))
    off, off_d = offsets_of(torch, lens, first)
    pairs = len(lens) // 2
    logp = O.rows(on_host(x), y.cpu().numpy(), kw.get("temperature", 1.0))[0]
    score = np.array([logp[a:b].sum() for a, b in zip(off[:-1], off[1:])]).reshape(pairs, 2)
    ref_d = torch.from_numpy((score + r.standard_normal((pairs, 2))).astype(np.float32)).cuda() if ref else None
    if not ref and kw.get("kind", "sigmoid") == "sigmoid":
        kw = dict(kw, beta=0.01)                    # raw scores are tens of units apart
    res = losses.preference_loss(x, y, off_d, ref_d, **kw)
    check_preference(torch, res, x, y, off, ref_d, kw)
    d = res["dlogits"]
    assert (d[:first] == 0).all() and (d[T - behind:] == 0).all()
    again = losses.preference_loss(x, y, off_d, ref_d, **kw)
    assert all(torch.equal(res[k], again[k]) for k in res)
    alone = losses.preference_loss(x, y, off_d, ref_d, grad=False, **kw)
    assert alone["dlogits"] is None and torch.equal(alone["loss"], res["loss"]) and torch.equal(alone["logp"], res["logp"])


@pytest.mark.parametrize("dtype,V,lens,kw", [
    ("bfloat16", 32768, [200, 0, 1, 300, 0, 0, 150, 249, 17, 83], dict(smoothing=0.1)),      # several pairs at once in flight
    ("float32", 9001, [700, 800], dict(kind="squared", average=True)),                        # one pair of unaligned rows
    ("bfloat16", 20001, [1, 2] * 500, dict(kind="hinge", temperature=1.2)),                   # pairs of three rows
    ("float32", 131072, [60, 70], dict(average=True))])
def test_preference_of_many_logits(cuda, losses, dtype, V, lens, kw):
    """Enough rows for several waves of CTAs."""
    torch = cuda
    first, behind = 3, 2
    T = first + sum(lens) + behind
    r, x, y = make(torch, getattr(torch, dtype), T, V, masked=range(3, T, 7))
    off, off_d = offsets_of(torch, lens, first)
    pairs = len(lens) // 2
    logp, _ = losses.token_logprob(x, y, kw.get("temperature", 1.0))
    lp = on_host(logp)
    held = [max(int((y[a:b] >= 0).sum()), 1) if kw.get("average") else 1 for a, b in zip(off[:-1], off[1:])]
    score = np.array([lp[a:b].sum() / n for a, b, n in zip(off[:-1], off[1:], held)]).reshape(pairs, 2)
    ref_d = torch.from_numpy((score + r.standard_normal((pairs, 2))).astype(np.float32)).cuda()
    res = losses.preference_loss(x, y, off_d, ref_d, **kw)
    check_preference(torch, res, x, y, off, ref_d, kw)
    assert (res["dlogits"][:first] == 0).all() and (res["dlogits"][T - behind:] == 0).all()
    for _ in range(3):
        again = losses.preference_loss(x, y, off_d, ref_d, **kw)
        assert all(torch.equal(res[k], again[k]) for k in res)
    alone = losses.preference_loss(x, y, off_d, ref_d, grad=False, **kw)
    assert torch.equal(alone["loss"], res["loss"]) and torch.equal(alone["logp"], res["logp"])
    y[T // 2] = V
    bad = losses.preference_loss(x, y, off_d, ref_d, **kw)
    assert bad["loss"].isnan() and bad["dlogits"][T // 2].isnan().all()
    y[T // 2] = 0
    off_d[1] = T + 1
    bad = losses.preference_loss(x, y, off_d, ref_d, **kw)
    assert bad["loss"].isnan() and bad["dlogits"].isnan().all() and bad["logp"][0].isnan().all()
    off_d[1] = int(off[1])
    inside = losses.preference_loss(x, y, off_d, ref_d, out=x, **kw)
    assert inside["dlogits"] is x and x.isfinite().all()


def test_preference_of_impossible_answers(cuda, losses):
    """An answer of probability 0: the limits of the losses."""
    torch = cuda
    _, x, y = make(torch, torch.float32, 4, 30)
    off = torch.arange(5, dtype=torch.int32, device="cuda")
    x[1, int(y[1])] = -float("inf")                 # the rejected answer of the first pair
    for kind in ("sigmoid", "hinge"):
        res = losses.preference_loss(x, y, off, kind=kind, beta=0.01)
        rest = losses.preference_loss(x[2:], y[2:], off[:3], kind=kind, beta=0.01)
        assert res["logp"][0, 1] == -float("inf") and (res["dlogits"][:2] == 0).all()
        assert float(res["loss"]) == pytest.approx(float(rest["loss"]) / 2, rel=4 * U)
        assert (res["dlogits"][2:] == rest["dlogits"] / 2).all()
    assert losses.preference_loss(x, y, off, smoothing=0.1)["loss"] == float("inf")
    assert losses.preference_loss(x, y, off, kind="squared")["loss"] == float("inf")
    x[0, int(y[0])] = -float("inf")                 # and the chosen one
    assert losses.preference_loss(x, y, off)["loss"].isnan()


def check_policy(torch, res, x, y, old, adv, ref, kw, off=None):
    tau = kw.get("temperature", 1.0)
    okw = {("tau" if k == "temperature" else k): v for k, v in kw.items() if k != "offsets"}
    for k in ("kl", "scale"):
        if k in kw:
            okw[k] = float(np.float32(kw[k]))
    if off is not None:
        okw["off"] = off
    ys, h = y.cpu().numpy(), [None if v is None else v.double().cpu().numpy() for v in (old, adv, ref)]
    loss, terms, logp, coef = O.policy(on_host(x), ys, h[0], h[1], h[2], **okw)
    want, _, _, p, elogp, ep = rows_and_bounds(x, y, tau)
    assert (np.abs(on_host(res["logp"]) - want) <= elogp).all()
    # the ratio: logp's error and the difference's rounding in the exponent, 4 u of expf and the product
    w = O.policy_weights(ys, kw.get("reduction", "tokens"), off)
    r = np.where(w > 0, np.exp(logp - h[0]), 0.0)
    er = elogp + U * (np.abs(logp - h[0]) + 6)
    eterm = w * np.abs(h[1]) * r * er
    ekl = np.zeros_like(w)
    if h[2] is not None:
        u = np.where(w > 0, h[2] - logp, 0.0)
        eu = elogp + U * (np.abs(u) + 6)
        ekl = w * (np.exp(u) * eu + eu + U * (np.exp(u) + np.abs(u) + 1))
    kl, scale = abs(okw.get("kl", 0.0)), abs(okw.get("scale", 1.0))
    t = on_host(res["terms"])
    small = 4 * U
    assert abs(t[0] - terms[0]) <= eterm.sum() + small * (w * np.abs(h[1]) * (r + 1)).sum()
    assert abs(t[1] - terms[1]) <= ekl.sum() + small * abs(terms[1])
    assert abs(t[2] - terms[2]) <= small * abs(terms[2])
    etotal = scale * (eterm.sum() + kl * ekl.sum() + small * (w * np.abs(h[1]) * (r + 1)).sum() + small * kl * abs(terms[1]))
    assert abs(float(res["loss"]) - loss) <= etotal + small * abs(loss)
    ecoef = scale * (eterm + kl * (ekl + 4 * U * w)) + 8 * U * np.abs(coef)
    check_gradient(torch, res["dlogits"], x, y, coef, tau, p, ep, ecoef)


def away(drift, clip):
    """No ratio within a thousandth of a border of the clipping range, where the loss has no derivative."""
    for b in (np.log(1 - clip[0]) if clip[0] < 1 else -99.0, np.log(1 + clip[1])):
        drift = np.where(np.abs(drift - b) < 1e-3, drift + 4e-3, drift)
    return drift


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V,lens,kw", [
    (1000, [5, 1, 0, 9], dict()),
    (2, [30, 2], dict(kl=0.1, reduction="sequences")),
    (10, [400, 13, 1], dict(kl=0.05, clip=(0.1, 0.3), scale=2.0)),
    (257, [3, 0, 60], dict(reduction="sum", temperature=0.5)),
    (16, [33, 5], dict(kl=0.2)),
    (63, [37], dict(temperature=0.8)),
    (120, [41, 1], dict(kl=0.1, reduction="sequences")),
    (256, [19, 2], dict(kl=0.1)),
    (500, [6, 11], dict(reduction="sequences")),
    (10, [1, 0, 2, 3] * 400, dict(kl=0.1, reduction="sequences")),
    (10, [40] * 130, dict(reduction="sequences")),
    (4099, [3, 4], dict(kl=0.3, reduction="sequences", temperature=1.5)),
    (20003, [2, 0, 7], dict(kl=0.01)),
    (50001, [4, 1], dict(reduction="sequences")),
    (131073, [3], dict(kl=0.02, clip=(1.0, 0.0))),
    (262147, [2], dict()),
    (500000, [2], dict(kl=0.02))])
def test_policy(cuda, losses, dtype, V, lens, kw):
    torch = cuda
    sequences = kw.get("reduction") == "sequences"
    first, behind = (2, 3) if sequences else (0, 0)
    T = first + sum(lens) + behind
    r, x, y = make(torch, getattr(torch, dtype), T, V, masked=range(1, T, 6))
    off, off_d = offsets_of(torch, lens, first)
    logp = O.rows(on_host(x), y.cpu().numpy(), kw.get("temperature", 1.0))[0]
    drift = away(0.3 * r.standard_normal(T), kw.get("clip", (0.2, 0.2)))
    old, ref, adv = (torch.from_numpy(v.astype(np.float32)).cuda() for v in
                     (logp - drift, logp + 0.5 * r.standard_normal(T), r.standard_normal(T)))
    if sequences:
        kw = dict(kw, offsets=off_d)
    ref = ref if kw.get("kl") else None
    res = losses.policy_loss(x, y, old, adv, ref, **kw)
    check_policy(torch, res, x, y, old, adv, ref, kw, off if sequences else None)
    again = losses.policy_loss(x, y, old, adv, ref, **kw)
    assert all(torch.equal(res[k], again[k]) for k in res)
    alone = losses.policy_loss(x, y, old, adv, ref, grad=False, **kw)
    assert alone["dlogits"] is None and all(torch.equal(alone[k], res[k]) for k in ("loss", "terms", "logp"))


def test_policy_ratios_that_overflow(cuda, losses):
    torch = cuda
    _, x, y = make(torch, torch.float32, 4, 50)
    logp, _ = losses.token_logprob(x, y)
    old = logp.clone()
    old[0] -= 200.0                                  # ratio inf, clipped by a positive advantage
    old[1] -= 200.0                                  # and taken by none
    adv = torch.tensor([2.0, 0.0, 1.0, -1.0], device="cuda")
    res = losses.policy_loss(x, y, old, adv, reduction="sum")
    assert float(res["loss"]) == pytest.approx(-2.0 * 1.2 - 1.0 + 1.0, rel=1e-6)
    assert (res["dlogits"][:2] == 0).all() and res["dlogits"].isfinite().all()
    adv[0] = -2.0
    assert float(losses.policy_loss(x, y, old, adv, reduction="sum")["loss"]) == float("inf")
    # a KL term over a target that the policy cannot take
    x[2, int(y[2])] = -float("inf")
    res = losses.policy_loss(x, y, logp, adv, logp, kl=0.5)
    assert float(res["terms"][1]) == float("inf")


def expected_choice(x, k, mask):
    return O.balance(x, k, mask)[2]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (7, 5, 5), (33, 8, 1), (100, 64, 6), (257, 128, 8), (64, 256, 8),
                                   (1000, 7, 2), (40, 384, 16), (31, 1000, 3), (20, 1024, 64), (3000, 16, 4)])
@pytest.mark.parametrize("masked", [False, True])
def test_balance(cuda, losses, dtype, T, E, k, masked):
    torch = cuda
    dtype = getattr(torch, dtype)
    r, x, _ = make(torch, dtype, T, E, pad=E % 3, shift=E % 2)
    mask = None
    if masked:
        m = (r.random(T) < 0.7).astype(np.uint8) * 3
        mask = torch.from_numpy(m).cuda()
    res = losses.balance_loss(x, k, mask=mask, alpha=0.5)
    xs = on_host(x)
    loss, counts, choice, g = O.balance(xs, k, None if mask is None else m, alpha=0.5)
    assert (res["choice"].cpu().numpy() == choice).all()
    assert (res["counts"].cpu().numpy() == counts).all()
    check_balance(torch, res, xs, loss, counts, g, k, 0.5, T if mask is None else int((m > 0).sum()))
    again = losses.balance_loss(x, k, mask=mask, alpha=0.5)
    assert all(torch.equal(res[q], again[q]) for q in res)
    alone = losses.balance_loss(x, k, mask=mask, alpha=0.5, grad=False)
    assert torch.equal(alone["loss"], res["loss"]) and alone["dlogits"] is None
    inside = losses.balance_loss(x, k, mask=mask, alpha=0.5, out=x)
    assert torch.equal(x, res["dlogits"]) and torch.equal(inside["choice"], res["choice"])


def check_balance(torch, res, xs, loss, counts, g, k, alpha, n):
    """p's relative error e is that of the rows above (at most 32 additions deep per lane, 6 across), w's 2 u;
    the inner product s = w p adds positive terms, so s (e + chain); p (w - s) adds p |w - s| e + p (w + s)(...)."""
    E = xs.shape[1]
    D = xs.max(1, keepdims=True) - xs
    D = np.where(np.isfinite(D), D, 0.0)
    chain = 48
    with np.errstate(all="ignore"):
        p = np.where(np.isfinite(xs), np.exp(xs - xs.max(1, keepdims=True)), 0.0)
    p = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
    mean = (4 * D * p).sum(1, keepdims=True)
    e = U * (4 * D + mean + 12 + chain)
    w = alpha * E / (k * max(n, 1) ** 2) * counts[None, :]
    s = (p * w).sum(1, keepdims=True)
    es = (p * w * (e + chain * U)).sum(1, keepdims=True)
    h = half_step(torch, res["dlogits"].dtype)
    tol = p * (e * np.abs(w - s) + es + 4 * U * (w + s)) + h * np.abs(g)
    err = np.abs(on_host(res["dlogits"]) - g)
    assert (err <= tol * (1 + h) + 1e-37).all(), (err / (tol + 1e-37)).max()
    assert abs(float(res["loss"]) - loss) <= es.sum() + 2 * U * abs(loss)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("E", [5, 16, 33, 64, 128, 200, 256, 300, 512, 700])
def test_balance_choice_among_equals(cuda, losses, dtype, E):
    """Few distinct logits, zeros of both signs, infinities, NaN: the order is (value, lowest expert)."""
    torch = cuda
    r = np.random.default_rng(E)
    for k in (1, 2, 7, 8, 9, 33, 64):
        if k > E:
            continue
        for levels in (1, 2, 40, 100000):
            T = int(r.integers(1, 120))
            x = (r.integers(0, levels, (T, E)) - levels // 2).astype(np.float32) * np.float32(1e-3)
            for value, share in ((-np.inf, 0.1), (np.nan, 0.02), (-0.0, 0.02), (np.inf, 0.01)):
                x[r.random((T, E)) < share] = value
            x = torch.from_numpy(x).cuda().to(getattr(torch, dtype))
            mask = (r.random(T) < 0.8).astype(np.uint8)
            got = losses.balance_loss(x, k, mask=torch.from_numpy(mask).cuda(), grad=False)
            key = np.nan_to_num(x.float().cpu().numpy(), nan=-np.inf, posinf=np.inf, neginf=-np.inf) + 0.0
            order = np.argsort(-key, axis=1, kind="stable")[:, :k]
            want = np.where(np.take_along_axis(key, order, 1) > -np.inf, order, -1)
            want[mask == 0] = -1
            assert (got["choice"].cpu().numpy() == want).all(), (k, levels)
            assert (got["counts"].cpu().numpy() == np.bincount(want[want >= 0], minlength=E)).all()


def test_balance_ties_masks_and_given_choices(cuda, losses):
    torch = cuda
    x = torch.zeros(6, 40, device="cuda")
    x[1, 7:9] = 1.0
    x[2, :] = -float("inf")                         # no expert left
    x[3, 2:] = -float("inf")                        # fewer than k
    x[4, 39] = float("inf")
    x[5, 5:] = LOWEST
    x = x[[0, 1, 2, 3, 5]]
    res = losses.balance_loss(x, 3, alpha=1.0)
    assert res["choice"].tolist() == [[0, 1, 2], [7, 8, 0], [-1, -1, -1], [0, 1, -1], [0, 1, 2]]
    loss, counts, _, g = O.balance(on_host(x), 3, alpha=1.0)
    assert (res["dlogits"][2] == 0).all()
    check_balance(torch, res, np.where(np.isneginf(on_host(x)), -1e300, on_host(x)), loss, counts, g, 3, 1.0, 5)
    given = torch.tensor([[3, 3, 4], [-1, 40, 39], [0, 1, 2], [1, 1, 1], [39, 0, -7]], dtype=torch.int32, device="cuda")
    keep = given.clone()
    mask = torch.tensor([1, 1, 0, 1, 1], dtype=torch.uint8, device="cuda")
    res = losses.balance_loss(x, 3, mask=mask, choice=given, alpha=2.0)
    loss, counts, _, g = O.balance(on_host(x), 3, mask.cpu().numpy(), keep.cpu().numpy(), alpha=2.0)
    assert res["choice"] is given and torch.equal(given, keep)
    assert (res["counts"].cpu().numpy() == counts).all()
    check_balance(torch, res, np.where(np.isneginf(on_host(x)), -1e300, on_host(x)), loss, counts, g, 3, 2.0, 4)
    nothing = losses.balance_loss(x, 3, mask=torch.zeros_like(mask))
    assert float(nothing["loss"]) == 0 and (nothing["counts"] == 0).all() and (nothing["dlogits"] == 0).all()
    x[0, 3] = float("nan")
    bad = losses.balance_loss(x, 3)
    assert bad["loss"].isnan() and bad["dlogits"][0].isnan().any() and bad["dlogits"][1].isfinite().all()
    assert 3 not in bad["choice"][0].tolist()


def test_nothing_to_do(cuda, losses):
    torch = cuda
    x, y = torch.zeros(0, 9, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    f = torch.zeros(0, device="cuda")
    off = torch.zeros(1, dtype=torch.int32, device="cuda")
    logp, stats = losses.token_logprob(x, y)
    assert logp.shape == (0,) and losses.token_logprob_grad(x, y, stats, f).shape == (0, 9)
    assert float(losses.preference_loss(x, y, off)["loss"]) == 0
    assert float(losses.preference_loss(x, y, torch.zeros(3, dtype=torch.int32, device="cuda"))["loss"]) == \
        pytest.approx(np.log(2), rel=4 * U)
    for red in ("tokens", "sequences", "sum"):
        res = losses.policy_loss(x, y, f, f, reduction=red, offsets=off if red == "sequences" else None)
        assert float(res["loss"]) == 0 and (res["terms"] == 0).all()
    res = losses.balance_loss(x, 2)
    assert float(res["loss"]) == 0 and (res["counts"] == 0).all()
    # rows, but no targets and no sequences
    x, y = torch.randn(5, 9, device="cuda"), torch.full((5,), -1, dtype=torch.int32, device="cuda")
    f = torch.zeros(5, device="cuda")
    for red in ("tokens", "sequences", "sum"):
        res = losses.policy_loss(x, y, f, f, reduction=red, offsets=off if red == "sequences" else None)
        assert float(res["loss"]) == 0 and (res["dlogits"] == 0).all()
    y[:] = 2
    res = losses.policy_loss(x, y, f, f + 1, reduction="sequences", offsets=off)
    assert float(res["loss"]) == 0 and (res["dlogits"] == 0).all()
    res = losses.preference_loss(x, y, off)
    assert float(res["loss"]) == 0 and (res["dlogits"] == 0).all()


def test_targets_and_offsets_that_are_none(cuda, losses):
    torch = cuda
    for V in (50, 9001):
        _, x, y = make(torch, torch.bfloat16, 6, V)
        y[2] = V
        f = torch.zeros(6, device="cuda")
        logp, stats = losses.token_logprob(x, y)
        assert logp[2].isnan() and logp[[0, 1, 3, 4, 5]].isfinite().all()
        d = losses.token_logprob_grad(x, y, stats, f + 1)
        assert d[2].isnan().all() and d[[0, 1, 3, 4, 5]].isfinite().all()
        res = losses.policy_loss(x, y, f - 5, f + 1)
        assert res["loss"].isnan() and res["dlogits"][2].isnan().all() and res["dlogits"][[0, 1, 3]].isfinite().all()
        off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
        assert losses.preference_loss(x, y, off)["loss"].isnan()
        y[2] = 1
        many = [0] * 200 + [3, 2] + [4] * 199
        for bad in ([0, 3, 2], [-1, 3, 4], [0, 3, 7], [5, 3, 1], [0, -2, 4], [0, 1 << 30, 4], many):
            off = torch.tensor(bad, dtype=torch.int32, device="cuda")
            res = losses.preference_loss(x, y, off)
            assert res["loss"].isnan() and res["dlogits"].isnan().all(), bad
            res = losses.policy_loss(x, y, f - 5, f + 1, offsets=off, reduction="sequences")
            assert res["loss"].isnan() and res["terms"].isnan().all() and res["dlogits"].isnan().all(), bad


def test_far_offsets(cuda, losses):
    """Elements beyond 2^31 of a tensor are reached (bf16, 9.7 GB; a few rows carry targets)."""
    torch = cuda
    T, V = 37000, 131072
    x = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    y = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    sel = [0, 16384, 32768, T - 1]
    r = np.random.default_rng(3)
    rows = torch.from_numpy(r.standard_normal((4, V)).astype(np.float32)).cuda().bfloat16()
    x[sel] = rows
    yr = torch.from_numpy(r.integers(0, V, 4).astype(np.int32)).cuda()
    y[sel] = yr
    logp, stats = losses.token_logprob(x, y)
    want = losses.token_logprob(rows, yr)
    assert torch.equal(logp[sel], want[0]) and torch.equal(stats[sel], want[1])
    assert int((logp != 0).sum()) == 4
    small = losses.policy_loss(rows, yr, want[0], torch.ones(4, device="cuda"))
    res = losses.policy_loss(x, y, logp, torch.ones(T, device="cuda"), out=x)
    assert torch.equal(res["dlogits"][sel], small["dlogits"]) and res["loss"] == small["loss"]
    res["dlogits"][sel] = 0
    assert not res["dlogits"].any()


def step(losses, x, y, off, router):
    """One training step's losses: scores by a frozen copy, both losses over the answers, the router's balance."""
    ref, _ = losses.token_logprob(x.float() * 0.9, y)
    pol = losses.policy_loss(x, y, ref, ref * 0 + 1.5, ref, kl=0.1, offsets=off, reduction="sequences")
    pref = losses.preference_loss(x, y, off, beta=0.2, average=True)
    bal = losses.balance_loss(router, 2, mask=(y >= 0).to(y.dtype).byte(), alpha=0.1)
    return [ref, pol["loss"], pol["dlogits"], pref["loss"], pref["dlogits"], bal["loss"], bal["counts"], bal["dlogits"]]


def setting(torch, seed, V=3000, T=80):
    _, x, y = make(torch, torch.bfloat16, T, V, seed=seed, masked=range(0, T, 9))
    off = torch.tensor([0, 20, 35, 60, 80], dtype=torch.int32, device="cuda")
    _, router, _ = make(torch, torch.bfloat16, T, 16, seed=seed + 1)
    return x, y, off, router


def test_streams(cuda, losses):
    torch = cuda
    args = setting(torch, 5)
    want = step(losses, *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step(losses, *args)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # two calls at once, on streams that are given and on the current one
    others = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    out = [losses.preference_loss(*args[:3], beta=0.2, average=True, stream=s) for s in others]
    out.append(losses.preference_loss(*args[:3], beta=0.2, average=True, stream=others[0].cuda_stream))
    torch.cuda.synchronize()
    assert all(torch.equal(o["dlogits"], want[4]) and torch.equal(o["loss"], want[3]) for o in out)


def test_graphs(cuda, losses):
    """Two captured steps replayed at once, with new inputs in place."""
    torch = cuda
    sets = [setting(torch, 7), setting(torch, 8)]
    step(losses, *sets[0])
    graphs, outs, streams = [], [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(losses, *s))
        graphs.append(g)
        streams.append(torch.cuda.Stream())
    for seed in (11, 21):
        fresh = [setting(torch, seed), setting(torch, seed + 5)]
        for s, f in zip(sets, fresh):
            s[0].copy_(f[0]), s[1].copy_(f[1]), s[3].copy_(f[3])
        torch.cuda.synchronize()
        for _ in range(3):
            for g, q in zip(graphs, streams):
                with torch.cuda.stream(q):
                    g.replay()
        torch.cuda.synchronize()
        for s, o in zip(sets, outs):
            assert all(torch.equal(a, b) for a, b in zip(step(losses, *s), o))


def test_refusals(cuda, losses):
    torch = cuda
    x, y = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    f = torch.zeros(4, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    B = losses.B
    for bad in (lambda: losses.token_logprob(x.half(), y), lambda: losses.token_logprob(x[0], y),
                lambda: losses.token_logprob(x.t(), y), lambda: losses.token_logprob(x, y.long()),
                lambda: losses.token_logprob(x, y[:3]), lambda: losses.token_logprob(x, y.cpu()),
                lambda: losses.token_logprob(x[:, :0], y), lambda: losses.token_logprob(x[:1].expand(4, 8), y),
                lambda: losses.token_logprob_grad(x, y, f, f),
                lambda: losses.token_logprob_grad(x, y, torch.zeros(4, 2, device="cuda"), f, out=x.bfloat16()),
                lambda: losses.preference_loss(x, y, off[:2]), lambda: losses.preference_loss(x, y, off, f),
                lambda: losses.preference_loss(x, y, None),
                lambda: losses.policy_loss(x, y, f, f[:3]), lambda: losses.policy_loss(x, y, f, f, offsets=off),
                lambda: losses.policy_loss(x, y, f, f, reduction="sequences"),
                lambda: losses.policy_loss(x, y, f, f, grad=False, out=x),
                lambda: losses.balance_loss(x, 2, mask=y), lambda: losses.balance_loss(x, 2, choice=y)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    for bad in (lambda: losses.token_logprob(x, y, 0.0), lambda: losses.preference_loss(x, y, off, beta=0.0),
                lambda: losses.preference_loss(x, y, off, smoothing=2.0), lambda: losses.policy_loss(x, y, f, f, kl=0.1),
                lambda: losses.policy_loss(x, y, f, f, clip=(-1.0, 0.2)), lambda: losses.balance_loss(x, 0),
                lambda: losses.balance_loss(x, 9), lambda: losses.balance_loss(torch.zeros(2, 2000, device="cuda"), 2)):
        with pytest.raises(B.PGCError):
            bad()
    with pytest.raises(KeyError):
        losses.preference_loss(x, y, off, kind="none")


@pytest.mark.parametrize("which", ["preference", "policy", "balance"])
def test_differences(cuda, losses, which):
    """Along random directions d: (F(x + s d) - F(x - s d)) / 2 s, s = 2^-5.  Its error is s^2 / 6 |F'''| with
    |F'''| <= 8 max|d|^3 sum|coef| for these losses, and 2^-22 |F| / s of the losses' rounding."""
    torch = cuda
    T, V = 40, 300
    r, x, y = make(torch, torch.float32, T, V, seed=9)
    off = torch.tensor([0, 12, 20, 28, 40], dtype=torch.int32, device="cuda")
    logp, _ = losses.token_logprob(x, y)
    old = logp - 0.05
    adv = torch.from_numpy(r.standard_normal(T).astype(np.float32)).cuda()
    chosen = losses.balance_loss(x, 4)["choice"]
    f = {"preference": lambda v: losses.preference_loss(v, y, off, beta=0.3, average=True),
         "policy": lambda v: losses.policy_loss(v, y, old, adv, logp + 0.3, kl=0.2, clip=(0.9, 3.0)),
         "balance": lambda v: losses.balance_loss(v, 4, choice=chosen, alpha=1.0)}[which]
    base = f(x)
    s = 2.0 ** -5
    for _ in range(4):
        d = torch.from_numpy(r.uniform(-0.5, 0.5, (T, V)).astype(np.float32)).cuda()
        up, down = f(x + s * d)["loss"].double(), f(x - s * d)["loss"].double()
        want = float((base["dlogits"].double() * d.double()).sum())
        got = float((up - down) / (2 * s))
        tol = s * s / 6 * 8 * 0.125 * 3.0 + 2.0 ** -22 * (abs(float(up)) + abs(float(down)) + 1) / (2 * s)
        assert abs(got - want) <= tol, (got, want, tol)
