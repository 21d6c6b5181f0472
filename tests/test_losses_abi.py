"""The losses on rows of logits without a GPU: bad arguments are refused
before any CUDA call, and workspace sizes are monotone in the sizes."""

import ctypes as C

import pytest

P = 1 << 20            # an aligned address that no refused call follows


def logits(B, **kw):
    v = dict(x=P, target=P, grad=P, rows=4, classes=10, ld=10, grad_ld=10, dtype=B.BF16, temperature=1.0)
    v.update(kw)
    return B.Logits(*[v[n] for n, _ in B.Logits._fields_])


BAD_ROWS = [dict(x=None), dict(target=None), dict(rows=-1), dict(rows=1 << 31), dict(classes=0), dict(classes=1 << 31),
            dict(ld=9), dict(ld=(1 << 31) + 1), dict(dtype=2), dict(dtype=-1), dict(temperature=0.0),
            dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
            dict(temperature=1e-45), dict(temperature=4e-39), dict(x=P + 1), dict(target=P + 2), dict(dtype=0, x=P + 2)]
BAD_GRAD = [dict(grad_ld=9), dict(grad_ld=(1 << 31) + 1), dict(grad=P + 1), dict(grad=P, x=P, grad_ld=16),
            dict(dtype=0, grad=P + 2)]


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_rows_are_refused(libpgc, kw):
    B = libpgc
    z = logits(B, **kw)
    assert B.lib.pgc_token_logprob(z, P, P, None) == B.EINVAL
    assert B.lib.pgc_token_logprob_grad(z, P, P, None) == B.EINVAL
    assert preference(B, z) == B.EINVAL
    assert policy(B, z) == B.EINVAL


@pytest.mark.parametrize("kw", BAD_GRAD)
def test_gradients_are_refused(libpgc, kw):
    B = libpgc
    z = logits(B, **kw)
    assert B.lib.pgc_token_logprob_grad(z, P, P, None) == B.EINVAL
    assert preference(B, z) == B.EINVAL
    assert policy(B, z) == B.EINVAL


def test_null_structures_and_outputs(libpgc):
    B, z = libpgc, logits(libpgc)
    assert B.lib.pgc_token_logprob(None, P, P, None) == B.EINVAL
    assert B.lib.pgc_token_logprob(z, None, P, None) == B.EINVAL
    assert B.lib.pgc_token_logprob(z, P, None, None) == B.EINVAL
    assert B.lib.pgc_token_logprob(z, P, P + 4, None) == B.EINVAL          # pairs of floats
    assert B.lib.pgc_token_logprob_grad(None, P, P, None) == B.EINVAL
    assert B.lib.pgc_token_logprob_grad(logits(B, grad=None), P, P, None) == B.EINVAL
    assert B.lib.pgc_token_logprob_grad(z, None, P, None) == B.EINVAL
    assert B.lib.pgc_token_logprob_grad(z, P, None, None) == B.EINVAL


def preference(B, z, kind=0, pairs=1, off=P, ref=None, beta=0.1, margin=0.0, smoothing=0.0, scale=1.0, loss=P, logp=P,
               ws=P, size=1 << 30):
    return B.lib.pgc_preference_loss(z, kind, pairs, off, ref, beta, margin, smoothing, 0, scale, loss, logp, ws, size,
                                     None)


@pytest.mark.parametrize("kw", [
    dict(kind=3), dict(kind=-1), dict(pairs=-1), dict(pairs=1 << 31), dict(off=None), dict(off=P + 1), dict(ref=P + 2),
    dict(beta=0.0), dict(beta=-1.0), dict(beta=float("nan")), dict(margin=float("inf")), dict(smoothing=-0.1),
    dict(smoothing=1.1), dict(scale=float("nan")), dict(loss=None), dict(logp=None), dict(ws=None), dict(ws=P + 8)])
def test_preference_is_refused(libpgc, kw):
    assert preference(libpgc, logits(libpgc), **kw) == libpgc.EINVAL


def policy(B, z, reduction=0, sequences=0, off=None, old=P, adv=P, ref=None, low=0.2, high=0.2, kl=0.0, scale=1.0,
           loss=P, terms=P, logp=P, ws=P, size=1 << 30):
    return B.lib.pgc_policy_loss(z, reduction, sequences, off, old, adv, ref, low, high, kl, scale, loss, terms, logp,
                                 ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(reduction=3), dict(reduction=-1), dict(reduction=1, sequences=1), dict(reduction=1, sequences=-1, off=P),
    dict(old=None), dict(adv=None), dict(kl=0.1), dict(kl=float("nan"), ref=P), dict(low=-0.1), dict(low=1.5),
    dict(high=-0.1), dict(high=float("inf")), dict(scale=float("inf")), dict(loss=None), dict(terms=None),
    dict(logp=None), dict(ws=None), dict(ws=P + 4), dict(old=P + 1), dict(adv=P + 2), dict(ref=P + 3)])
def test_policy_is_refused(libpgc, kw):
    assert policy(libpgc, logits(libpgc), **kw) == libpgc.EINVAL


def balance(B, dtype=1, rows=4, experts=8, x=P, ld=8, mask=None, k=2, given=0, choice=P, alpha=0.01, loss=P, counts=P,
            grad=P, grad_ld=8, ws=P, size=1 << 30):
    return B.lib.pgc_balance_loss(dtype, rows, experts, x, ld, mask, k, given, choice, alpha, loss, counts, grad,
                                  grad_ld, ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(experts=0), dict(k=0), dict(k=9), dict(ld=7),
    dict(grad_ld=7), dict(alpha=float("nan")), dict(x=None), dict(choice=None), dict(loss=None), dict(counts=None),
    dict(ws=None), dict(ws=P + 8), dict(x=P + 1), dict(grad=P + 1), dict(choice=P + 2), dict(grad=P, grad_ld=9),
    dict(dtype=0, x=P + 2)])
def test_balance_is_refused(libpgc, kw):
    assert balance(libpgc, **kw) == libpgc.EINVAL


def test_balance_limits(libpgc):
    assert balance(libpgc, experts=1025, ld=1025, grad_ld=1025) == libpgc.ENOTSUP
    assert balance(libpgc, experts=128, ld=128, grad_ld=128, k=65) == libpgc.ENOTSUP


def workspace(f, *args):
    n = C.c_int64(-1)
    return f(*args, C.byref(n)), n.value


def test_workspace_sizes(libpgc):
    B = libpgc
    sizes = [workspace(B.lib.pgc_loss_workspace, r, s) for r, s in [(0, 0), (1, 0), (1000, 0), (1000, 10000), (1 << 20, 0)]]
    assert all(rc == B.OK for rc, _ in sizes)
    assert [n for _, n in sizes] == sorted(n for _, n in sizes) and sizes[0][1] > 0
    for args in [(-1, 0), (0, -1), (1 << 31, 0), (0, 1 << 31)]:
        assert workspace(B.lib.pgc_loss_workspace, *args)[0] == B.EINVAL
    assert B.lib.pgc_loss_workspace(1, 1, None) == B.EINVAL
    rc, n = workspace(B.lib.pgc_balance_workspace, 100, 8)
    assert rc == B.OK and n > 0
    for args in [(-1, 8), (1 << 31, 8), (4, 0), (4, 1025)]:
        assert workspace(B.lib.pgc_balance_workspace, *args)[0] == B.EINVAL
    # one byte short
    z = logits(B, rows=1000, grad=None)
    need = workspace(B.lib.pgc_loss_workspace, 1000, 4)[1]
    assert preference(B, z, pairs=2, size=need - 1) == B.ESCRATCH
    need = workspace(B.lib.pgc_loss_workspace, 1000, 0)[1]
    assert policy(B, z, size=need - 1) == B.ESCRATCH
    assert balance(B, size=n - 1) == B.ESCRATCH


def test_tensors_are_refused(libpgc):
    torch = pytest.importorskip("torch")
    from paper_2607_20739_gb300 import losses
    x, y = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        losses.token_logprob(x, y)
    with pytest.raises(TypeError):
        losses.balance_loss(x.numpy(), 2)
    with pytest.raises(ValueError, match="CUDA"):
        losses.policy_loss(x, y, x[:, 0], x[:, 0])
