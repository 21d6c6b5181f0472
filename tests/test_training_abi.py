"""Token scores, experts' rows and AdamW without a GPU: bad arguments are
refused before any CUDA call."""

import ctypes as C

import pytest

from test_losses_abi import BAD_GRAD, BAD_ROWS, P, logits


def scores(B, z, k=4, logp=P, entropy=P, top=P, top_logp=P, stats=P):
    return B.lib.pgc_token_scores(z, k, logp, entropy, top, top_logp, stats, None)


def scores_grad(B, z, stats=P, entropy=P, dlogp=P, dentropy=P):
    return B.lib.pgc_token_scores_grad(z, stats, entropy, dlogp, dentropy, None)


@pytest.mark.parametrize("kw", [k for k in BAD_ROWS if k != dict(target=None)])
def test_rows_are_refused(libpgc, kw):
    B = libpgc
    assert scores(B, logits(B, **kw)) == B.EINVAL
    assert scores_grad(B, logits(B, **kw)) == B.EINVAL


@pytest.mark.parametrize("kw", BAD_GRAD)
def test_gradients_are_refused(libpgc, kw):
    assert scores_grad(libpgc, logits(libpgc, **kw)) == libpgc.EINVAL


@pytest.mark.parametrize("kw", [dict(k=-1), dict(logp=None), dict(entropy=None), dict(top=None), dict(top_logp=None),
                                dict(stats=None), dict(stats=P + 4), dict(logp=P + 2), dict(entropy=P + 1), dict(top=P + 2),
                                dict(top_logp=P + 1)])
def test_scores_are_refused(libpgc, kw):
    B = libpgc
    assert scores(B, logits(B), **kw) == B.EINVAL
    assert scores(B, logits(B, target=None), logp=P) == B.EINVAL
    assert scores(B, None) == B.EINVAL
    assert scores(B, logits(B), k=65) == B.ENOTSUP


@pytest.mark.parametrize("kw", [dict(stats=None), dict(entropy=None), dict(dlogp=None, dentropy=None), dict(stats=P + 4),
                                dict(entropy=P + 2), dict(dlogp=P + 1), dict(dentropy=P + 2)])
def test_scores_grad_is_refused(libpgc, kw):
    B = libpgc
    assert scores_grad(B, logits(B), **kw) == B.EINVAL
    assert scores_grad(B, None) == B.EINVAL
    assert scores_grad(B, logits(B, grad=None)) == B.EINVAL
    assert scores_grad(B, logits(B, target=None)) == B.EINVAL          # dlogp without targets


def test_no_rows_launch_nothing(libpgc):
    B = libpgc
    z = logits(B, rows=0, x=None, target=None, grad=None)
    assert scores(B, z, logp=None, entropy=None, top=None, top_logp=None, stats=None) == B.OK
    assert scores_grad(B, z, None, None, None, None) == B.OK
    # the gradient's fields are not looked at going forward
    assert scores(B, logits(B, rows=0, grad=P + 1, grad_ld=0)) == B.OK
    assert spread(B, tokens=0, x=None, place=None) == B.OK
    assert join(B, tokens=0, out=None, place=None) == B.OK
    assert join_grad(B, tokens=0, dy=None, place=None, weight=None, dweight=None) == B.OK
    assert adamw(B, []) == B.OK
    assert adamw(B, [tensor(B, n=0, param=None, grad=None, m=None, v=None), tensor(B, grad=None)]) == B.OK


def route(B, tokens=4, k=2, experts=8, choice=P, place=P, slot=P, offsets=P, ws=P, size=1 << 30):
    return B.lib.pgc_route(tokens, k, experts, choice, place, slot, offsets, ws, size, None)


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(k=0), dict(tokens=1 << 30, k=2), dict(tokens=1 << 31, k=1), dict(experts=0),
                                dict(choice=None), dict(place=None), dict(slot=None), dict(offsets=None), dict(ws=None),
                                dict(ws=P + 8), dict(choice=P + 1), dict(place=P + 2), dict(slot=P + 2), dict(offsets=P + 1)])
def test_route_is_refused(libpgc, kw):
    assert route(libpgc, **kw) == libpgc.EINVAL


def test_route_limits(libpgc):
    B = libpgc
    assert route(B, experts=1025) == B.ENOTSUP
    assert route(B, k=65) == B.ENOTSUP
    n = C.c_int64()
    assert B.lib.pgc_route_workspace(100, 8, 64, C.byref(n)) == B.OK and n.value > 0
    assert route(B, tokens=100, k=8, experts=64, size=n.value - 1) == B.ESCRATCH
    assert B.lib.pgc_route_workspace(100, 8, 64, None) == B.EINVAL
    assert B.lib.pgc_route_workspace(100, 8, 1025, C.byref(n)) == B.ENOTSUP
    sizes = []
    for tokens in (0, 1, 1000, 1 << 20):
        assert B.lib.pgc_route_workspace(tokens, 8, 256, C.byref(n)) == B.OK
        sizes.append(n.value)
    assert sizes == sorted(sizes)


def spread(B, dtype=1, tokens=4, k=2, d=16, x=P, ld=16, place=P, rows=8, out=P, out_ld=16):
    return B.lib.pgc_spread(dtype, tokens, k, d, x, ld, place, rows, out, out_ld, None)


def join(B, dtype=1, tokens=4, k=2, d=16, x=P, ld=16, rows=8, place=P, weight=P, out=P, out_ld=16):
    return B.lib.pgc_join(dtype, tokens, k, d, x, ld, rows, place, weight, out, out_ld, None)


def join_grad(B, dtype=1, tokens=4, k=2, d=16, dy=P, dy_ld=16, x=P, ld=16, rows=8, place=P, weight=P, out=P, out_ld=16, dweight=P):
    return B.lib.pgc_join_grad(dtype, tokens, k, d, dy, dy_ld, x, ld, rows, place, weight, out, out_ld, dweight, None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(tokens=-1), dict(k=0), dict(tokens=1 << 30, k=2), dict(d=0), dict(d=1 << 31), dict(d=(1 << 30) + 1, ld=1 << 31, out_ld=1 << 31),
                                dict(ld=15), dict(out_ld=15), dict(ld=(1 << 31) + 1), dict(rows=-1), dict(rows=1 << 31), dict(x=None),
                                dict(out=None), dict(place=None), dict(place=P + 2), dict(x=P + 1), dict(out=P + 1),
                                dict(dtype=0, x=P + 2), dict(dtype=0, out=P + 2)])
def test_moves_are_refused(libpgc, kw):
    B = libpgc
    assert spread(B, **kw) == B.EINVAL
    assert join(B, **kw) == B.EINVAL
    assert join_grad(B, **kw) == B.EINVAL


def test_other_moves_are_refused(libpgc):
    B = libpgc
    for f in (spread, join, join_grad):
        assert f(B, k=65) == B.ENOTSUP
    assert join(B, weight=P + 1) == B.EINVAL
    for kw in (dict(weight=None), dict(dweight=None), dict(weight=P + 2), dict(dweight=P + 1), dict(dy=None), dict(dy=P + 1),
               dict(dy_ld=15), dict(out=P, x=P, out_ld=17)):
        assert join_grad(B, **kw) == B.EINVAL


def tensor(B, **kw):
    v = dict(param=P, grad=P, copy=None, m=P, v=P, m_scale=P, v_scale=P, n=10)
    v.update(kw)
    return B.AdamWTensor(*[v[n] for n, _ in B.AdamWTensor._fields_])


def adamw(B, tensors, count=None, **kw):
    v = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, step_at=None, lr_at=None, grad_scale=None,
             seed=0, param_dtype=B.F32, grad_dtype=B.F32, bits=32)
    v.update(kw)
    s = B.AdamW(*[v[n] for n, _ in B.AdamW._fields_])
    return B.lib.pgc_adamw_step(s, (B.AdamWTensor * len(tensors))(*tensors), len(tensors) if count is None else count, None)


@pytest.mark.parametrize("kw", [dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=-0.1), dict(beta1=1.0), dict(beta2=1.0),
                                dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("inf")), dict(weight_decay=float("nan")),
                                dict(step=0), dict(step=-1), dict(step_at=P + 4), dict(lr_at=P + 2), dict(grad_scale=P + 1),
                                dict(param_dtype=2), dict(grad_dtype=-1), dict(bits=16), dict(count=-1), dict(count=1 << 31)])
def test_adamw_is_refused(libpgc, kw):
    assert adamw(libpgc, [tensor(libpgc)], **kw) == libpgc.EINVAL


@pytest.mark.parametrize("kw", [dict(param=None), dict(m=None), dict(v=None), dict(n=-1), dict(n=(1 << 38) + 1), dict(param=P + 2),
                                dict(grad=P + 1), dict(copy=P + 1), dict(m=P + 2), dict(v=P + 1)])
def test_tensors_are_refused(libpgc, kw):
    """Also behind a good one: nothing is launched before all are seen."""
    B = libpgc
    assert adamw(B, [tensor(B), tensor(B, **kw)]) == B.EINVAL


def test_scales_are_asked_for_with_8_bits(libpgc):
    B = libpgc
    for kw in (dict(m_scale=None), dict(v_scale=None), dict(m_scale=P + 2), dict(v_scale=P + 1)):
        assert adamw(B, [tensor(B, **kw)], bits=8) == B.EINVAL
    assert B.lib.pgc_adamw_step(None, None, 0, None) == B.EINVAL


def test_torch_forms_refuse(libpgc):
    torch = pytest.importorskip("torch")
    from paper_2607_20739_gb300 import experts, losses, optim
    x, y = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        losses.token_scores(x, y)
    with pytest.raises(TypeError):
        losses.token_scores_grad(x.numpy(), y, y)
    with pytest.raises(ValueError, match="CUDA"):
        experts.route(torch.zeros(4, 2, dtype=torch.int32), 8)
    with pytest.raises(TypeError):
        experts.route([[1]], 8)
    r = experts.Routes(4, 2, 8, torch.zeros(4, 2, dtype=torch.int32), None, None)
    with pytest.raises(ValueError, match="CUDA"):
        experts.spread(x, r)
    with pytest.raises(ValueError, match="CUDA"):
        experts.join(x, r)
    with pytest.raises(ValueError, match="CUDA"):
        optim.AdamW([x])
    with pytest.raises(TypeError):
        optim.AdamW([x.numpy()])
    with pytest.raises(ValueError, match="bits"):
        optim.AdamW([], bits=16)
    optim.AdamW([]).step([])
    with pytest.raises(ValueError, match="grads"):
        optim.AdamW([]).step([x])
