"""What a call does not use it does not check."""

from test_losses_abi import P, logits


def test_token_logprob_does_not_look_at_the_gradient(libpgc):
    B = libpgc
    for kw in (dict(grad_ld=0), dict(grad=P + 1), dict(grad=P, x=P, grad_ld=16), dict(grad_ld=(1 << 31) + 1)):
        z = logits(B, rows=0, **kw)                 # no rows: nothing is launched
        assert B.lib.pgc_token_logprob(z, None, None, None) == B.OK, kw
        assert B.lib.pgc_token_logprob_grad(z, None, None, None) == B.EINVAL, kw
