"""Losses on rows of logits where rows are split, many to a CTA, masked or far
from zero, against the 64-bit oracle (bounds: test_gpu_row_losses.py)."""

import numpy as np
import pytest

from test_gpu_row_losses import U, check_gradient, check_policy, losses, make, on_host, rows_and_bounds  # noqa: F401

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
