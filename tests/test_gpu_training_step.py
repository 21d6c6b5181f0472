"""The operators of a training step together: a layer of experts between two
products, trained by log probabilities with an entropy bonus and the router's
balance loss, updated by AdamW; against autograd of the same layer in 64 bits."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def reference(torch, W, x, y, a, b, choice, k, alpha, counts, n):
    """Loss and gradients by autograd in 64 bits, with the experts that were chosen."""
    P = {name: w.detach().double().requires_grad_(True) for name, w in W.items()}
    h = x.double() @ P["in"]
    gate = torch.softmax(h @ P["router"], 1)
    weight = torch.gather(gate, 1, choice.long())
    out = torch.zeros_like(h)
    for j in range(k):
        made = torch.bmm(h[:, None, :], P["experts"][choice[:, j].long()])[:, 0]
        out = out + weight[:, j:j + 1] * made
    q = torch.log_softmax(out @ P["head"], 1)
    loss = (q[torch.arange(len(y)), y.long()] * a.double()).sum() + (-(q.exp() * q).sum(1) * b.double()).sum()
    loss = loss + alpha * counts.numel() / (k * n * n) * (gate.sum(0) * counts.double()).sum()
    loss.backward()
    return {name: p.grad for name, p in P.items()}


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_of_a_model_with_experts(cuda, bits):
    torch = cuda
    from paper_2607_20739_gb300 import experts, losses, optim
    T, d, E, k, V, alpha = 200, 48, 12, 3, 501, 0.01
    g = torch.Generator(device="cuda").manual_seed(3)
    W = {"in": torch.randn(d, d, generator=g, device="cuda") / d ** 0.5, "router": torch.randn(d, E, generator=g, device="cuda") * 0.3,
         "experts": torch.randn(E, d, d, generator=g, device="cuda") / d ** 0.5, "head": torch.randn(d, V, generator=g, device="cuda") * 0.3}
    x = torch.randn(T, d, generator=g, device="cuda")
    y = torch.randint(V, (T,), generator=g, device="cuda").to(torch.int32)
    a, b = -torch.ones(T, device="cuda") / T, torch.full((T,), -0.1 / T, device="cuda")
    opt = optim.AdamW(list(W.values()), lr=1e-3, bits=bits)
    torch.backends.cuda.matmul.allow_tf32 = False
    for t in range(3):
        h = x @ W["in"]
        router = h @ W["router"]
        bal = losses.balance_loss(router, k, alpha=alpha)
        choice = bal["choice"]
        gate = torch.softmax(router, 1)
        weight = torch.gather(gate, 1, choice.long())
        r = experts.route(choice, E)
        assert torch.equal(r.offsets[1:] - r.offsets[:-1], bal["counts"])
        rows = experts.spread(h, r)
        ends = r.offsets.tolist()
        spans = [slice(ends[e], ends[e + 1]) for e in range(E)]
        made = torch.cat([rows[s] @ W["experts"][e] for e, s in enumerate(spans)])
        out = experts.join(made, r, weight)
        logits = out @ W["head"]
        s = losses.token_scores(logits, y, 5)
        assert torch.equal(s["top"][:, 0].long(), logits.argmax(1))

        dlogits = losses.token_scores_grad(logits, y, s["stats"], s["entropy"], a, b)
        dout = dlogits @ W["head"].t()
        dmade, dweight = experts.join_grad(dout, made, r, weight)
        drows = torch.cat([dmade[q] @ W["experts"][e].t() for e, q in enumerate(spans)])
        dexperts = torch.stack([rows[q].t() @ dmade[q] for e, q in enumerate(spans)])
        dgate = torch.zeros_like(gate).scatter_(1, choice.long(), dweight)
        drouter = gate * (dgate - (gate * dgate).sum(1, keepdim=True)) + bal["dlogits"]
        dh = experts.spread_grad(drows, r) + drouter @ W["router"].t()
        grads = {"in": x.t() @ dh, "router": h.t() @ drouter, "experts": dexperts, "head": out.t() @ dlogits}

        want = reference(torch, W, x, y, a, b, choice, k, alpha, bal["counts"], T)
        for name in W:
            # sums of at most T V products in single precision, a few products deep
            rel = float((grads[name].double() - want[name]).norm() / want[name].norm())
            assert rel < 1e-5, (name, rel)
        old = {name: w.clone() for name, w in W.items()}
        opt.step([grads[name] for name in W])
        for name in W:
            moved = (W[name] - old[name]).abs()
            assert torch.isfinite(W[name]).all() and moved.max() > 0
            if t == 0:                      # a first step is lr against the gradient, and the decay
                keep = old[name].double() * (1 - 1e-3 * 0.01)
                step = 1e-3 * grads[name].double() / (grads[name].double().abs() + 1e-8)
                assert ((W[name].double() - (keep - step)).abs() <= 2.0 ** -24 * 40 * (1e-3 + old[name].double().abs())).all()
