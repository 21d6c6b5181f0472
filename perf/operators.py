"""Losses on rows of logits, with their gradients, as cases to be measured.

A user's program has the logits of a step in hand (one row per token, from a
product that another library or a kernel of its own made) and asks for a loss
over them and for the loss's gradient with respect to every logit:

  logprob       log softmax at each row's target, which the reference model and
                the sampling policy are scored with (direction "forward"), and
                its gradient for given weights of the rows (direction "gradient")
  preference    paired log ratios of whole sequences: chosen against rejected
  policy        clipped probability ratios with a KL term
  balance       a router's top k choice, its per-expert counts and its balance loss

Every case is one call that such a program makes once a step.  With ``own``
false the same results come from elementary torch operations in single
precision (sums over sequences in double).
"""

from __future__ import annotations

import math

import torch

own = False


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _logprob(name, direction, T, V, dtype, masked=False, temperature=1.0):
    """T rows of V logits; masked: one row in eight has no target."""
    return {"name": name, "op": "logprob", "direction": direction, "T": T, "V": V, "dtype": dtype, "masked": masked,
            "temperature": temperature}


def _preference(name, pairs, length, V, dtype, kind="sigmoid", smoothing=0.0, average=False, prompt=False):
    """pairs of sequences of up to length rows; prompt: the first quarter of each has no target."""
    return {"name": name, "op": "preference", "pairs": pairs, "length": length, "V": V, "dtype": dtype, "kind": kind,
            "smoothing": smoothing, "average": average, "prompt": prompt}


def _policy(name, sequences, length, V, dtype, kl=0.0, reduction="tokens", prompt=False, temperature=1.0):
    return {"name": name, "op": "policy", "sequences": sequences, "length": length, "V": V, "dtype": dtype, "kl": kl,
            "reduction": reduction, "prompt": prompt, "temperature": temperature}


def _balance(name, T, E, k, dtype, masked=False):
    """T tokens routed to k of E experts; masked: one token in eight is padding."""
    return {"name": name, "op": "balance", "T": T, "E": E, "k": k, "dtype": dtype, "masked": masked}


def listed():
    return [
        # one token scored against a vocabulary: a call is its latency
        _logprob("logprob_t1_v32768", "forward", 1, 32768, "bf16"),
        # a batch scored by the reference model, a large vocabulary: bound by reading the logits
        _logprob("logprob_t4096_v131072", "forward", 4096, 131072, "bf16"),
        # the gradient in single precision over an odd vocabulary, whose rows start at every 4-byte offset
        _logprob("logprob_grad_t2000_v50001_f32", "gradient", 2000, 50001, "f32", masked=True),
        # a preference head over a thousand classes, short answers: small enough to be launches
        _preference("preference_p4_l48_v1000_f32", 4, 48, 1000, "f32"),
        # an ordinary preference step: sixteen pairs of answers behind their prompts
        _preference("preference_p16_l256_v32768", 16, 256, 32768, "bf16", prompt=True),
        # long answers, large vocabulary, per-token averages and squared error
        _preference("preference_p4_l1000_v131072", 4, 1000, 131072, "bf16", kind="squared", average=True),
        # a policy over a thousand actions, a few hundred decisions
        _policy("policy_s8_l40_v1000", 8, 40, 1000, "bf16"),
        # an ordinary policy step: answers behind prompts, KL to a reference, mean of sequence means
        _policy("policy_s32_l256_v32768", 32, 256, 32768, "bf16", kl=0.05, reduction="sequences", prompt=True),
        # an odd vocabulary in half precision, a sampling temperature
        _policy("policy_s12_l300_v100003", 12, 300, 100003, "bf16", kl=0.01, temperature=0.7),
        # a router of eight experts, one sequence
        _balance("balance_t512_e8_k2_f32", 512, 8, 2, "f32"),
        # a router of 128 experts over a padded batch
        _balance("balance_t16384_e128_k8", 16384, 128, 8, "bf16", masked=True),
        # the largest batch and router in single precision
        _balance("balance_t65536_e256_k8_f32", 65536, 256, 8, "f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = 4096 * 131072        # logits of a drawn case at most


def draw(rng):
    op = rng.choice(["logprob", "preference", "policy", "balance"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    most = MOST if dtype == "bf16" else MOST // 2
    if op == "balance":
        E = rng.choice([8, 16, 64, 128, 256, rng.randint(4, 384)])
        T = min(_log_uniform(rng, 1, 65536), 65536 * 256 // E)
        case = _balance("", T, E, rng.randint(1, min(8, E)), dtype, rng.random() < 0.5)
    else:
        V = rng.choice([1000, 32768, 65536, 131072, _log_uniform(rng, 100, 200000), _log_uniform(rng, 20000, 200000)])
        rows = max(1, most // V)
        temperature = rng.choice([1.0, 1.0, 0.6, 1.3])
        if op == "logprob":
            T = _log_uniform(rng, 1, min(rows, 16384))
            case = _logprob("", rng.choice(["forward", "gradient"]), T, V, dtype, rng.random() < 0.5, temperature)
        else:
            length = _log_uniform(rng, 1, min(2048, max(1, rows // 2)))
            most_seq = max(1, min(rows, 16384) // length)
            prompt = rng.random() < 0.5
            if op == "preference":
                pairs = _log_uniform(rng, 1, max(1, min(64, most_seq // 2)))
                case = _preference("", pairs, length, V, dtype, rng.choice(["sigmoid", "hinge", "squared"]),
                                   rng.choice([0.0, 0.1]), rng.random() < 0.3, prompt)
            else:
                sequences = _log_uniform(rng, 1, min(128, most_seq))
                case = _policy("", sequences, length, V, dtype, rng.choice([0.0, 0.01, 0.1]),
                               rng.choice(["tokens", "sequences"]), prompt, temperature)
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

BETA = 0.1                  # the preference loss's inverse temperature of log ratios
CLIP = (0.2, 0.28)
ALPHA = 0.01                # the balance loss's coefficient


def _lengths(case):
    """Rows of every sequence, prompt and answer."""
    n = 2 * case["pairs"] if case["op"] == "preference" else case["sequences"]
    m = case["length"]
    return [m - (i * 29 + 7) % (m // 2 + 1) for i in range(n)]


def _prompts(case):
    return [m // 4 if case["prompt"] else 0 for m in _lengths(case)]


def _rows(case):
    return case["T"] if "T" in case else sum(_lengths(case))


def _generator(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + k) % (1 << 62))
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _logits(case, seed):
    """Logits as a model gives them: a spread of a few units, the target's
    usually among the largest."""
    T, V = _rows(case), case["V"] if "V" in case else case["E"]
    g = _generator(seed, 1)
    x = torch.empty((T, V), dtype=_dtype(case), device="cuda")
    for r in range(0, T, 1024):
        n = min(1024, T - r)
        x[r:r + n] = torch.randn((n, V), generator=g, device="cuda") * 2.0
    return x


def _targets(case, seed, x):
    T, V = x.shape
    g = _generator(seed, 2)
    y = torch.randint(V, (T,), generator=g, device="cuda")
    boost = 12.0 * torch.rand((T,), generator=g, device="cuda")
    at = torch.arange(T, device="cuda")
    x[at, y] = (x[at, y].float() + boost).to(x.dtype)
    y = y.to(torch.int32)
    if case["op"] == "logprob":
        if case["masked"]:
            y[3::8] = -1
    else:
        start = 0
        for m, p in zip(_lengths(case), _prompts(case)):
            y[start:start + p] = -1
            start += m
    return y


def _offsets(case):
    at = [0]
    for m in _lengths(case):
        at.append(at[-1] + m)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _logp64(x, y, temperature):
    """Log probability of every row's target in double, zero without one."""
    out = torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
    for r in range(0, x.shape[0], 1024):
        z = x[r:r + 1024].double() / temperature
        t = y[r:r + 1024].long()
        lp = z.gather(1, t.clamp(min=0)[:, None])[:, 0] - torch.logsumexp(z, 1)
        out[r:r + 1024] = torch.where(t >= 0, lp, torch.zeros_like(lp))
    return out


def _away_from_borders(ratio_log):
    """The clipped loss has no derivative at a border of its clipping range:
    no ratio lies within a thousandth of one."""
    for border in (math.log(1.0 - CLIP[0]), math.log(1.0 + CLIP[1])):
        near = (ratio_log - border).abs() < 1e-3
        ratio_log = torch.where(near, ratio_log + 4e-3, ratio_log)
    return ratio_log


def prepare(case, seed):
    g = _generator(seed, 3)
    x = _logits(case, seed)
    T = x.shape[0]
    state = {"case": case, "logits": x}
    if case["op"] == "balance":
        # routers favour some experts
        x += (torch.randn((x.shape[1],), generator=g, device="cuda") * 0.7).to(x.dtype)
        state["mask"] = None
        if case["masked"]:
            state["mask"] = torch.ones(T, dtype=torch.uint8, device="cuda")
            state["mask"][5::8] = 0
        return state
    y = state["target"] = _targets(case, seed, x)
    if case["op"] == "logprob":
        if case["direction"] == "gradient":
            state["dlogp"] = torch.randn((T,), generator=g, device="cuda") / T
            # what the forward call returned beside the log probabilities: the
            # largest logit, and the logarithm of the sum of the exponentials of
            # the logits' distances from it over the temperature
            state["stats"] = _stats64(x, y, case["temperature"]).float()
        return state
    off = state["offsets"] = _offsets(case)
    logp = _logp64(x, y, case["temperature"] if case["op"] == "policy" else 1.0)
    if case["op"] == "preference":
        sums = torch.stack([logp[a:b].sum() for a, b in _spans(case)])
        counts = torch.tensor([max(1, m - p) for m, p in zip(_lengths(case), _prompts(case))], device="cuda")
        if case["average"]:
            sums = sums / counts
        noise = torch.randn(sums.shape, generator=g, device="cuda").double() * (0.5 if case["average"] else 6.0)
        state["ref_logp"] = (sums - noise).float().view(-1, 2)
    else:
        drift = _away_from_borders(torch.randn((T,), generator=g, device="cuda").double() * 0.2)
        state["old_logp"] = (logp - drift).float()
        state["ref_logp"] = (logp - torch.randn((T,), generator=g, device="cuda").double() * 0.4).float() \
            if case["kl"] else None
        gain = torch.randn((off.numel() - 1,), generator=g, device="cuda")
        state["advantage"] = torch.repeat_interleave(gain, (off[1:] - off[:-1]).long()).contiguous()
    return state


def _spans(case):
    at = 0
    for m in _lengths(case):
        yield at, at + m
        at += m


def _stats64(x, y, temperature):
    out = torch.zeros((x.shape[0], 2), dtype=torch.float64, device="cuda")
    for r in range(0, x.shape[0], 1024):
        z = x[r:r + 1024].double() / temperature
        top = z.max(1).values
        s = torch.stack([x[r:r + 1024].amax(1).double(), torch.log(torch.exp(z - top[:, None]).sum(1))], 1)
        out[r:r + 1024] = torch.where((y[r:r + 1024] >= 0)[:, None], s, torch.zeros_like(s))
    return out


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    case = state["case"]
    op = _OWN if own else _PLAIN
    return op[case["op"]](state, case)


def _own_logprob(s, case):
    from paper_2607_20739_gb300 import losses
    if case["direction"] == "forward":
        logp, stats = losses.token_logprob(s["logits"], s["target"], temperature=case["temperature"])
        return {"logp": logp, "stats": stats}
    return {"dlogits": losses.token_logprob_grad(s["logits"], s["target"], s["stats"], s["dlogp"],
                                                 temperature=case["temperature"])}


def _own_preference(s, case):
    from paper_2607_20739_gb300 import losses
    r = losses.preference_loss(s["logits"], s["target"], s["offsets"], s["ref_logp"], beta=BETA, kind=case["kind"],
                               smoothing=case["smoothing"], average=case["average"])
    return {"loss": r["loss"], "logp": r["logp"], "dlogits": r["dlogits"]}


def _own_policy(s, case):
    from paper_2607_20739_gb300 import losses
    r = losses.policy_loss(s["logits"], s["target"], s["old_logp"], s["advantage"], s["ref_logp"], clip=CLIP,
                           kl=case["kl"], offsets=s["offsets"] if case["reduction"] == "sequences" else None,
                           reduction=case["reduction"], temperature=case["temperature"])
    return {"loss": r["loss"], "terms": r["terms"], "logp": r["logp"], "dlogits": r["dlogits"]}


def _own_balance(s, case):
    from paper_2607_20739_gb300 import losses
    r = losses.balance_loss(s["logits"], case["k"], mask=s["mask"], alpha=ALPHA)
    return {"loss": r["loss"], "counts": r["counts"], "choice": r["choice"], "dlogits": r["dlogits"]}


_OWN = {"logprob": _own_logprob, "preference": _own_preference, "policy": _own_policy, "balance": _own_balance}


def _row_stats(x, temperature):
    """Logits over temperature, their maximum, exponentials and the sum of these."""
    z = x.float() / temperature
    top = torch.amax(z, 1)
    e = torch.exp(z - top[:, None])
    return z, top, e, e.sum(1)


def _at_target(z, y):
    return z.gather(1, y.long().clamp(min=0)[:, None])[:, 0]


def _row_gradient(p, y, coef, temperature, dtype):
    """coef times the gradient of the target's log probability, rounded once; p is overwritten."""
    coef = torch.where(y >= 0, coef, torch.zeros_like(coef)) / temperature
    p *= -coef[:, None]
    p.scatter_add_(1, y.long().clamp(min=0)[:, None], coef[:, None])
    return p.to(dtype)


def _plain_logprob(s, case):
    x, y, tau = s["logits"], s["target"], case["temperature"]
    if case["direction"] == "forward":
        z, top, e, total = _row_stats(x, tau)
        log_sum = torch.log(total)
        valid = y >= 0
        logp = torch.where(valid, _at_target(z, y) - top - log_sum, 0.0)
        stats = torch.where(valid[:, None], torch.stack([x.amax(1).float(), log_sum], 1), 0.0)
        return {"logp": logp, "stats": stats}
    p = torch.exp((x.float() - s["stats"][:, :1]) / tau - s["stats"][:, 1:])
    return {"dlogits": _row_gradient(p, y, s["dlogp"], tau, x.dtype)}


def _row_sequence(offsets, T):
    """The sequence of every row."""
    return torch.searchsorted(offsets[1:].contiguous(), torch.arange(T, dtype=torch.int32, device="cuda"), right=True)


def _plain_preference(s, case):
    x, y, off = s["logits"], s["target"], s["offsets"]
    z, top, e, total = _row_stats(x, 1.0)
    valid = y >= 0
    logp = torch.where(valid, _at_target(z, y) - top - torch.log(total), 0.0)
    seq = _row_sequence(off, x.shape[0])
    n = off.numel() - 1
    sums = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, seq, logp.double())
    counts = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, seq, valid.double())
    share = torch.ones_like(counts)
    if case["average"]:
        share = 1.0 / counts.clamp(min=1.0)
    sums = (sums * share).view(-1, 2)
    ratio = sums - s["ref_logp"].double()
    gap = ratio[:, 0] - ratio[:, 1]
    h, eps = BETA * gap, case["smoothing"]
    if case["kind"] == "sigmoid":
        # log(1 + exp(-h)) without overflow
        soft = torch.log1p(torch.exp(-h.abs()))
        loss = (1.0 - eps) * (soft + (-h).clamp(min=0)) + eps * (soft + h.clamp(min=0))
        slope = BETA * (1.0 / (1.0 + torch.exp(-h)) - (1.0 - eps))
    elif case["kind"] == "hinge":
        loss = (1.0 - eps) * (1.0 - h).clamp(min=0) + eps * (1.0 + h).clamp(min=0)
        slope = BETA * (eps * (h > -1.0).double() - (1.0 - eps) * (h < 1.0).double())
    else:
        up, down = gap - 0.5 / BETA, gap + 0.5 / BETA
        loss = (1.0 - eps) * up * up + eps * down * down
        slope = 2.0 * ((1.0 - eps) * up + eps * down)
    slope = slope / gap.numel()
    coef = (torch.stack([slope, -slope], 1).view(-1) * share).float()
    p = e.div_(total[:, None])
    return {"loss": loss.mean().float(), "logp": sums.float(),
            "dlogits": _row_gradient(p, y, coef[seq], 1.0, x.dtype)}


def _plain_policy(s, case):
    x, y, tau = s["logits"], s["target"], case["temperature"]
    z, top, e, total = _row_stats(x, tau)
    valid = y >= 0
    logp = torch.where(valid, _at_target(z, y) - top - torch.log(total), 0.0)
    if case["reduction"] == "tokens":
        weight = valid.float() / valid.sum().clamp(min=1).float()
    else:
        seq = _row_sequence(s["offsets"], x.shape[0])
        n = s["offsets"].numel() - 1
        counts = torch.zeros(n, device="cuda").index_add_(0, seq, valid.float())
        full = (counts > 0).sum().clamp(min=1).float()
        weight = torch.where(valid, 1.0 / (counts.clamp(min=1.0)[seq] * full), 0.0)
    gain = s["advantage"]
    ratio = torch.exp(logp - s["old_logp"])
    inside = ratio.clamp(1.0 - CLIP[0], 1.0 + CLIP[1])
    free = ratio * gain <= inside * gain
    term = -torch.where(free, ratio * gain, inside * gain)
    slope = torch.where(free, -ratio * gain, 0.0)
    kl = torch.zeros_like(term)
    if case["kl"]:
        away = s["ref_logp"] - logp
        kl = torch.exp(away) - away - 1.0
        slope = slope + case["kl"] * (1.0 - torch.exp(away))
    terms = [torch.where(valid, weight * t, 0.0).double().sum() for t in (term, kl, (~free).float())]
    p = e.div_(total[:, None])
    return {"loss": (terms[0] + case["kl"] * terms[1]).float(), "terms": torch.stack(terms).float(), "logp": logp,
            "dlogits": _row_gradient(p, y, weight * slope, tau, x.dtype)}


def _plain_balance(s, case):
    x, k = s["logits"], case["k"]
    T, E = x.shape
    z, top, e, total = _row_stats(x, 1.0)
    p = e / total[:, None]
    on = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
    choice = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :k]
    choice = torch.where(on[:, None], choice, -1).to(torch.int32)
    counts = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    where = torch.where(on[:, None], choice.long(), E).reshape(-1)
    counts = counts.index_add_(0, where, torch.ones_like(where, dtype=torch.int32))[:E].contiguous()
    n = on.sum().clamp(min=1).float()
    weight = ALPHA * E / (k * n * n) * counts.float()
    inner = p @ weight
    grad = torch.where(on[:, None], p * (weight[None, :] - inner[:, None]), 0.0)
    return {"loss": torch.where(on, inner, 0.0).double().sum().float(), "counts": counts, "choice": choice,
            "dlogits": grad.to(x.dtype)}


_PLAIN = {"logprob": _plain_logprob, "preference": _plain_preference, "policy": _plain_policy,
          "balance": _plain_balance}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Rows with a target read once, gradients of all rows written once.
    Operations: subtract, scale, exponential and add for the sum; the same
    and a product for the gradient."""
    T, size = _rows(case), 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "balance":
        E, k = case["E"], case["k"]
        on = T - len(range(5, T, 8)) if case["masked"] else T
        return {"bytes": float((on + T) * E * size + T * k * 4 + E * 4 + (T if case["masked"] else 0)),
                "flops": 9.0 * on * E}
    V = case["V"]
    if case["op"] == "logprob":
        on = T - len(range(3, T, 8)) if case["masked"] else T
        if case["direction"] == "forward":
            return {"bytes": float(on * V * size + T * 16), "flops": 4.0 * on * V}
        return {"bytes": float((on + T) * V * size + T * 16), "flops": 5.0 * on * V}
    on = T - sum(_prompts(case))
    per_row = 4 if case["op"] == "preference" else 20
    return {"bytes": float((on + T) * V * size + T * per_row + len(_lengths(case)) * 16), "flops": 9.0 * on * V}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _softmax64(x, y, coef, temperature):
    """coef (one_hot(y) - softmax(x / temperature)) / temperature, zero rows without a target."""
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    for r in range(0, x.shape[0], 512):
        p = torch.softmax(x[r:r + 512].double() / temperature, 1).neg_()
        t = y[r:r + 512].long()
        at = torch.arange(p.shape[0], device="cuda")
        p[at, t.clamp(min=0)] += 1.0
        c = torch.where(t >= 0, coef[r:r + 512].double(), 0.0) / temperature
        out[r:r + 512] = p.mul_(c[:, None])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    x = s["logits"]
    if case["op"] == "balance":
        return _exact_balance(s, case)
    y = s["target"]
    valid = y >= 0
    tau = case.get("temperature", 1.0)
    if case["op"] == "logprob" and case["direction"] == "gradient":
        return {"dlogits": _softmax64(x, y, s["dlogp"], tau)}
    logp = _logp64(x, y, tau)
    if case["op"] == "logprob":
        return {"logp": logp, "stats": _stats64(x, y, tau)}
    coef = torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
    spans = list(_spans(case))
    if case["op"] == "preference":
        score, counts = [], []
        for a, b in spans:
            m = int(valid[a:b].sum())
            counts.append(max(m, 1) if case["average"] else 1)
            score.append(float(logp[a:b].sum()) / counts[-1])
        ref = s["ref_logp"].double().cpu().reshape(-1).tolist()
        pairs, eps, total = case["pairs"], case["smoothing"], 0.0
        for i in range(pairs):
            gap = torch.tensor((score[2 * i] - ref[2 * i]) - (score[2 * i + 1] - ref[2 * i + 1]),
                               dtype=torch.float64, requires_grad=True)
            h = BETA * gap
            if case["kind"] == "sigmoid":
                f = -(1 - eps) * torch.nn.functional.logsigmoid(h) - eps * torch.nn.functional.logsigmoid(-h)
            elif case["kind"] == "hinge":
                f = (1 - eps) * torch.relu(1 - h) + eps * torch.relu(1 + h)
            else:
                f = (1 - eps) * (gap - 0.5 / BETA) ** 2 + eps * (gap + 0.5 / BETA) ** 2
            f.backward()
            total += float(f.detach()) / pairs
            for side, sign in ((2 * i, 1.0), (2 * i + 1, -1.0)):
                coef[slice(*spans[side])] = sign * float(gap.grad) / pairs / counts[side]
        return {"loss": torch.tensor(total, dtype=torch.float64),
                "logp": torch.tensor(score, dtype=torch.float64).view(-1, 2), "dlogits": _softmax64(x, y, coef, 1.0)}
    weight = torch.zeros_like(coef)
    if case["reduction"] == "tokens":
        weight[:] = 1.0 / max(1, int(valid.sum()))
    else:
        held = [int(valid[a:b].sum()) for a, b in spans]
        full = sum(m > 0 for m in held)
        for (a, b), m in zip(spans, held):
            if m:
                weight[a:b] = 1.0 / (m * full)
    weight = torch.where(valid, weight, 0.0)
    at = logp.clone().requires_grad_(True)
    ratio = torch.exp(at - s["old_logp"].double())
    gain = s["advantage"].double()
    bounded = torch.minimum(torch.maximum(ratio, torch.tensor(1.0 - CLIP[0], dtype=torch.float64, device="cuda")),
                            torch.tensor(1.0 + CLIP[1], dtype=torch.float64, device="cuda"))
    term = -torch.minimum(ratio * gain, bounded * gain)
    kl = torch.zeros_like(term)
    if case["kl"]:
        away = s["ref_logp"].double() - at
        kl = torch.exp(away) - away - 1.0
    clipped = (bounded * gain < ratio * gain).double()
    loss = (weight * (term + case["kl"] * kl)).sum()
    loss.backward()
    terms = torch.stack([(weight * t).sum() for t in (term.detach(), kl.detach(), clipped.detach())])
    return {"loss": loss.detach(), "terms": terms, "logp": logp, "dlogits": _softmax64(x, y, at.grad, tau)}


def _exact_balance(s, case):
    x, k = s["logits"].double(), case["k"]
    T, E = x.shape
    on = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
    # the k largest one after another, ties to the lowest index
    left = x.clone()
    index = torch.arange(E, device="cuda")
    choice = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    counts = torch.zeros(E, dtype=torch.int64, device="cuda")
    for j in range(k):
        top = left.max(1, keepdim=True).values
        best = torch.where(left == top, index, E).min(1).values
        choice[:, j] = torch.where(on, best, -1).to(torch.int32)
        counts += torch.bincount(best[on], minlength=E)
        left.scatter_(1, best[:, None], -math.inf)
    n = max(1, int(on.sum()))
    z = x.requires_grad_(True)
    mean = (torch.softmax(z, 1) * on[:, None]).sum(0) / n
    loss = ALPHA * E * ((counts.double() / (k * n)) * mean).sum()
    loss.backward()
    return {"loss": loss.detach(), "counts": counts.to(torch.int32), "choice": choice, "dlogits": z.grad}
