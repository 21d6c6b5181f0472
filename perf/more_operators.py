"""What a training step of a model with experts needs around its losses, as cases to be measured.

  scores   log probability of each row's token with the row's entropy and its k
           likeliest classes (direction "forward"), and the logits' gradient
           for derivatives of both (direction "gradient")
  experts  tokens to their experts and back, from a router's choice:
             "spread"       slots sorted by expert, and the tokens' rows copied in that order
             "join"         the experts' rows back at their tokens, weighted and added
             "join_grad"    the gradient of that: of the experts' rows and of the weights
             "spread_grad"  the gradient of the copy: the rows' gradients added at their tokens
  adamw    one AdamW step over many tensors, with moments in 32 bits or in 8

Every case is what such a program calls once a step.  With ``own`` false the
same results come from elementary torch operations in single precision.
"""

from __future__ import annotations

import math

import torch

own = False


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _scores(name, direction, T, V, dtype, k=0, masked=False, temperature=1.0):
    """T rows of V logits, k alternatives (forward); masked: one row in eight has no target."""
    return {"name": name, "op": "scores", "direction": direction, "T": T, "V": V, "dtype": dtype, "k": k,
            "masked": masked, "temperature": temperature}


def _experts(name, direction, T, E, k, d, dtype, masked=False):
    """T tokens of width d to k of E experts; masked: one token in eight is
    padding, and one choice in sixteen was dropped."""
    return {"name": name, "op": "experts", "direction": direction, "T": T, "E": E, "k": k, "d": d, "dtype": dtype,
            "masked": masked}


def _adamw(name, bits, layers, width, params, grads, copies=False, scaled=False):
    """A stack of layers of that width.  copies: bf16 copies of the parameters
    are written beside them; scaled: the gradients are multiplied by a factor on the device."""
    return {"name": name, "op": "adamw", "bits": bits, "layers": layers, "width": width, "params": params,
            "grads": grads, "copies": copies, "scaled": scaled}


def listed():
    return [
        # a sampled token with its twenty alternatives, as a server returns it: a call is its latency
        _scores("scores_t1_v32768_k20", "forward", 1, 32768, "bf16", k=20),
        # a batch of long answers scored over a large vocabulary: bound by reading the logits
        _scores("scores_t4096_v131072_k20", "forward", 4096, 131072, "bf16", k=20),
        # a policy over a thousand actions with an entropy bonus, a few hundred decisions
        _scores("scores_grad_t300_v1000", "gradient", 300, 1000, "bf16"),
        # the same in single precision over an odd vocabulary, whose rows start at every 4-byte offset
        _scores("scores_grad_t2000_v50001_f32", "gradient", 2000, 50001, "f32", masked=True, temperature=0.7),
        # eight tokens of a decoding step to their experts: launches
        _experts("spread_t8_e64_k8_d2048", "spread", 8, 64, 8, 2048, "bf16"),
        # a batch of prompts: bound by writing the copies
        _experts("spread_t16384_e128_k8_d2048", "spread", 16384, 128, 8, 2048, "bf16"),
        # the way back for a padded batch, wider rows
        _experts("join_t8192_e64_k4_d5120", "join", 8192, 64, 4, 5120, "bf16", masked=True),
        # its gradient in single precision, rows of an odd width
        _experts("join_grad_t10000_e256_k6_d1001_f32", "join_grad", 10000, 256, 6, 1001, "f32", masked=True),
        # a small network: nineteen tensors, of which most are a few lines of memory
        _adamw("adamw_l2_w64", 32, 2, 64, "f32", "f32"),
        # four hundred million parameters in single precision
        _adamw("adamw_l8_w2048", 32, 8, 2048, "f32", "f32", scaled=True),
        # parameters and gradients in half precision, moments in 8 bits; an odd width
        _adamw("adamw8_l6_w1001_bf16", 8, 6, 1001, "bf16", "bf16"),
        # single-precision parameters with half-precision copies for the model, moments in 8 bits
        _adamw("adamw8_l8_w2048_copies", 8, 8, 2048, "f32", "bf16", copies=True, scaled=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_LOGITS = 4096 * 131072             # bf16 logits of a drawn case at most (fp32: half of them)
MOST_SLOTS = 16384 * 8 * 2048           # elements of the experts' rows at most (the same)


def draw(rng):
    op = rng.choice(["scores", "experts", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    share = 1 if dtype == "bf16" else 2
    if op == "scores":
        V = rng.choice([1000, 32768, 131072, _log_uniform(rng, 100, 200000), _log_uniform(rng, 20000, 200000)])
        T = _log_uniform(rng, 1, max(1, min(16384, MOST_LOGITS // share // V)))
        direction = rng.choice(["forward", "gradient"])
        # a gradient also writes what it reads
        T = T if direction == "forward" else (T + 1) // 2
        case = _scores("", direction, T, V, dtype, rng.choice([0, 1, 5, 20, rng.randint(2, 32)]) if direction == "forward" else 0,
                       rng.random() < 0.5, rng.choice([1.0, 1.0, 0.6, 1.3]))
    elif op == "experts":
        E = rng.choice([8, 64, 128, 256, rng.randint(4, 512)])
        k = rng.randint(1, min(8, E))
        d = rng.choice([1024, 2048, 4096, 7168, _log_uniform(rng, 16, 8192)])
        T = _log_uniform(rng, 1, max(1, min(65536, MOST_SLOTS // share // (k * d))))
        direction = rng.choice(["spread", "join", "join_grad", "spread_grad"])
        T = T if direction != "join_grad" else (T + 1) // 2
        case = _experts("", direction, T, E, k, d, dtype, rng.random() < 0.5)
    else:
        width = _log_uniform(rng, 16, 2048)
        layers = _log_uniform(rng, 1, max(1, min(64, 8 * 2048 * 2048 // (width * width))))
        bits = rng.choice([32, 8])
        params = rng.choice(["f32", "bf16"])
        case = _adamw("", bits, layers, width, params, rng.choice(["f32", "bf16"]), params == "f32" and rng.random() < 0.5,
                      rng.random() < 0.5)
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

LR, BETAS, EPS, DECAY, SEED = 3e-4, (0.9, 0.95), 1e-8, 0.1, 20240607
BLOCK = 256                             # elements with a common scale, of moments in 8 bits
BEFORE = 100                            # steps that were made before the measured one


def _generator(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + k) % (1 << 62))
    return g


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _normal(shape, dtype, g, scale=1.0):
    """Normal values, made in parts: no single-precision copy of the whole."""
    x = torch.empty(shape, dtype=dtype, device="cuda")
    flat = x.view(-1)
    for r in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - r)
        flat[r:r + n] = torch.randn((n,), generator=g, device="cuda") * scale
    return x


def _slots(case):
    """Slots that hold an expert."""
    T, k = case["T"], case["k"]
    if not case["masked"]:
        return T * k
    return sum(1 for t in range(T) if t % 8 != 5) * k - sum(
        1 for s in range(9, T * k, 16) if (s // k) % 8 != 5)


def _shapes(case):
    """The tensors of the stack: matrices, and vectors a few lines long."""
    w = case["width"]
    layer = [(w, w)] * 4 + [(4 * w, w), (w, 4 * w)] + [(w,)] * 2 + [(4 * w,)]
    return layer * case["layers"] + [(w,)]


def _sizes(case):
    return [math.prod(s) for s in _shapes(case)]


def prepare(case, seed):
    return {"scores": _prepare_scores, "experts": _prepare_experts, "adamw": _prepare_adamw}[case["op"]](case, seed)


def _prepare_scores(case, seed):
    """Logits as a model gives them: a spread of a few units, the token's usually among the largest."""
    T, V = case["T"], case["V"]
    x = _normal((T, V), _type(case["dtype"]), _generator(seed, 1), 2.0)
    g = _generator(seed, 2)
    y = torch.randint(V, (T,), generator=g, device="cuda")
    at = torch.arange(T, device="cuda")
    x[at, y] = (x[at, y].float() + 12.0 * torch.rand((T,), generator=g, device="cuda")).to(x.dtype)
    y = y.to(torch.int32)
    if case["masked"]:
        y[3::8] = -1
    state = {"case": case, "logits": x, "target": y}
    if case["direction"] == "gradient":
        state["dlogp"] = torch.randn((T,), generator=g, device="cuda") / T
        state["dentropy"] = torch.randn((T,), generator=g, device="cuda") * 0.5 / T
        # what the forward call returned
        s = _scores64(x, y, 0, case["temperature"])
        state["stats"], state["entropy"] = s["stats"].float(), s["entropy"].float()
    return state


def _prepare_experts(case, seed):
    T, E, k, d = case["T"], case["E"], case["k"], case["d"]
    dtype, direction = _type(case["dtype"]), case["direction"]
    g = _generator(seed, 1)
    # routers favour some experts; every token's are different ones
    likes = torch.randn((E,), generator=g, device="cuda") + torch.randn((T, E), generator=g, device="cuda")
    choice = torch.topk(likes, k, dim=1).indices.to(torch.int32)
    if case["masked"]:
        choice[5::8] = -1
        choice.view(-1)[9::16] = -1
    state = {"case": case, "choice": choice}
    if direction == "spread":
        state["x"] = _normal((T, d), dtype, g)
    else:
        routes = _sorted_slots(choice, E)
        state["place"], state["slot"], state["offsets"] = routes["place"], routes["slot"], routes["offsets"]
        state["rows"] = _normal((T * k, d), dtype, g)
        weight = torch.rand((T, k), generator=g, device="cuda") + 0.1
        state["weight"] = weight / weight.sum(1, keepdim=True)
        if direction == "join_grad":
            state["dy"] = _normal((T, d), dtype, g)
    # rows behind the last expert's are left as they were: zeros
    state["buffer"] = torch.zeros((T * k, d), dtype=dtype, device="cuda") \
        if case["masked"] and direction in ("spread", "join_grad") else None
    if own:
        from paper_2607_20739_gb300 import experts
        state["routes"] = None if direction == "spread" else \
            experts.Routes(T, k, E, state["place"], state["slot"], state["offsets"])
    return state


def _prepare_adamw(case, seed):
    """Every tensor is a view of one buffer and starts on a multiple of a
    block; what lies between them is zero and stays it."""
    sizes = _sizes(case)
    padded = [-(-n // BLOCK) * BLOCK for n in sizes]
    starts = [0]
    for n in padded:
        starts.append(starts[-1] + n)
    N, g = starts[-1], _generator(seed, 1)
    gaps = torch.zeros(N, dtype=torch.bool, device="cuda")
    for a, n, b in zip(starts, sizes, starts[1:]):
        gaps[a + n:b] = True
    # gradients differ in size from one part of a matrix to another
    spread = torch.exp(torch.randn((N // BLOCK, 8), generator=g, device="cuda")) * 1e-3
    spread = spread.repeat_interleave(BLOCK // 8, 1).view(-1)
    p = _normal((N,), torch.float32, g, 0.02).masked_fill_(gaps, 0.0).to(_type(case["params"]))
    grad = (_normal((N,), torch.float32, g) * spread).masked_fill_(gaps, 0.0).to(_type(case["grads"]))
    m = (_normal((N,), torch.float32, g) * spread * 0.2).masked_fill_(gaps, 0.0)
    v = ((_normal((N,), torch.float32, g, 0.3) + 1.0).square_() * spread.square()).masked_fill_(gaps, 0.0)
    state = {"case": case, "t": BEFORE, "p": p, "grad": grad, "starts": starts, "sizes": sizes,
             "copy": p.to(torch.bfloat16) if case["copies"] else None,
             "scale": 0.25 + 0.5 * torch.rand((), generator=g, device="cuda") if case["scaled"] else None}
    if case["bits"] == 8:
        middle = torch.full((N,), 1 << 15, dtype=torch.int64, device="cuda")     # to nearest
        m, state["m_scale"] = _encode_m(m, middle)
        v, state["v_scale"] = _encode_v(v, middle)
    state["m"], state["v"] = m, v
    del gaps, spread
    if own:
        from paper_2607_20739_gb300 import optim
        views = lambda t, per=1: None if t is None else [  # noqa: E731
            t[a // per:a // per + -(-n // per)].view(s if per == 1 else (-1,)) for a, n, s in zip(starts, sizes, _shapes(case))]
        kept = {"t": BEFORE, "m": views(m), "v": views(v)}
        if case["bits"] == 8:
            kept["m_scale"], kept["v_scale"] = views(state["m_scale"], BLOCK), views(state["v_scale"], BLOCK)
        state["grads"] = views(grad)
        state["optimizer"] = optim.AdamW(views(p), lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, bits=case["bits"],
                                         copies=views(state["copy"]), seed=SEED, state=kept)
    return state


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    case = state["case"]
    return (_OWN if own else _PLAIN)[case["op"]](state, case)


def _own_scores(s, case):
    from paper_2607_20739_gb300 import losses
    if case["direction"] == "forward":
        r = losses.token_scores(s["logits"], s["target"], case["k"], temperature=case["temperature"])
        return {"logp": r["logp"], "entropy": r["entropy"], "stats": r["stats"], "top": r["top"], "top_logp": r["top_logp"]}
    return {"dlogits": losses.token_scores_grad(s["logits"], s["target"], s["stats"], s["entropy"], s["dlogp"], s["dentropy"],
                                                temperature=case["temperature"])}


def _own_experts(s, case):
    from paper_2607_20739_gb300 import experts
    direction = case["direction"]
    if direction == "spread":
        r = experts.route(s["choice"], case["E"])
        rows = experts.spread(s["x"], r, out=s["buffer"])
        return {"place": r.place, "slot": r.slot, "offsets": r.offsets, "rows": rows}
    if direction == "join":
        return {"y": experts.join(s["rows"], s["routes"], s["weight"])}
    if direction == "spread_grad":
        return {"dx": experts.spread_grad(s["rows"], s["routes"])}
    drows, dweight = experts.join_grad(s["dy"], s["rows"], s["routes"], s["weight"], out=s["buffer"])
    return {"drows": drows, "dweight": dweight}


def _own_adamw(s, case):
    s["optimizer"].step(s["grads"], grad_scale=s["scale"])
    return _updated(s, case)


_OWN = {"scores": _own_scores, "experts": _own_experts, "adamw": _own_adamw}


def _plain_scores(s, case):
    x, y, tau, k = s["logits"], s["target"], case["temperature"], case["k"]
    valid = y >= 0
    at = y.long().clamp(min=0)[:, None]
    if case["direction"] == "gradient":
        q = (x.float() - s["stats"][:, :1]) / tau - s["stats"][:, 1:]
        a, b = s["dlogp"] / tau, s["dentropy"] / tau
        g = -torch.exp(q) * (a[:, None] + b[:, None] * (q + s["entropy"][:, None]))
        g.scatter_add_(1, at, a[:, None])
        return {"dlogits": torch.where(valid[:, None], g, 0.0).to(x.dtype)}
    f = x.float()
    top = torch.amax(f, 1)
    z = (f - top[:, None]) / tau
    e = torch.exp(z)
    total = e.sum(1)
    log_sum = torch.log(total)
    entropy = log_sum - (e * z).sum(1) / total
    logp = z.gather(1, at)[:, 0] - log_sum
    # the k largest, of equal ones the lower class first: as whole numbers, no two of a row are equal
    bits = (f + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7fffffff)).to(torch.int64) << 32
    key += torch.arange(x.shape[1] - 1, -1, -1, device="cuda")
    best = x.shape[1] - 1 - (torch.topk(key, k, dim=1).values & 0xffffffff) if k else at[:, :0]
    on = valid[:, None]
    return {"logp": torch.where(valid, logp, 0.0), "entropy": torch.where(valid, entropy, 0.0),
            "stats": torch.where(on, torch.stack([top, log_sum], 1), 0.0),
            "top": torch.where(on, best, -1).to(torch.int32),
            "top_logp": torch.where(on, z.gather(1, best) - log_sum[:, None], -math.inf)}


def _sorted_slots(choice, E):
    """Slots (token times k plus place in its choice) sorted by expert, in
    their order within one: slot of each row (-1 behind the last), row of each slot, first row of each expert."""
    flat = choice.reshape(-1).long()
    flat = torch.where(flat >= 0, flat, E)
    experts, order = torch.sort(flat, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, flat, torch.ones_like(flat))
    offsets = torch.cumsum(counts, 0) - counts
    row = torch.empty_like(flat)
    row[order] = torch.where(experts < E, torch.arange(flat.numel(), device="cuda"), -1)
    return {"place": row.view(choice.shape).to(torch.int32), "slot": torch.where(experts < E, order, -1).to(torch.int32),
            "offsets": offsets.to(torch.int32)}


def _plain_experts(s, case):
    direction, T, k = case["direction"], case["T"], case["k"]
    if direction == "spread":
        r = _sorted_slots(s["choice"], case["E"])
        token = r["slot"].long().clamp(min=0) // k
        rows = s["x"][token]
        if s["buffer"] is not None:
            rows = torch.where((r["slot"] >= 0)[:, None], rows, s["buffer"])
        return {**r, "rows": rows}
    on, at = s["place"] >= 0, s["place"].long().clamp(min=0)
    got = torch.where(on[:, :, None], s["rows"][at].float(), 0.0)
    if direction == "spread_grad":
        return {"dx": got.sum(1).to(s["rows"].dtype)}
    if direction == "join":
        return {"y": (got * s["weight"][:, :, None]).sum(1).to(s["rows"].dtype)}
    dy = s["dy"].float()[:, None, :]
    part = (dy * s["weight"][:, :, None]).to(s["rows"].dtype)
    drows = torch.empty_like(s["rows"]) if s["buffer"] is None else s["buffer"].clone()
    drows[s["place"][on].long()] = part[on]
    return {"drows": drows, "dweight": (got * dy).sum(2)}


# Moments in 8 bits.  A block of 256 elements has a scale, a power of two.  A first
# moment is an 8-bit float (4 bits of exponent, 3 of fraction) times it, the largest one between 2^7 and 2^8.
# A second moment has no sign: 16 steps an octave from 2^5 down to 2^-3
# (codes 255 to 127), 8 below (codes to 1, 2^-19 x 1.25), and 0, which stands for zero alone.
# Between two codes chance decides: r of 2^16 lets a share r / 2^16 of them go up.

def _mix(h):
    """32 bits scattered: 32-bit products by odd numbers, and shifts."""
    h = h & 0xffffffff
    h = ((h ^ (h >> 16)) * 0x6A09E667) & 0xffffffff
    h = ((h ^ (h >> 15)) * 0xBB67AE85) & 0xffffffff
    return h ^ (h >> 16)


def _as_float(bits):
    return bits.to(torch.int32).view(torch.float32)


def _scaled(x, shift):
    """Blocks of magnitudes over their scale, and the scale: the largest one's power of two less `shift`."""
    x = x.view(-1, BLOCK)
    top = (x.amax(1).view(torch.int32) >> 23).to(torch.int64)       # its exponent
    held = top >= 16
    scale = torch.where(held, _as_float(torch.where(held, top - shift, 0) << 23), 0.0)
    over = torch.where(held, _as_float(torch.where(held, 254 + shift - top, 0) << 23), 0.0)
    return (x * over[:, None]).view(-1), scale


def _encode_m(m, chance):
    y, scale = _scaled(m.abs(), 7)
    bits = y.view(torch.int32).to(torch.int64) - (120 << 23)
    bits = torch.where(y >= 2.0 ** -6, bits, (y * 2.0 ** 29).to(torch.int64))
    code = (bits + (chance << 4) + 8) >> 20
    code += (m < 0).to(torch.int64) << 7
    return code.to(torch.uint8).view(torch.float8_e4m3fn), scale


def _encode_v(v, chance):
    y, scale = _scaled(v, 4)
    bits = y.view(torch.int32).to(torch.int64)
    high = ((bits + (chance << 3) + 4) >> 19) - 1857
    low = (((bits + (chance << 4) + 8) >> 20) - 865).clamp(min=1)
    code = torch.where(y >= 2.0 ** -3, high, torch.where(y > 0, low, 0))
    return code.to(torch.uint8), scale


def _decode_m(code, scale):
    return (code.float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _decode_v(code, scale):
    c = code.to(torch.int64)
    bits = torch.where(c >= 127, (c + 1857) << 19, (c + 865) << 20)
    value = torch.where(c > 0, _as_float(bits), 0.0)
    return (value.view(-1, BLOCK) * scale[:, None]).view(-1)


def _chances(s, case, t):
    """32 random bits for every element, by seed, step, tensor and index."""
    starts = torch.tensor(s["starts"], dtype=torch.int64, device="cuda")
    key = _mix(_mix(_mix(torch.tensor(SEED, dtype=torch.int64)) + t) + torch.arange(len(s["sizes"]))).cuda()
    key = _mix(key)                     # the upper 32 bits of an index are 0
    length = starts[1:] - starts[:-1]
    index = torch.arange(s["p"].numel(), device="cuda") - starts[:-1].repeat_interleave(length)
    return _mix(index ^ key.repeat_interleave(length))


def _updated(s, case):
    """The state's own buffers.  The codes of second moments are whole numbers,
    the same to the bit however they are computed: products, sums and shifts in one order."""
    out = {"p": s["p"], "m": s["m"], "v": s["v"]}
    if case["copies"]:
        out["copy"] = s["copy"]
    if case["bits"] == 8:
        out |= {"m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    return out


def _plain_adamw(s, case):
    s["t"] += 1
    t = s["t"]
    g = s["grad"].float()
    if s["scale"] is not None:
        g = g * s["scale"]
    small = case["bits"] == 8
    m = _decode_m(s["m"], s["m_scale"]) if small else s["m"]
    v = _decode_v(s["v"], s["v_scale"]) if small else s["v"]
    m = m * BETAS[0] + g * (1.0 - BETAS[0])
    v = v * BETAS[1] + g * g * (1.0 - BETAS[1])
    step = m / (1.0 - BETAS[0] ** t) / (torch.sqrt(v / (1.0 - BETAS[1] ** t)) + EPS)
    p = s["p"].float() * (1.0 - LR * DECAY) - LR * step
    s["p"].copy_(p)
    if case["copies"]:
        s["copy"].copy_(p)
    if small:
        r = _chances(s, case, t)
        for name, (code, scale) in (("m", _encode_m(m, r & 0xffff)), ("v", _encode_v(v, r >> 16))):
            s[name].copy_(code)
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _updated(s, case)


_PLAIN = {"scores": _plain_scores, "experts": _plain_experts, "adamw": _plain_adamw}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Every input read once and every output written once.  Operations: six
    a logit for the sums and the comparison, eight for the gradient; a product and a sum for each
    element that is weighted; fifteen for an updated parameter."""
    if case["op"] == "scores":
        T, V, size = case["T"], case["V"], 2 if case["dtype"] == "bf16" else 4
        on = T - len(range(3, T, 8)) if case["masked"] else T
        if case["direction"] == "forward":
            return {"bytes": float(on * V * size + T * (20 + 8 * case["k"])), "flops": 6.0 * on * V}
        return {"bytes": float((on + T) * V * size + T * 24), "flops": 8.0 * on * V}
    if case["op"] == "experts":
        T, k, d, size = case["T"], case["k"], case["d"], 2 if case["dtype"] == "bf16" else 4
        rows, direction = _slots(case), case["direction"]
        if direction == "spread":
            return {"bytes": float((T + rows) * d * size + T * k * 12 + case["E"] * 4), "flops": 0.0}
        if direction == "join_grad":
            return {"bytes": float((T + 2 * rows) * d * size + T * k * 12), "flops": 3.0 * rows * d}
        return {"bytes": float((T + rows) * d * size + T * k * (8 if direction == "join" else 4)), "flops": 2.0 * rows * d}
    n = sum(_sizes(case))
    p, g = (2 if case[x] == "bf16" else 4 for x in ("params", "grads"))
    each = 2 * p + g + (2 if case["copies"] else 0) + (16 if case["bits"] == 32 else 4 + 16.0 / BLOCK)
    return {"bytes": float(n * each), "flops": 15.0 * n}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _scores64(x, y, k, tau):
    T, V = x.shape
    out = {"logp": torch.zeros(T, dtype=torch.float64, device="cuda"), "entropy": torch.zeros(T, dtype=torch.float64, device="cuda"),
           "stats": torch.zeros((T, 2), dtype=torch.float64, device="cuda"),
           "top": torch.full((T, k), -1, dtype=torch.int32, device="cuda"),
           "top_logp": torch.full((T, k), -math.inf, dtype=torch.float64, device="cuda")}
    step = max(1, (1 << 26) // V)
    for r in range(0, T, step):
        f = x[r:r + step].double()
        t = y[r:r + step].long()
        on = torch.nonzero(t >= 0)[:, 0]
        f, t = f[on], t[on]
        if not f.shape[0]:
            continue
        q = torch.log_softmax(f / tau, 1)
        m = f.max(1).values
        out["logp"][r + on] = q.gather(1, t[:, None])[:, 0]
        out["entropy"][r + on] = -(q.exp() * q).sum(1)
        out["stats"][r + on] = torch.stack([m, torch.logsumexp((f - m[:, None]) / tau, 1)], 1)
        # one after another, ties to the lowest class
        for j in range(k):
            top = f.max(1, keepdim=True).values
            best = torch.where(f == top, torch.arange(V, device="cuda"), V).min(1).values
            out["top"][r + on, j] = best.to(torch.int32)
            out["top_logp"][r + on, j] = q.gather(1, best[:, None])[:, 0]
            f.scatter_(1, best[:, None], -math.inf)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"scores": _exact_scores, "experts": _exact_experts, "adamw": _exact_adamw}[case["op"]](s, case)


def _exact_scores(s, case):
    x, y, tau = s["logits"], s["target"], case["temperature"]
    if case["direction"] == "forward":
        return _scores64(x, y, case["k"], tau)
    T, V = x.shape
    out = torch.zeros((T, V), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // V)
    for r in range(0, T, step):
        t = y[r:r + step].long()
        on = torch.nonzero(t >= 0)[:, 0]
        f = x[r:r + step][on].double().requires_grad_(True)
        q = torch.log_softmax(f / tau, 1)
        logp = q.gather(1, t[on][:, None])[:, 0]
        entropy = -(q.exp() * q).sum(1)
        (logp * s["dlogp"][r + on].double() + entropy * s["dentropy"][r + on].double()).sum().backward()
        out[r + on] = f.grad
    return {"dlogits": out}


def _exact_experts(s, case):
    T, k, d, direction = case["T"], case["k"], case["d"], case["direction"]
    if direction == "spread":
        # whole numbers on the host: a bucket for each expert, filled in order
        buckets = [[] for _ in range(case["E"])]
        for slot, e in enumerate(s["choice"].reshape(-1).tolist()):
            if e >= 0:
                buckets[e].append(slot)
        slots, offsets = [], [0]
        for b in buckets:
            slots += b
            offsets.append(len(slots))
        order = torch.tensor(slots, dtype=torch.int64, device="cuda")
        place = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
        place[order] = torch.arange(len(slots), dtype=torch.int32, device="cuda")
        rows = torch.zeros((T * k, d), dtype=torch.float64, device="cuda")
        rows[:len(slots)] = s["x"].double()[order // k]
        slot = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
        slot[:len(slots)] = order.to(torch.int32)
        return {"place": place.view(T, k), "slot": slot,
                "offsets": torch.tensor(offsets, dtype=torch.int32, device="cuda"), "rows": rows}
    y = torch.zeros((T, d), dtype=torch.float64, device="cuda")
    drows = torch.zeros((T * k, d), dtype=torch.float64, device="cuda") if direction == "join_grad" else None
    dweight = torch.zeros((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        on = torch.nonzero(s["place"][:, j] >= 0)[:, 0]
        at = s["place"][on, j].long()
        w = s["weight"][on, j].double()[:, None] if direction != "spread_grad" else 1.0
        if direction == "join_grad":
            dy = s["dy"][on].double()
            drows[at] = w * dy
            dweight[on, j] = (s["rows"][at].double() * dy).sum(1)
        else:
            y[on] += w * s["rows"][at].double()
    if direction == "join_grad":
        return {"drows": drows, "dweight": dweight}
    return {"y" if direction == "join" else "dx": y}


def _exact_adamw(s, case):
    """Parameters and 32-bit moments.  Moments in 8 bits are rounded by chance:
    the same results to the bit are asked of them."""
    parts = []
    N, t = s["p"].numel(), BEFORE + 1
    small = case["bits"] == 8
    step = 1 << 26
    for a in range(0, N, step):
        b = min(N, a + step)
        blocks = slice(a // BLOCK, -(-b // BLOCK))
        g = s["grad"][a:b].double() * (1.0 if s["scale"] is None else s["scale"].double())
        if small:
            m = s["m"][a:b].to(torch.float64) * s["m_scale"][blocks].double().repeat_interleave(BLOCK)
            c = s["v"][a:b].to(torch.float64)
            # code c is 16 steps an octave above code 127 = 2^-3, 8 below
            high, low = torch.floor((c - 127) / 16), torch.floor((c - 127) / 8)
            v = torch.where(c >= 127, (1 + (c - 127 - 16 * high) / 16) * torch.exp2(high - 3),
                            (1 + (c - 127 - 8 * low) / 8) * torch.exp2(low - 3))
            v = torch.where(c > 0, v, 0.0) * s["v_scale"][blocks].double().repeat_interleave(BLOCK)
        else:
            m, v = s["m"][a:b].double(), s["v"][a:b].double()
        m = m + (1.0 - BETAS[0]) * (g - m)
        v = v + (1.0 - BETAS[1]) * (g * g - v)
        p = s["p"][a:b].double()
        p = p - LR * (DECAY * p + (m / (1.0 - BETAS[0] ** t)) / ((v / (1.0 - BETAS[1] ** t)).sqrt() + EPS))
        parts.append((p, None, None) if small else (p, m, v))
    p = torch.cat([q[0] for q in parts])
    out = {"p": p, "m": None if small else torch.cat([q[1] for q in parts]),
           "v": None if small else torch.cat([q[2] for q in parts])}
    if case["copies"]:
        out["copy"] = p
    if small:
        out |= {"m_scale": None, "v_scale": None}
    return out
