"""Token scores, the way of tokens to their experts and back, and AdamW in 64
bits, written from their definitions (include/pgc.h): numpy only.  The 8-bit
moments are computed in single precision, one rounding after another, as their
definition asks for.
"""

from __future__ import annotations

import numpy as np


# ---- token scores ----------------------------------------------------------------

def log_probabilities(x, tau=1.0):
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        z = (x - x.max(1, keepdims=True)) / tau
        return z - np.log(np.exp(z).sum(1, keepdims=True))


def entropy(q):
    with np.errstate(all="ignore"):
        p = np.exp(q)
        return -np.where(p > 0, p * q, np.where(np.isnan(q), np.nan, 0.0)).sum(1)


def top(x, k):
    """Classes of the k largest logits above -inf, largest first, ties to the lower class; -1 behind them."""
    x = np.asarray(x, np.float64)
    out = np.full((x.shape[0], k), -1, np.int32)
    for t in range(x.shape[0]):
        order = np.argsort(-x[t], kind="stable")[:k]
        order = order[x[t, order] > -np.inf]
        out[t, :len(order)] = order
    return out


def scores_gradient(x, y, a, b, tau=1.0):
    """Gradient of sum_t a_t q_t,y_t + b_t H_t; zeros in rows of negative target or without derivatives."""
    q = log_probabilities(x, tau)
    h = entropy(q)
    g = np.zeros_like(q)
    for t in range(len(q)):
        if (y is not None and y[t] < 0) or (a[t] == 0 and b[t] == 0):
            continue
        with np.errstate(all="ignore"):
            p = np.exp(q[t])
            g[t] = -p * a[t] - b[t] * np.where(p > 0, p * (q[t] + h[t]), 0.0)
        if a[t] != 0:
            g[t, y[t]] += a[t]
        g[t] /= tau
    return g


# ---- experts ---------------------------------------------------------------------

def route(choice, experts):
    """(place, slot, offsets)"""
    choice = np.asarray(choice)
    flat = choice.reshape(-1)
    place, slot = np.full(flat.shape, -1, np.int32), np.full(flat.shape, -1, np.int32)
    offsets, at = [0], 0
    on = np.flatnonzero((flat >= 0) & (flat < experts))
    order = on[np.argsort(flat[on], kind="stable")]
    counts = np.bincount(flat[on], minlength=experts)
    for e in range(experts):
        at += int(counts[e])
        offsets.append(at)
    place[order] = np.arange(len(order))
    slot[:len(order)] = order
    return place.reshape(choice.shape), slot, np.array(offsets, np.int32)


def join(rows, place, weight=None):
    """(y, sum of the terms' magnitudes)"""
    T, k = place.shape
    y, size = np.zeros((T, rows.shape[1])), np.zeros((T, rows.shape[1]))
    for t in range(T):
        for j in range(k):
            if 0 <= place[t, j] < len(rows):
                term = rows[place[t, j]] * (1.0 if weight is None else float(weight[t, j]))
                y[t] += term
                size[t] += np.abs(term)
    return y, size


def join_grad(dy, rows, place, weight):
    """({row: gradient}, dweight, sum of its terms' magnitudes)"""
    T, k = place.shape
    drows, dweight, size = {}, np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            r = int(place[t, j])
            if 0 <= r < len(rows):
                drows[r] = float(weight[t, j]) * dy[t]
                dweight[t, j] = (dy[t] * rows[r]).sum()
                size[t, j] = np.abs(dy[t] * rows[r]).sum()
    return drows, dweight, size


# ---- AdamW -----------------------------------------------------------------------

BLOCK = 256


def adamw(p, g, m, v, t, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, decay=0.01):
    """(p', m', v') in 64 bits"""
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    with np.errstate(all="ignore"):
        step = (m / (1 - betas[0] ** t)) / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
    return p * (1 - lr * decay) - lr * step, m, v


def mix(h):
    h = np.asarray(h, np.uint64) & np.uint64(0xffffffff)
    for shift, odd in ((16, 0x6A09E667), (15, 0xBB67AE85)):
        h = (h ^ (h >> np.uint64(shift))) * np.uint64(odd) & np.uint64(0xffffffff)
    return h ^ (h >> np.uint64(16))


def chances(seed, t, tensor, index):
    """32 random bits for elements `index` of a tensor at step t."""
    index = np.asarray(index, np.uint64)
    key = mix(mix(mix(np.uint64(seed)) + np.uint64(t)) + np.uint64(tensor))
    return mix((index & np.uint64(0xffffffff)) ^ mix(key + (index >> np.uint64(32))))


def decode_m(code):
    """Values of the codes, before their scale."""
    c = np.asarray(code, np.int64)
    e, f = (c & 0x7f) >> 3, (c & 7) / 8.0
    value = np.where(e > 0, (1 + f) * 2.0 ** (e - 7), f * 2.0 ** -6)
    return np.where(c & 0x80, -value, value)


def decode_v(code):
    c = np.asarray(code, np.int64)
    def steps(per):
        e = np.floor_divide(c - 127, per)
        return (1 + (c - 127 - e * per) / per) * 2.0 ** (e - 3)
    return np.where(c == 0, 0.0, np.where(c >= 127, steps(16), steps(8)))


def block_scales(x, shift):
    """Scale of every block: 2^(e - shift), e the exponent of its largest magnitude."""
    x = np.abs(np.asarray(x, np.float32))
    out = np.zeros(-(-len(x) // BLOCK), np.float32)
    for i in range(len(out)):
        top = x[i * BLOCK:(i + 1) * BLOCK].max()
        if not np.isfinite(x[i * BLOCK:(i + 1) * BLOCK]).all():
            out[i] = np.nan
        elif top >= 2.0 ** -111:
            out[i] = np.float32(2.0 ** (np.frexp(top)[1] - 1 - shift))
    return out


def encode(x, scale, codes, chance, step_bits=16):
    """The code of |x| / scale among increasing values `codes`: the upper neighbour if chance, of
    2^16, is among the share of its place between the two."""
    y = np.abs(np.asarray(x, np.float64)) / scale
    low = np.clip(np.searchsorted(codes, y, side="right") - 1, 0, len(codes) - 2)
    share = (y - codes[low]) / (codes[low + 1] - codes[low])
    up = share + (np.asarray(chance, np.float64) + 0.5) / 2.0 ** step_bits >= 1.0
    return low + up


def adamw8(p, g, m, v, ms, vs, t, tensor, seed, betas, grad_scale=None, index=0, **kw):
    """One tensor's step: (p' in 64 bits, m codes, v codes, scales).  g in the gradients' type as float32."""
    f = np.float32
    n = len(p)
    at = np.arange(n) // BLOCK
    with np.errstate(all="ignore"):
        g = np.asarray(g, f) * (f(1) if grad_scale is None else f(grad_scale))
        mv = (decode_m(m).astype(f) * ms[at]).astype(f)
        vv = (decode_v(v).astype(f) * vs[at]).astype(f)
        m1 = mv * f(betas[0]) + g * f(1 - betas[0])
        v1 = vv * f(betas[1]) + (g * g) * f(1 - betas[1])
        q = adamw(np.asarray(p, np.float64), g.astype(np.float64), mv.astype(np.float64), vv.astype(np.float64), t, betas=betas, **kw)[0]
        ms1, vs1 = block_scales(m1, 7), block_scales(v1, 4)
        h = chances(seed, t, tensor, index + np.arange(n, dtype=np.uint64))
        mcodes, vcodes = decode_m(np.arange(0x79)), decode_v(np.arange(256))
        live_m, live_v = ms1[at] > 0, vs1[at] > 0
        mc = np.where(live_m, encode(m1, np.where(live_m, ms1[at], 1), mcodes, h & np.uint64(0xffff)) + 0x80 * (m1 < 0), 0)
        vc = encode(v1, np.where(live_v, vs1[at], 1), vcodes, h >> np.uint64(16))
        vc = np.where(live_v & (v1 > 0), np.maximum(vc, 1), 0)
    return q, mc.astype(np.uint8), vc.astype(np.uint8), ms1, vs1
