"""Plain 64-bit forms of the full-rank operators, written from their definitions (numpy, no code of the library)."""
import math

import numpy as np

EPS32 = 2.0 ** -24          # half a step of fp32, relative
EPS16 = 2.0 ** -8           # of bf16
BLOCK = 128


def adamw(w, u, v, g, t, lr, beta1, beta2, eps, wd, bias_correction=True):
    """(w, u, v, size of the update's terms): the last bounds what rounding can do to the update."""
    u_terms = beta1 * np.abs(u) + (1 - beta1) * np.abs(g)
    u = beta1 * u + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    c1, c2 = (1 - beta1 ** t, 1 - beta2 ** t) if bias_correction else (1.0, 1.0)
    den = np.sqrt(v / c2) + eps
    with np.errstate(all="ignore"):
        n = np.where(den == 0, 0.0, u / c1 / den)
        size = np.where(den == 0, 0.0, u_terms / c1 / den)
    return w - lr * (n + wd * w), u, v, size


def adamw_bounds(w_new, w_old, u_terms, v_new, size, lr, wd, w_bf16):
    """Largest errors of the fp32 step, in halves of a step.  u: five roundings (beta, 1 - beta, s g, their product, the sum) act on its terms; v: seven (s g
    counts twice), on a sum of positive terms.  The update lr sqrt(c2) / c1 u / (sqrt(v) + eps sqrt(c2)): 5 of u, 3.5 of v and 2 of its root (one unit), 1 of
    the sum, 2 of the reciprocal (one unit), 1 of the product, 3 of lr sqrt(c2) / c1: 17.5.  W - lr wd W: 1 of lr wd, and 1 of the result, which is at
    most the new weight and the update; 1 of the new weight: 20 of the update cover it.  A weight in bf16 is rounded once more; 2^-126 where results are
    subnormal."""
    tiny = 2.0 ** -126
    bw = EPS32 * (2 * np.abs(w_new) + lr * (20 * size + 4 * wd * np.abs(w_old))) + tiny
    if w_bf16:
        bw = bw * (1 + EPS16) + EPS16 * np.abs(w_new)
    return bw, 5 * EPS32 * u_terms + tiny, 7 * EPS32 * v_new + tiny


def thresholds(t, n):
    """theta 2^17 of n elements at step t, of the first and of the second moment."""
    def low(x):
        return x & np.uint64(0xFFFFFFFF)
    x = low(np.uint64(t) * np.uint64(0x9E3779B1) + low(np.arange(n, dtype=np.uint64) * np.uint64(0xBB67AE85)))
    x = low((x ^ x >> np.uint64(15)) * np.uint64(0x6A09E667))
    x = x ^ x >> np.uint64(14)
    return x >> np.uint64(15), x % np.uint64(1 << 17)


def in_8_bits(x, w, signed):
    """The values that 8-bit codes stand for, in float64; w: thresholds in 1 / 2^17."""
    x = np.asarray(x, dtype=np.float64)
    out = np.empty_like(x)
    lo = -126 if signed else -254
    least = 2.0 ** math.floor(lo / 8) * (1 + (lo % 8) / 8)
    for b in range(0, x.size, BLOCK):
        part, theta = x[b:b + BLOCK], np.asarray(w[b:b + BLOCK], dtype=np.float64) / 2 ** 17
        most = np.float32(np.abs(part).max())
        if not most <= 2.0 ** 127:
            out[b:b + BLOCK] = np.nan
            continue
        if most == 0:
            out[b:b + BLOCK] = 0
            continue
        scale = 2.0 ** max(math.ceil(math.log2(most)), -126)
        y = np.minimum(np.abs(part) / scale, 1.0)
        m, e = np.frexp(y)
        eighths = (2 * m - 1) * 8
        f = np.floor(eighths)
        f = f + (eighths - f + theta >= 1)
        q = np.minimum(np.ldexp(1 + f / 8, e - 1), 1.0)
        under = np.where(y / least + theta >= 1, least, 0.0) if signed else np.full_like(y, least)
        q = np.where(y < least, under, q)
        out[b:b + BLOCK] = np.where(y > 0, q, 0.0) * scale * np.sign(part)
    return out


def embed_gradient(ids, dy, vocab, scale, pad_id=-1):
    """(sum, sum of magnitudes, tokens) of every row of the vocabulary."""
    ids, dy = ids.reshape(-1), dy.reshape(-1, dy.shape[-1])
    keep = (ids >= 0) & (ids < vocab) & (ids != pad_id)
    total, size, count = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1])), np.zeros(vocab)
    np.add.at(total, ids[keep], scale * dy[keep])
    np.add.at(size, ids[keep], abs(scale) * np.abs(dy[keep]))
    np.add.at(count, ids[keep], 1)
    return total, size, count


def embed_bound(total, size, count, out_bf16, old=None):
    """fp32 sum of `count` terms, the product with the scale (itself rounded) and, with `old`, one sum more; then the output's rounding."""
    b = EPS32 * (count[:, None] + 2) * size + 2.0 ** -126
    if old is not None:
        total = total + old
        b = b + EPS32 * np.abs(total)
    return b * (1 + EPS16) + EPS16 * np.abs(total) if out_bf16 else b


def in_8_bits_of_many(x, w, signed):
    """in_8_bits for millions of elements: all blocks at once."""
    x = np.asarray(x, dtype=np.float64)
    pad = -x.size % BLOCK
    b = np.pad(x, (0, pad)).reshape(-1, BLOCK)
    theta = np.pad(np.asarray(w, dtype=np.float64), (0, pad)).reshape(-1, BLOCK) / 2 ** 17
    lo = -126 if signed else -254
    least = 2.0 ** math.floor(lo / 8) * (1 + (lo % 8) / 8)
    most = np.abs(b).max(axis=1, keepdims=True).astype(np.float32).astype(np.float64)
    held = (most > 0) & (most <= 2.0 ** 127)
    m, e = np.frexp(np.where(held, most, 1.0))
    scale = np.ldexp(1.0, np.maximum(np.where(m == 0.5, e - 1, e), -126))
    y = np.minimum(np.abs(b) / scale, 1.0)
    m, e = np.frexp(y)
    eighths = (2 * m - 1) * 8
    f = np.floor(eighths)
    f = f + (eighths - f + theta >= 1)
    q = np.minimum(np.ldexp(1 + f / 8, e - 1), 1.0)
    under = np.where(y / least + theta >= 1, least, 0.0) if signed else np.full_like(y, least)
    q = np.where(y < least, under, q)
    out = np.where(y > 0, q, 0.0) * scale * np.sign(b)
    out = np.where(held, out, np.where(most == 0, 0.0, np.nan))
    return out.reshape(-1)[:x.size]
