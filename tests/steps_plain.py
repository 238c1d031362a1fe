"""Plain forms of the client's other steps (pvmvmd_block_norm, pvmvmd_glu, pvmvmd_sample) in numpy: the definitions
with every rounding, and the same formulas in 64 bits without them."""
import numpy as np

Q = 2013265921
F = np.float32
MAX = F(3.402823466e38)
LOG2E = F(1.4426950408889634)
COEF = [F(c) for c in (-0.00132647157, 0.00967151299, -0.0555073395, 0.240222424, -0.693147004)]


def centred(v):
    v = np.asarray(v).astype(np.int64) & 0xFFFFFFFF
    return np.where(v > (Q - 1) // 2, v - Q, v)


def field(n):
    n = np.asarray(n, np.int64)
    return np.where(n < 0, n + Q, n).astype(np.int32)


def read(x, scale=1.0, token=None, channel=None, is_field=False, wide=False):
    """x (numpy: integers of field elements, or 32-bit values) with its scales, rounded step by step or in 64 bits."""
    t = np.float64 if wide else F
    v = (centred(x) if is_field else np.asarray(x)).astype(t)
    c = t(F(scale))
    if token is not None:
        c = (c * token.astype(t))[:, None]
    v = v * c
    return v if channel is None else v * channel.astype(t)


def norm(x, kind, w=None, b=None, eps=1e-6, add=0.0, wide=False):
    t = np.float64 if wide else F
    x = x.astype(t)
    if kind == "layer":
        x = x - x.astype(np.float64).mean(-1, keepdims=True).astype(t)
    inv = (1 / np.sqrt(np.square(x.astype(np.float64)).mean(-1, keepdims=True) + np.float64(F(eps)))).astype(t)
    x = x * inv
    if w is not None or add:
        x = x * ((w.astype(t) if w is not None else t(1)) + t(F(add)))
    return x if b is None else x + b.astype(t)


def integers(z, scale, limit, dynamic):
    """-> (integers, steps or None)"""
    if not dynamic:
        with np.errstate(invalid="ignore"):
            v = z * F(scale)
            return np.rint(np.clip(np.where(np.isnan(v), F(0), v), F(-limit), F(limit))).astype(np.int64), None
    big = np.abs(z).max(-1, keepdims=True)
    fine = np.isfinite(z).all(-1, keepdims=True)
    with np.errstate(all="ignore"):
        m = np.minimum(F(limit) / big, MAX)
        n = np.where(fine, np.rint(np.clip(z * m, F(-limit), F(limit))), 0)
        step = np.where(fine, big / F(limit), F(np.nan))
    return n.astype(np.int64), step[:, 0].astype(F)


def poly(f):
    p = f * COEF[0] + COEF[1]
    for c in COEF[2:]:
        p = p * f + c
    return p * f + F(1)


def power(d):
    """2^-d"""
    d = np.clip(d, F(-128), F(125))
    n = np.rint(d)
    return (poly(d - n).view(np.int32) - (n.astype(np.int32) << 23)).view(F)


def act(x, name):
    with np.errstate(all="ignore"):
        if name == "none":
            return x
        if name == "relu":
            return np.where(x < 0, F(0), x)
        if name == "gelu":
            c = 2 * np.sqrt(2 / np.pi) * 1.4426950408889634
            d = (x * x * F(0.044715 * c) + F(c)) * x
        else:
            d = x * LOG2E
        e = F(1) + power(np.where(np.isnan(d), F(0), d).astype(F))
        r = (F(1) if name == "sigmoid" else x) / e
        return np.where(np.isnan(x), x, r).astype(F)


def act64(x, name):
    if name == "none":
        return x
    if name == "relu":
        return np.maximum(x, 0)
    with np.errstate(over="ignore"):
        if name == "gelu":
            return x / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x**3)))
        return (1 if name == "sigmoid" else x) / (1 + np.exp(-x))


def distances(l, m, channel=None, allowed=None):
    """x of a row: 32-bit values, -infinity where a token may not be chosen."""
    with np.errstate(all="ignore"):
        x = l * F(m)
        if channel is not None:
            x = x * channel
        x = np.where(x > -np.inf, np.minimum(x, MAX), F(-np.inf)).astype(F)
    if allowed is not None:
        i = np.arange(len(x))
        x = np.where((allowed[i // 32].astype(np.int64) >> (i % 32)) & 1 == 1, x, F(-np.inf)).astype(F)
    return x


def weights(x):
    """Whole numbers of Python, of any length."""
    with np.errstate(all="ignore"):
        d = np.fmin(x.max() - x, F(63))
    n = np.rint(d)
    r = np.rint(poly((d - n).astype(F)) * F(4194304)).astype(np.int64)
    return [(int(a) << 18) >> int(b) for a, b in zip(r, n)]


def kept(x, top_k=0, top_p=1.0, min_p=0.0):
    """(weights, indexes of the tokens that the limits leave), in the vocabulary's order."""
    w = weights(x)
    order = sorted((i for i in range(len(x)) if x[i] > -np.inf), key=lambda i: (-float(x[i]), i))
    if top_k >= 1:
        order = order[:top_k]
    if top_p < 1:
        part = (sum(w[i] for i in order) * int(float(F(max(top_p, 0))) * 2**31)) >> 31
        before, left = 0, []
        for i in order:
            if left and before >= part:
                break
            left.append(i)
            before += w[i]
        order = left
    least = int(float(F(min(max(min_p, 0), 1))) * 2**31) << 9 if min_p > 0 else 0
    return w, sorted(i for i in order if w[i] >= least)


def sample(x, temperature, top_k, top_p, min_p, word):
    """-> (token, log of its probability)"""
    if not (x > -np.inf).any():
        return -1, -np.inf
    if not temperature > 0:
        return int(np.argmax(x)), 0.0
    w, left = kept(x, top_k, top_p, min_p)
    Z = sum(w[i] for i in left)
    at, run = (Z * (int(word) & 0xFFFFFFFF)) >> 32, 0
    for i in left:
        run += w[i]
        if run > at:
            return i, float(np.log(w[i] / Z))
    raise AssertionError("the whole is more than a part of it")


def sample_long(x, temperature, top_k, top_p, min_p, word):
    """The same for many tokens, whose sums fit 62 bits: numpy's sorts and sums of whole numbers of 64 bits."""
    with np.errstate(all="ignore"):
        d = np.fmin(x.max() - x, F(63))
    n = np.rint(d)
    w = (np.rint(poly((d - n).astype(F)) * F(4194304)).astype(np.int64) << 18) >> n.astype(np.int64)
    keep = w >= (int(float(F(min(max(min_p, 0), 1))) * 2**31) << 9)
    if 0 < top_k < len(x) or top_p < 1:
        order = np.lexsort((np.arange(len(x)), -x.astype(np.float64)))
        last = top_k if 0 < top_k < len(x) else len(x)
        run = np.cumsum(w[order[:last]])
        if top_p < 1:
            part = int(run[-1]) * int(float(F(top_p)) * 2**31) >> 31
            last = max(1, int(np.searchsorted(run, part, side="left")) + 1)
        limits = np.zeros(len(x), bool)
        limits[order[:last]] = True
        keep &= limits
    run = np.cumsum(np.where(keep, w, 0))
    i = int(np.searchsorted(run, int(run[-1]) * (int(word) & 0xFFFFFFFF) >> 32, side="right"))
    return i, float(np.log(int(w[i]) / int(run[-1])))


def multiplier(scale, token_scale, temperature):
    with np.errstate(all="ignore"):
        m = F(scale) if token_scale is None else F(scale) * F(token_scale)
        if temperature > 0:
            m = m * (LOG2E / F(temperature))
            m = np.minimum(m, MAX) if not np.isnan(m) else m
    return m
