"""Group-scaled rows in plain numpy, for the tests: the storage format read field by field, the
quantisation rule in 32-bit steps as it is defined, products and gradients in 64 bits."""
import math

import numpy as np

TINY = np.float32(2.0 ** -100)


def unpack(words, cols, bits, signed):
    """int64 (rows, cols) from int32/uint32 words."""
    w = np.asarray(words).view(np.uint32).astype(np.uint64)
    per = 32 // bits
    q = np.zeros((w.shape[0], cols), dtype=np.int64)
    for j in range(cols):
        q[:, j] = (w[:, j // per] >> np.uint64(j % per * bits)) & np.uint64((1 << bits) - 1)
    if signed:
        q = np.where(q >= 1 << (bits - 1), q - (1 << bits), q)
    return q


def spare_bits(words, cols, bits):
    """What the last word of every row holds behind the row's end (0 by the format)."""
    used = (cols - 1) % (32 // bits) + 1
    last = np.asarray(words).view(np.uint32)[:, -1].astype(np.uint64)
    return last >> np.uint64(used * bits)


def values(q, scale, zero, group):
    """float64 values of whole numbers q (rows, cols)."""
    at = np.arange(q.shape[1]) // group
    z = 0 if zero is None else zero.astype(np.int64)[:, at]
    with np.errstate(invalid="ignore"):
        return scale.astype(np.float64)[:, at] * (q - z)


def quantize(x, bits, signed, group):
    """(q, scale, zero) of float32 rows, every step rounded as the rule says."""
    f = np.float32
    rows, cols = x.shape
    groups = -(-cols // group)
    top = f((1 << (bits - 1)) - 1 if signed else (1 << bits) - 1)
    q = np.zeros((rows, cols), dtype=np.int64)
    scale = np.zeros((rows, groups), dtype=f)
    zero = np.zeros((rows, groups), dtype=np.uint8)
    with np.errstate(all="ignore"):
        for g in range(groups):
            v = x[:, g * group:(g + 1) * group].astype(f)
            low = np.zeros(rows, f) if signed else np.minimum(f(0), np.fmin.reduce(v, axis=1))
            span = np.abs(v).max(axis=1) if signed else np.maximum(f(0), np.fmax.reduce(v, axis=1)) - low
            bad = ~np.isfinite(v).all(axis=1) | ~np.isfinite(span)
            none = span < TINY
            inv = np.where(none | bad, f(0), top / np.where(none | bad, f(1), span)).astype(f)
            scale[:, g] = np.where(bad, f(np.nan), np.where(none, f(0), span * (f(1) / top)))
            z = np.where(bad, f(0), np.clip(np.rint(-low * inv), f(0), top)) if not signed else np.zeros(rows, f)
            t = np.rint(np.where(bad[:, None], f(0), v) * inv[:, None]) + z[:, None]
            q[:, g * group:(g + 1) * group] = np.where(bad[:, None], 0, np.clip(t, -top if signed else f(0), top))
            zero[:, g] = z
    return q, scale, None if signed else zero


def activation(g, act):
    """act(g) and act'(g) in 64 bits."""
    erf = np.vectorize(math.erf, otypes=[np.float64])
    if act == "silu":
        p = 1 / (1 + np.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + erf(g / math.sqrt(2)))
    return g * p, p + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
