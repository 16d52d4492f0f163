"""CPU oracle of the base layer's operators (TEST INFRASTRUCTURE ONLY; shares nothing with the library), from their formulas: rows and weights in 8 bits,
products, routing, norms between blocks.

What a choice of codes is decided by (quotients, products, the rounding) is computed in 32 bits with one rounding per operation, as the
library's contract has it; everything else in 64 bits.
"""
import math

import numpy as np

BLOCK = 128
TINY = np.float32(2.0 ** -100)


def e4m3_table():
    """Value of each of the 127 codes that are not negative and not NaN."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


_TABLE = e4m3_table()
_MIDDLE = (_TABLE[:-1] + _TABLE[1:]) / 2


def to_codes(x):
    """Bytes of the nearest e4m3 values, ties to the even code; |x| up to 464."""
    a = np.abs(np.asarray(x, np.float64))
    low, high = np.searchsorted(_MIDDLE, a, side="left"), np.searchsorted(_MIDDLE, a, side="right")  # they differ at a tie
    c = np.where(low == high, low, np.where(low % 2 == 0, low, high))
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def values(codes):
    c = codes.astype(np.int64)
    return np.where(c & 128, -1.0, 1.0) * _TABLE[c & 127]


def _scale(amax, bad):
    amax = amax.astype(np.float32)
    none = (amax < TINY) | bad
    with np.errstate(all="ignore"):
        s = np.where(bad, np.float32(np.nan), np.where(none, np.float32(0), amax / np.float32(448)))
        inv = np.where(none, np.float32(0), np.float32(448) / amax)
    return s.astype(np.float32), inv.astype(np.float32)


def _coded(x, inv):
    with np.errstate(all="ignore"):
        return to_codes(np.where(inv == 0, np.float32(0), x * inv).astype(np.float32))


def rows(x):
    """x [rows, k] (float32) -> codes (bytes), scales [blocks, rows]."""
    x = np.asarray(x, np.float32)
    n, k = x.shape
    pad = np.pad(x, ((0, 0), (0, -k % BLOCK))).reshape(n, -1, BLOCK)
    bad = ~np.isfinite(pad).all(-1)
    s, inv = _scale(np.where(bad, 0, np.abs(np.nan_to_num(pad)).max(-1)), bad)
    return _coded(pad, inv[..., None]).reshape(n, -1)[:, :k], np.ascontiguousarray(s.T)


def weights(w):
    """w [n, k] (float32) -> codes, scales [blocks of n, blocks of k]."""
    w = np.asarray(w, np.float32)
    n, k = w.shape
    pad = np.pad(w, ((0, -n % BLOCK), (0, -k % BLOCK)))
    t = pad.reshape(pad.shape[0] // BLOCK, BLOCK, pad.shape[1] // BLOCK, BLOCK)
    bad = ~np.isfinite(t).all((1, 3))
    s, inv = _scale(np.where(bad, 0, np.abs(np.nan_to_num(t)).max((1, 3))), bad)
    return _coded(t, inv[:, None, :, None]).reshape(pad.shape)[:n, :k], s


def row_values(codes, scales):
    return values(codes) * np.repeat(scales.astype(np.float64), BLOCK, 0)[:codes.shape[1]].T


def weight_values(codes, scales):
    n, k = codes.shape
    return values(codes) * np.repeat(np.repeat(scales.astype(np.float64), BLOCK, 0)[:n], BLOCK, 1)[:, :k]


def activated(x, act):
    """x [rows, 2k] in 64 bits -> act(first half) * second half."""
    a, b = np.split(x, 2, axis=1)
    with np.errstate(over="ignore"):
        z = a if act == "silu" else 2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)
        return a / (1 + np.exp(-z)) * b


def norm(v, weight=None, bias=None, eps=1e-6, center=False, offset=0.0):
    if center:
        v = v - v.mean(-1, keepdims=True)
    y = v / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    if weight is not None:
        y = y * (offset + weight)
    return y if bias is None else y + bias


def gathered(block, places, place_weights):
    out = np.zeros((len(places), block.shape[1]))
    for t in range(len(places)):
        for p, w in zip(places[t], place_weights[t]):
            if 0 <= p < len(block):
                out[t] += np.float64(w) * block[p]
    return out


def route(logits, k, renormalise=True, scale=1.0):
    """-> experts, weights, offsets, rows, places by loops over tokens."""
    n, e = logits.shape
    experts, places = np.full((n, k), -1, np.int32), np.full((n, k), -1, np.int32)
    w = np.zeros((n, k))
    for t in range(n):
        x = logits[t].astype(np.float64)
        bad = np.isnan(x).any() or np.isposinf(x).any()
        order = sorted((i for i in range(e) if x[i] > -math.inf), key=lambda i: (-x[i], i))[:k]
        experts[t, :len(order)] = order
        if bad:
            w[t] = math.nan
        elif order:
            top = x[order[0]]
            p = np.exp(x[order] - top)
            w[t, :len(order)] = scale * p / (p.sum() if renormalise else np.exp(x[x > -math.inf] - top).sum())
    of = [[(t, j) for t in range(n) for j in range(k) if experts[t, j] == i] for i in range(e)]
    offsets = np.concatenate([[0], np.cumsum([len(o) for o in of])]).astype(np.int32)
    rows = np.full(n * k, -1, np.int32)
    at = 0
    for o in of:
        for t, j in o:
            rows[at], places[t, j] = t, at
            at += 1
    return experts, w, offsets, rows, places
