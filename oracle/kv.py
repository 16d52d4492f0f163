"""CPU oracle of rotary positions, the 4-bit KV cache and attention over it (TEST INFRASTRUCTURE ONLY; shares nothing with
the library).  Written from the formulas in 64 bits, one row at a time; `chosen(..., bits=32)` makes the same choices of codes in
fp32, one rounding per operation, which the library's bytes have to equal.

Pins (tests/test_oracle_kv.py): closed forms and hand-worked rows.
"""
import math

import numpy as np


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, low=0.0, high=0.0, original_len=0):
    f = []
    for j in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base
        x = b ** (-2 * j / rot)
        if scaling == "linear":
            x /= factor
        if scaling == "turns":
            turns = original_len * x / (2 * math.pi)
            u = min(1.0, max(0.0, (turns - low) / (high - low)))
            x = (1 - u) * x / factor + u * x
        f.append(x)
    return np.array(f)


def angles(freqs, positions, magnitude=1.0):
    """[positions][rot/2][2] of (cos, sin)."""
    a = np.asarray(positions, np.float64)[:, None] * freqs[None, :]
    return np.stack([magnitude * np.cos(a), magnitude * np.sin(a)], -1)


def rotate(x, cs, interleaved, inverse=False):
    """x [tokens, heads, d], cs [tokens, rot/2, 2]; in x's own precision, one rounding per operation."""
    rot = 2 * cs.shape[1]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    if inverse:
        sin = -sin
    first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    y = x.copy()
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def to_bf16(x):
    """Nearest bf16 of fp32 values (ties to even), as fp32."""
    x = np.asarray(x, np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), r, x)


def chosen(x, bits=64):
    """x [rows, d] -> (codes, scale, min): what a row is kept as."""
    t = np.float32 if bits == 32 else np.float64
    x = np.asarray(x).astype(t)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        s = to_bf16(((hi - lo) / t(15)).astype(np.float32)).astype(t)
        m = to_bf16(lo.astype(np.float32)).astype(t)
        bad = ~(np.isfinite(x).all(-1) & np.isfinite(s) & np.isfinite(m))
        s = np.where(s < 2.0 ** -100, t(0), s)
        q = np.where(s[:, None] > 0, (x - m[:, None]) / np.where(s > 0, s, 1)[:, None], t(0))
        c = np.clip(np.rint(q), 0, 15)
    c[bad] = 0
    s[bad] = np.nan
    m[bad] = np.nan
    return c.astype(np.int64), s, m


def value_nibble(token, d, head_dim):
    """(byte in the block of 32 tokens, high nibble?) of a value's code."""
    u = token % 32
    g, n = u % 16 // 4, u // 16 * 4 + u % 4
    quarter, rest = divmod(d, head_dim // 4)
    tile, r = rest // 4, quarter * 4 + rest % 4
    word = ((tile // 4 * 4 + g) * 16 + r) * 4 + tile % 4
    return 4 * word + n // 2, n % 2


class KvOracle:
    """The pages as bytes, written and read one row at a time."""

    def __init__(self, pages, heads, head_dim, page_tokens):
        self.p, self.h, self.d, self.t = pages, heads, head_dim, page_tokens  # pages: uint8 [n, bytes], changed in place
        self.nib = np.array([[value_nibble(t, d, head_dim) for d in range(head_dim)] for t in range(32)])

    def _head(self, page, head):
        n = self.t * (self.d + 8)
        return self.p[page, head * n:(head + 1) * n]

    def write(self, page, slot, head, values, codes, s, m):
        b, d, t = self._head(page, head), self.d, self.t
        par = np.array([s, m], np.float32).view(np.uint32) >> 16
        par = np.where(np.isnan([s, m]), 0x7FC0, par).astype(np.uint16).view(np.uint8)
        at = t * d + (t * 4 if values else 0) + slot * 4
        b[at:at + 4] = par
        c = np.asarray(codes).astype(np.uint8)
        if values:  # every channel has a byte of its own
            nib = self.nib[slot % 32]
            byte = t * d // 2 + slot // 32 * 16 * d + nib[:, 0]
            b[byte] = np.where(nib[:, 1] == 1, b[byte] & 0x0F | c << 4, b[byte] & 0xF0 | c)
        else:
            b[slot * (d // 2):(slot + 1) * (d // 2)] = c[0::2] | c[1::2] << 4

    def row(self, page, slot, head, values):
        """The values that a row stands for, in 64 bits."""
        b, d, t = self._head(page, head), self.d, self.t
        if values:
            nib = self.nib[slot % 32]
            byte = b[t * d // 2 + slot // 32 * 16 * d + nib[:, 0]].astype(np.int64)
            c = np.where(nib[:, 1] == 1, byte >> 4, byte & 15)
        else:
            byte = b[slot * (d // 2):(slot + 1) * (d // 2)].astype(np.int64)
            c = np.stack([byte & 15, byte >> 4], -1).reshape(-1)
        at = t * d + (t * 4 if values else 0) + slot * 4
        with np.errstate(invalid="ignore"):  # a scale or min may be NaN
            s, m = (b[at:at + 4].copy().view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
            return m + s * c


def attend(q, keys, values, scale, places, causal=True, window=0, holes=()):
    """q [rows, heads, d]; keys, values [places, kv heads, d]; places[row]: its own.  -> (out, A, X): A bounds what a rounding of
    a weight can move (sum of weight * |value|), X the size of a logit's terms (max over seen keys of scale * sum |q k|)."""
    rows, heads, d = q.shape
    n, kvh = keys.shape[:2]
    out, amp, size = np.zeros((rows, heads, d)), np.zeros((rows, heads)), np.zeros((rows, heads))
    for r in range(rows):
        see = np.ones(n, bool)
        see[list(holes)] = False
        if causal:
            see &= np.arange(n) <= places[r]
            if window:
                see &= np.arange(n) > places[r] - window
        if not see.any():
            continue
        for h in range(heads):
            k, v = keys[see, h // (heads // kvh)], values[see, h // (heads // kvh)]
            t = scale * (k @ q[r, h])
            p = np.exp(t - t.max())
            p /= p.sum()
            out[r, h] = p @ v
            amp[r, h] = p @ np.abs(v).max(-1)
            size[r, h] = (scale * (np.abs(k) @ np.abs(q[r, h]))).max()
    return out, amp, size
