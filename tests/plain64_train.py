"""Plain 64-bit definitions (numpy) of the products with an epilogue, the gated recurrence over a
segment's events, and the AdamW step with states in 32 or 8 bits.  They share no code with the
library."""
import math

import numpy as np
from scipy.special import erfc as _erfc

from tests.plain64 import grid


# ------------------------------------------------------------------ products
def act(kind, z):
    if kind == "relu":
        return np.maximum(z, 0)
    if kind == "gelu":
        return 0.5 * z * _erfc(-z / math.sqrt(2))
    if kind == "silu":
        return z / (1 + np.exp(-z))
    return z


def slope(kind, z):
    if kind == "relu":
        return (z > 0) * 1.0
    if kind == "gelu":
        return 0.5 * _erfc(-z / math.sqrt(2)) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        p = 1 / (1 + np.exp(-z))
        return p + z * p * (1 - p)
    return np.ones_like(z)


def linear(x, w, b, kind, res):
    """-> y, z"""
    z = x @ w.T + (0 if b is None else b)
    return act(kind, z) + (0 if res is None else res), z


def linear_bwd(x, w, kind, pre, dy):
    """-> dx, dw, db, dz"""
    dz = dy if kind == "none" else dy * slope(kind, pre)
    return dz @ w, dz.T @ x, dz.sum(0), dz


# ------------------------------------------------------------------ recurrence
def gate(g, dt):
    """-> a, u = 1 - a, du/dgate; dt: 1, or [E, 1]"""
    dt = np.maximum(dt, 0)
    rate = np.logaddexp(0, g)
    a = np.exp(-rate * dt)
    return a, -np.expm1(-rate * dt), a * dt / (1 + np.exp(-g))


def scan(off, x, g, dt, h0):
    """-> h [E, D], h_last [N, D]"""
    a, u, _ = gate(g, 1.0 if dt is None else dt[:, None])
    h = np.zeros_like(x)
    last = np.zeros((len(off) - 1, x.shape[1])) if h0 is None else h0.copy()
    for v in range(len(off) - 1):
        s = last[v].copy()
        for e in range(off[v], off[v + 1]):
            s = a[e] * s + u[e] * x[e]
            h[e] = s
        last[v] = s
    return h, last


def scan_bwd(off, x, g, dt, h0, dh, dlast):
    """-> dx, dgate, dh0"""
    a, u, k = gate(g, 1.0 if dt is None else dt[:, None])
    h, _ = scan(off, x, g, dt, h0)
    N, D = len(off) - 1, x.shape[1]
    dx, dg = np.zeros_like(x), np.zeros_like(x)
    d0 = np.zeros((N, D)) if dlast is None else dlast.copy()
    for v in range(N):
        d = d0[v].copy()
        for e in range(off[v + 1] - 1, off[v] - 1, -1):
            if dh is not None:
                d = d + dh[e]
            before = h[e - 1] if e > off[v] else (0 if h0 is None else h0[v])
            dx[e] = u[e] * d
            dg[e] = d * (x[e] - before) * k[e]
            d = a[e] * d
        d0[v] = d
    return dx, dg, d0


# ------------------------------------------------------------------ AdamW
def mix(x):
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x6A09E667)) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0xBB67AE85)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def rounding_bits(seed, t, tensor, n):
    """the 32 bits of each element of a tensor: low half for m, high half for v"""
    u = lambda k: np.array(k & 0xFFFFFFFF, np.uint64)
    key = mix(mix(u(seed ^ (t * 0x9E3779B9))) ^ u(tensor))
    return mix(mix(key) ^ np.arange(n, dtype=np.uint64))


def to_codes(x, r, root):
    """x: fp32 values in 64 bits -> (codes, scale bytes)"""
    g = grid(8)[:-1]
    n = len(x)
    codes, scales = np.zeros(n, np.uint8), np.zeros(-(-n // 32), np.uint8)
    for k in range(len(scales)):
        v, rr = x[32 * k:32 * k + 32], r[32 * k:32 * k + 32]
        if not np.isfinite(v).all():
            scales[k] = 255
            continue
        e = -127
        while np.abs(v).max() > 448 * 2.0 ** e:
            e += 1
        scales[k] = e + 127
        a = np.abs(v) / 2.0 ** e
        i = np.minimum(np.searchsorted(g, a, side="right") - 1, len(g) - 2)
        c = i + ((a - g[i]) / (g[i + 1] - g[i]) > rr / 65536.0)
        if root:
            c = np.where((c == 0) & (a > 0), 1, c)
        c = np.where(g[c] * 2.0 ** e >= 2.0 ** 128, c - 1, c)
        codes[32 * k:32 * k + 32] = c + 128 * (v < 0)
    return codes, scales


def from_codes(codes, scales):
    g = grid(8)
    with np.errstate(invalid="ignore"):
        s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
        return np.concatenate([g, -g])[codes] * np.repeat(s, 32)[:len(codes)]


def adamw(w, g, m, v, t, lr, b1, b2, eps, decay):
    """m, v: the moments -> w, m, v"""
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    step = (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return w - lr * (decay * w + step), m, v
