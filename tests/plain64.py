"""Plain 64-bit definitions of the layer operators (numpy): layer norm, rotary
positions, cached rows in 8 or 4 bits and the attention that reads them.  They
share no code with the library."""
import numpy as np

U = 2.0 ** -24                                  # half a step of fp32, relative
HALF = {"f32": U, "bf16": 2.0 ** -8}


# ------------------------------------------------------------------ layer norm
def layer_norm(h, gamma, beta, eps):
    mu = h.mean(1)
    r = 1.0 / np.sqrt(((h - mu[:, None]) ** 2).mean(1) + eps)
    xh = (h - mu[:, None]) * r[:, None]
    return xh * gamma + beta, mu, r


def layer_norm_bwd(h, gamma, mu, r, dy, dsum):
    xh = (h - mu[:, None]) * r[:, None]
    g = dy * gamma
    dx = r[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx + (0 if dsum is None else dsum), (dy * xh).sum(0), dy.sum(0)


# ------------------------------------------------------------------ rotary
def rotary(x, pos, axis, omega, pairs, interleaved, sign=1.0):
    """x [n, H, dh]"""
    y = x.copy()
    th = sign * pos[:, axis] * omega            # [n, pairs]
    c, s = np.cos(th)[:, None], np.sin(th)[:, None]
    a = np.arange(pairs) * (2 if interleaved else 1)
    b = a + (1 if interleaved else pairs)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


# ------------------------------------------------------------------ cached rows
def grid(fmt):
    """The values of the format's non-negative codes (NaN for 0x7f of e4m3)."""
    if fmt == 4:
        return np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
    v = [m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    v[-1] = np.nan
    return np.array(v)


def record(parts, width, fmt):
    """code bytes of a part, groups of a part, content bytes, stride"""
    code = -(-width // 8) * fmt
    groups = -(-width // 32)
    content = parts * (code + groups)
    first = -(-content // 16) * 16
    cand = [first] + [s for s in range(first + 16, content + content // 8 + 1, 16)]
    lines = [sum(-(-(k * s % 128 + content) // 128) for k in range(8)) for s in cand]
    return code, groups, content, cand[int(np.argmin(lines))]


def quantize(x, fmt):
    """x [..., width] (finite or not) -> (codes, scale bytes [..., groups])"""
    g = grid(fmt)
    g = g[~np.isnan(g)]
    width = x.shape[-1]
    codes = np.zeros(x.shape, np.uint8)
    scales = np.zeros(x.shape[:-1] + (-(-width // 32),), np.uint8)
    for k, a in enumerate(range(0, width, 32)):
        v = x[..., a:a + 32].astype(np.float64)
        bad = ~np.isfinite(v).all(-1)
        v = np.where(bad[..., None], 0.0, v)
        top = np.abs(v).max(-1)
        e = np.full(top.shape, -127)
        for p in range(-127, 128):               # the smallest scale that holds the largest value
            e = np.where(top > g[-1] * 2.0 ** p, p + 1, e)
        u = np.abs(v) / 2.0 ** e[..., None].astype(np.float64)
        i = np.clip(np.searchsorted(g, u, side="right") - 1, 0, len(g) - 2)
        lo, hi = u - g[i], g[i + 1] - u
        i = i + ((hi < lo) | ((hi == lo) & (i % 2 == 1)))
        codes[..., a:a + 32] = i + np.where(np.signbit(v), 1 << (fmt - 1), 0)
        codes[..., a:a + 32][bad] = 0
        scales[..., k] = np.where(bad, 255, e + 127)
    return codes, scales


def values(codes, scales, fmt):
    g = grid(fmt)
    t = np.concatenate([g, -g])
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    with np.errstate(invalid="ignore"):
        return t[codes] * np.repeat(s, 32, axis=-1)[..., :codes.shape[-1]]


def pack(codes, scales, fmt, fill=0):
    """codes [n, parts, width], scales [n, parts, groups] -> records [n, stride]"""
    n, parts, width = codes.shape
    code, groups, content, stride = record(parts, width, fmt)
    c = np.zeros((n, parts, -(-width // 8) * 8), np.uint8)
    c[..., :width] = codes
    if fmt == 4:
        c = c[..., 0::2] | (c[..., 1::2] << 4)
    out = np.full((n, stride), fill, np.uint8)
    out[:, :parts * code] = c.reshape(n, -1)
    out[:, parts * code:content] = scales.reshape(n, -1)
    return out


def unpack(rec, parts, width, fmt):
    code, groups, content, _ = record(parts, width, fmt)
    c = rec[:, :parts * code].reshape(len(rec), parts, code)
    if fmt == 4:
        c = np.stack([c & 15, c >> 4], -1).reshape(len(rec), parts, 2 * code)
    return values(c[..., :width], rec[:, parts * code:content].reshape(len(rec), parts, groups), fmt)


def slots(ids, bound, slot_map, rows):
    ok = (ids >= 0) & (ids < bound)
    s = np.where(ok, ids, 0)
    if slot_map is not None:
        s = slot_map[s].astype(np.int64)
    return np.where(ok & (s >= 0) & (s < rows), s, -1)


# ------------------------------------------------------------------ attention
def attention(off, Q, slot, KV, scale, slope):
    """KV [rows, 2H, dh]; edges with slot < 0 are left out.  Returns out, lse and
    per (segment, head): the largest |V|, the largest sum |q k| scale."""
    N, H, dh = Q.shape
    out, lse = np.zeros((N, H, dh)), np.full((N, H), -np.inf)
    vmax, qk = np.zeros((N, H)), np.zeros((N, H))
    for v in range(N):
        s = slot[off[v]:off[v + 1]]
        s = s[s >= 0]
        if len(s) == 0:
            continue
        K, V = KV[s, :H], KV[s, H:]
        pre = scale * (Q[v] * K).sum(-1)
        t = np.where(pre > 0, pre, slope * pre)
        m = t.max(0)
        p = np.exp(t - m)
        z = p.sum(0)
        out[v] = (p[..., None] * V).sum(0) / z[:, None]
        lse[v] = m + np.log(z)
        vmax[v] = np.abs(V).max((0, 2))
        qk[v] = abs(scale) * np.abs(Q[v] * K).sum(-1).max(0)
    return out, lse, vmax, qk
