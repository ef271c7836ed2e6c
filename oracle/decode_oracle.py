"""Plain fp64 numpy forms of the decoding operators, for the tests: rotary
positions, the 4-bit cache, attention over it, and log probabilities of given
tokens.  Written from their definitions; shares no code with the kernels."""
from __future__ import annotations

import math

import numpy as np

GROUP = 64


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def rotary_theta(rot, base, scaling="plain", factor=1.0, original_length=0, beta_fast=32.0, beta_slow=1.0):
    """Radians a position of each pair, and the amplitude."""
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2.0))
    th = base ** (-2.0 * i / rot)
    if scaling == "linear":
        th = th / factor
    if scaling == "parts":
        g = np.clip((original_length * th / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow), 0, 1)
        th = th * (g + (1 - g) / factor)
        return th, 0.1 * math.log(factor) + 1.0
    return th, 1.0


def turns(positions, freqs):
    """positions x frequencies (units of 2^-64 turns) as turns in [0, 1), in whole numbers up to the division."""
    return np.array([[((int(p) * int(f)) % (1 << 64)) / 2.0 ** 64 for f in freqs] for p in positions])


def rotary(x, positions, freqs, interleaved, amplitude, inverse=False):
    """x (tokens, heads, D) turned by positions; freqs as int64 words."""
    x = np.asarray(x, np.float64)
    half = len(freqs)
    phi = 2 * math.pi * turns(positions, freqs)[:, None, :] * (-1 if inverse else 1)
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    c, d = amplitude * (a * np.cos(phi) - b * np.sin(phi)), amplitude * (b * np.cos(phi) + a * np.sin(phi))
    y = x.copy()
    if interleaved:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = c, d
    else:
        y[..., :half], y[..., half:2 * half] = c, d
    return y


# ---------------------------------------------------------------------------
# the 4-bit cache
# ---------------------------------------------------------------------------
def kv4_quantize(x):
    """(codes, scales, zero points) of x (..., D): scales and zero points (..., D / 64); scale NaN for a group with
    a NaN or an infinity."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    lo, hi = np.minimum(g.min(-1), 0), np.maximum(g.max(-1), 0)
    s = (hi - lo) / 15
    unit = np.ldexp(1.0, np.maximum(np.frexp(np.maximum(s, 2.0 ** -14))[1] - 7, -20))
    s = np.minimum(np.ceil(s / unit) * unit, 4352.0)
    by = np.where(s > 0, s, 1.0)
    z = np.clip(np.rint(-lo / by), 0, 15)
    c = np.clip(np.rint(g / by[..., None]) + z[..., None], 0, 15)
    return c.reshape(x.shape).astype(np.int64), np.where(fine, s, np.nan), z.astype(np.int64)


def kv4_values(x):
    """What x stands for once it is held in 4 bits."""
    c, s, z = kv4_quantize(x)
    g = c.reshape(c.shape[:-1] + (-1, GROUP))
    return (s[..., None] * (g - z[..., None])).reshape(c.shape)


def kv4_encode(cache, page, k, v, table, first, heads):
    """Writes k and v (tokens, heads, D) of one sequence from position `first` on into cache (pages, heads, bytes)."""
    dim = k.shape[-1]
    half, groups = dim // 2, dim // GROUP
    for which, x in ((0, k), (1, v)):
        c, s, z = kv4_quantize(x)
        words = np.where(np.isnan(s), 0x7E00, s.astype(np.float16).view(np.uint16).astype(np.int64) | z)
        c = np.where(np.repeat(np.isnan(s), GROUP, -1), 0, c)
        byte = (c[..., :half] | c[..., half:] << 4).astype(np.uint8)
        for t in range(x.shape[0]):
            p = first + t
            pg, off = int(table[p // page]), p % page
            for h in range(heads):
                m = cache[pg, h]
                if which == 0:
                    m[off * half:(off + 1) * half] = byte[t, h]
                else:
                    at = page * half + off // 16 * half * 16 + off % 16
                    m[at:at + 16 * half:16] = byte[t, h]
                w = page * dim + 2 * (off * 2 + which) * groups
                m[w:w + 2 * groups] = words[t, h].astype("<u2").view(np.uint8)


def kv4_decode(cache, page, dim, table, n, head):
    """K and V (n, D) of one head of a sequence; tokens of pages outside the cache are NaN in `there`."""
    half, groups = dim // 2, dim // GROUP
    K, V, there = np.zeros((n, dim)), np.zeros((n, dim)), np.zeros(n, bool)
    for p in range(n):
        pg, off = int(table[p // page]), p % page
        if not 0 <= pg < cache.shape[0]:
            continue
        there[p] = True
        m = cache[pg, head]
        for which, out in ((0, K), (1, V)):
            at = page * half + off // 16 * half * 16 + off % 16
            byte = m[off * half:(off + 1) * half] if which == 0 else m[at:at + 16 * half:16]
            w = page * dim + 2 * (off * 2 + which) * groups
            word = m[w:w + 2 * groups].copy().view("<u2").astype(np.int64)
            s = (word & 0xFFF0).astype(np.uint16).view(np.float16).astype(np.float64)
            c = np.concatenate([byte & 15, byte >> 4]).astype(np.float64).reshape(groups, GROUP)
            out[p] = (s[:, None] * (c - (word & 15)[:, None])).reshape(-1)
    return K, V, there


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def attention(q, K, V, there, positions, scale, window=0):
    """q (rows, D) of one query head at `positions` over K and V (n, D): (out, lse, sum of p |v|, largest sum of
    |q k| scale a row sees)."""
    q = np.asarray(q, np.float64)
    j = np.arange(K.shape[0])
    out, lse = np.zeros_like(q), np.full(len(q), -np.inf)
    mass, reach = np.zeros_like(q), np.zeros(len(q))
    for r, p in enumerate(positions):
        seen = (j <= p) & there & ((j > p - window) if window else True)
        if not seen.any():
            continue
        x = scale * (K[seen] @ q[r])
        m = x.max()
        e = np.exp(x - m)
        lse[r] = m + np.log(e.sum())
        w = e / e.sum()
        out[r], mass[r] = w @ V[seen], w @ np.abs(V[seen])
        reach[r] = scale * (np.abs(K[seen]) @ np.abs(q[r])).max()
    return out, lse, mass, reach


# ---------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------
def logprobs(x, targets, scale, top):
    """(logprob, entropy, lse, top logprobs, top ids, p) of each row of x (rows, V)."""
    x = np.asarray(x, np.float64)
    z = scale * x
    m = z.max(-1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.where(np.isneginf(m), 0.0, np.exp(z - m))
        total = e.sum(-1)
        lse = np.where(np.isneginf(m[:, 0]), -np.inf, np.log(total) + m[:, 0])
        p = np.where(np.isneginf(m), 0.0, e / total[:, None])
        lp = np.where(np.isneginf(z), np.where(np.isnan(lse[:, None]), np.nan, -np.inf), z - lse[:, None])
        entropy = np.where(np.isneginf(lse), 0.0, -np.where(p > 0, p * lp, p).sum(-1))
    pick = np.array([0.0 if y < 0 else lp[r, y] if y < x.shape[1] else np.nan for r, y in enumerate(targets)])
    ids = np.stack([np.lexsort((np.arange(x.shape[1]), -row))[:top] for row in x]) if top else np.zeros((len(x), 0), int)
    return pick, entropy, lse, np.take_along_axis(lp, ids, 1), ids, p


def logprobs_backward(x, targets, scale, g_logprob, g_entropy):
    _, entropy, lse, _, _, p = logprobs(x, targets, scale, 0)
    with np.errstate(invalid="ignore"):
        lp = np.where(p > 0, scale * np.asarray(x, np.float64) - lse[:, None], 0.0)
    g = np.where(targets >= 0, g_logprob, 0.0)
    d = -p * (g[:, None] + g_entropy[:, None] * (lp + entropy[:, None]))
    for r, y in enumerate(targets):
        if 0 <= y < x.shape[1]:
            d[r, y] += g[r]
    return scale * d
