"""Plain forms in 64 bits of the operators of a decode step, written from their formulas (numpy alone), and the bounds
that their tests hold the kernels to.

Bounds.  u is the half-step of the type relative to the value: 2^-p for p significant bits (2^-8 for bfloat16, 2^-11 for
float16, 2^-24 for float32); e = 2^-24.

Rotation: the phase is exact, its conversion to float leaves pi 2^-25 in the angle, sine and cosine are good to 2 ulp, two
products and a sum follow: under 8 e (|x| + |y|) factor in all, then u |result| (2^-25 more below float16's normal range).

Attention: a score is a sum of D products in 32 bits, so off by at most (D + 4) e scale sum |q k|; call the largest of
these ds, with 4 e |s| more for the scaling and the exponential's argument.  Each weight is then off by a factor of 1 +- (2 ds + 4 e), numerator and denominator
alike, and rounded to the type (u); partial results are joined in 32 bits (16 e).  With A = sum p |v| / sum p:
|out error| <= (u + 4 ds + 64 e) A + u |out| (2^-24 for float16's subnormal weights and results), |lse error| <= 2 ds + 16 e (1 + |lse|).
"""
import math

import numpy as np

HALF_STEP = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}
E = 2.0 ** -24


def frequencies(rot, base=10000.0, scaling=None):
    scaling = scaling or {}
    kind, s = scaling.get("kind"), scaling.get("factor")
    if kind == "ntk" and rot > 2:
        base = base * s ** (rot / (rot - 2))
    out, magnitude = [], 1.0
    for i in range(rot // 2):
        t = 1.0 / base ** (2 * i / rot)
        if kind == "linear":
            t /= s
        if kind == "by_parts":
            turns = scaling["original_len"] * t / (2 * math.pi)
            ramp = (turns - scaling["low"]) / (scaling["high"] - scaling["low"])
            ramp = min(1.0, max(0.0, ramp))
            t = ramp * t + (1 - ramp) * t / s
            magnitude = 0.1 * math.log(s) + 1.0
        out.append(t)
    return np.array(out, np.float64), magnitude


def rotate(x, positions, theta, factor, layout, transposed=False):
    """(result, sum of magnitudes of each value's two terms); x [tokens, heads, dim] float64."""
    n = len(theta)
    angle = np.asarray(positions, np.float64)[:, None, None] * theta
    c, s = np.cos(angle) * factor, np.sin(angle) * factor
    if transposed:
        s = -s
    lo, hi = (np.arange(n), np.arange(n) + n) if layout == "half" else (2 * np.arange(n), 2 * np.arange(n) + 1)
    y, mag = x.copy(), np.abs(x)
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    mag[..., lo] = mag[..., hi] = (np.abs(a) + np.abs(b)) * factor
    return y, mag


def rotation_bound(y, mag, rot, dtype):
    bound = HALF_STEP[dtype] * np.abs(y) + 8 * E * mag + (2.0 ** -25 if dtype == "float16" else 1e-42)
    bound[..., rot:] = 0.0
    return bound


def attention(q, kc, vc, prefix_pages, prefix_len, table, lens, scale, dtype):
    """(out, lse, bound of out, bound of lse) in 64 bits; caches [pages, page_size, kv_heads, dim], read only where a
    query sees them."""
    B, new, H, D = q.shape
    page, kv = kc.shape[1], kc.shape[2]
    u = HALF_STEP[dtype]
    out, lse = np.zeros((B, new, H, D)), np.full((B, new, H), -np.inf)
    bo, bl = np.zeros((B, new, H, D)), np.zeros((B, new, H))
    g = H // kv
    pj = np.arange(prefix_len)
    pk, pv = kc[prefix_pages[pj // page], pj % page], vc[prefix_pages[pj // page], pj % page]
    for b in range(B):
        sj = np.arange(max(0, lens[b]))
        rows = table[b][sj // page], sj % page
        k, v = np.concatenate([pk, kc[rows]]), np.concatenate([pv, vc[rows]])
        for i in range(new):
            n = prefix_len + max(0, lens[b] - (new - 1 - i))
            if n == 0:
                continue
            for h in range(kv):
                x = q[b, i, h * g:(h + 1) * g]
                s = (x @ k[:n, h].T) * scale
                ds = (D + 4) * E * abs(scale) * (np.abs(x) @ np.abs(k[:n, h]).T).max(-1) + 4 * E * np.abs(s).max(-1)
                m = s.max(-1, keepdims=True)
                p = np.exp(s - m)
                total = p.sum(-1, keepdims=True)
                at = (b, i, slice(h * g, (h + 1) * g))
                out[at] = p @ v[:n, h] / total
                lse[at] = (m + np.log(total))[:, 0]
                mean = p @ np.abs(v[:n, h]) / total
                bo[at] = (u + 4 * ds[:, None] + 64 * E) * mean + u * np.abs(out[at])
                if dtype == "float16":
                    bo[at] += 2.0 ** -24 * (1 + np.abs(v[:n, h]).sum(0) / total)
                bl[at] = 2 * ds + 16 * E * (1 + np.abs(lse[at]))
    return out, lse, bo, bl
