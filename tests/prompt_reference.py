"""Plain forms in 64 bits of the operators of prompts, written from their formulas (numpy alone), and the bounds that their tests
hold the kernels to.

Bounds.  u is the half-step of the type relative to the value, e = 2^-24.  Forward as in serving_reference: a score of D products in 32
bits is off by ds = (D + 4) e scale sum |q k| + 4 e |s|, so with A = sum p |v| / sum p and n keys (sums in 32 bits: n e)
|out error| <= (u + 4 ds + (64 + n) e) A + u |out|, |lse error| <= 2 ds + (16 + n) e (1 + |lse|).

Backward, from the out and lse that the forward pass gave.  A weight p = exp(s - lse) is off by a factor of 1 +- w, w = ds + |lse error| +
8 e (1 + |lse| + max |s|), twice that to have its second order; rounded to the type for dv:
|dv error| <= sum p |dout| (u + 2 w + (64 + n) e) + u |dv|.
dp = dout . v is off by (D + 4) e sum |dout v|; e_i = dout . out by that of |dout out| and by sum |dout| |out error|; their
difference, call it t, by the sum r of these and 4 e |t|.  So ds = p t is off by p (2 w |t| + r (1 + 2 w)) and u p (|t| + r) for its rounding, and
|dq error| <= scale sum (that + (64 + n) e p |t|) |k| + u |dq|, dk likewise with q over the rows that see the key.
float16 has subnormal values: weights are held times 2^10, off by 2^-35; ds times a power of two that puts the largest |dout| between 1/2
and 1, off by 2^-25 of at most twice that; results by 2^-25.
"""
import numpy as np

from tests.serving_reference import E, HALF_STEP


def attention(q, k, v, scale, causal, dtype, dout=None, dlse=None):
    """One sequence: q [n, heads, dim] against k, v [m, kv_heads, dim], the last query beside the last key.  (out, lse) and their
    bounds; with dout also (dq, dk, dv) and theirs."""
    n, H, D = q.shape
    m, KV = k.shape[:2]
    g, u = H // KV, HALF_STEP[dtype]
    half = dtype == "float16"
    out, lse, bo, bl = np.zeros((n, H, D)), np.full((n, H), -np.inf), np.zeros((n, H, D)), np.zeros((n, H))
    grads = [np.zeros(x.shape) for x in (q, k, v)]
    bounds = [np.zeros(x.shape) for x in (q, k, v)]
    seen = np.arange(m)[None] <= np.arange(n)[:, None] + (m - n) if causal else np.ones((n, m), bool)
    some = seen.any(1)
    tiny = 2.0 ** -24 * np.abs(dout).max(initial=0.0) if half and dout is not None else 0.0
    for h in range(H):
        x, y, z = q[:, h], k[:, h // g], v[:, h // g]
        # (what is not seen may be infinite or NaN: it stays out of the sums)
        s = np.where(seen, np.einsum("id,jd->ij", x, y) * scale, -np.inf) if np.isfinite(y).all() else np.array(
            [[x[i] @ y[j] * scale if seen[i, j] else -np.inf for j in range(m)] for i in range(n)]).reshape(n, m)
        big = np.where(seen, (np.abs(x) @ np.abs(np.nan_to_num(y, posinf=0, neginf=0)).T), 0.0).max(1, initial=0.0)
        top = np.where(some, np.where(seen, s, -np.inf).max(1, initial=-np.inf), 0.0)
        most = np.where(seen, np.abs(np.where(seen, s, 0.0)), 0.0).max(1, initial=0.0)
        ds = (D + 4) * E * scale * big + 4 * E * most
        p = np.where(seen, np.exp(np.where(seen, s, 0.0) - top[:, None]), 0.0)
        total = np.where(some, p.sum(1), 1.0)[:, None]
        p = p / total
        z0 = np.where(np.isfinite(z), z, 0.0)
        out[:, h] = p @ z0
        lse[:, h] = np.where(some, top + np.log(total[:, 0]), -np.inf)
        mean = p @ np.abs(z0)
        bo[:, h] = (u + 4 * ds[:, None] + (64 + m) * E) * mean + u * np.abs(out[:, h])
        if half:
            bo[:, h] += 2.0 ** -24 * (1 + seen @ np.abs(z0) / total)
        size = 1 + np.abs(np.where(some, lse[:, h], 0.0))
        bl[:, h] = 2 * ds + (16 + m) * E * size
        if dout is None:
            continue
        d = dout[:, h]
        w = (2 * (ds + bl[:, h] + 8 * E * (size + most)))[:, None]
        dp = d @ z.T
        t = dp - (d * out[:, h]).sum(1, keepdims=True) + (0.0 if dlse is None else dlse[:, h:h + 1])
        r = (D + 4) * E * (np.abs(d) @ np.abs(z).T + (np.abs(d) * np.abs(out[:, h])).sum(1, keepdims=True)) + (
            np.abs(d) * bo[:, h]).sum(1, keepdims=True) + 4 * E * np.abs(t)
        off = p * (w * np.abs(t) + r * (1 + w)) + u * p * (np.abs(t) + r) + tiny * seen
        summed = p * np.abs(t)
        grads[0][:, h] += scale * (p * t) @ y
        grads[1][:, h // g] += scale * (p * t).T @ x
        grads[2][:, h // g] += p.T @ d
        bounds[0][:, h] += scale * (off + (64 + m) * E * summed) @ np.abs(y)
        bounds[1][:, h // g] += scale * (off + (64 + n * g) * E * summed).T @ np.abs(x)
        bounds[2][:, h // g] += (p * (u + w + (64 + n * g) * E) + (2.0 ** -35 if half else 0.0) * seen).T @ np.abs(d)
    bounds = [b + u * np.abs(x) + (2.0 ** -25 if half else 0.0) for b, x in zip(bounds, grads)]
    return (out, lse), (bo, bl), tuple(grads), tuple(bounds)


def packed(q, k, v, starts, scale, causal, dtype, dout=None, dlse=None):
    """The same over packed sequences: rows of none are 0, their lse -infinity."""
    T, H, D = q.shape
    res = [np.zeros(q.shape), np.full((T, H), -np.inf)], [np.zeros(q.shape), np.zeros((T, H))], [np.zeros(x.shape) for x in (q, k, v)], [
        np.zeros(x.shape) for x in (q, k, v)]
    for a, b in zip(starts[:-1], starts[1:]):
        got = attention(q[a:b], k[a:b], v[a:b], scale, causal, dtype, None if dout is None else dout[a:b],
                        None if dlse is None else dlse[a:b])
        for to, x in zip(res, got):
            for y, z in zip(to, x):
                y[a:b] = z
    return res
