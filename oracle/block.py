"""The operators between a block's projections in 64 bits, from their definitions (numpy, one sequence, head or row at a time),
each with a bound on what a computation in single precision with one rounding to fp16 may be off by.

Steps of a rounding: fp16 2^-11 of the value (half a step; 2^-25 below its normal numbers), fp32 2^-24.
"""
from __future__ import annotations

import numpy as np

H, F, TINY = 2.0 ** -11, 2.0 ** -24, 2.0 ** -25


def attention(q, k, v, q_offsets, kv_starts, kv_lens, head_dim, scale, causal, untouched):
    """q [M, heads * d], k, v [rows, kv heads * d] (any float type); `untouched` [M, heads * d]: what rows of no sequence hold.
    Returns (out, bound), both float64."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    d = head_dim
    heads, kv_heads = q.shape[1] // d, k.shape[1] // d
    out, bound = np.array(untouched, dtype=np.float64), np.zeros(q.shape)
    for s in range(len(q_offsets) - 1):
        q0, n = q_offsets[s], q_offsets[s + 1] - q_offsets[s]
        k0, m = kv_starts[s], kv_lens[s]
        for h in range(heads):
            g = h // (heads // kv_heads)
            for i in range(n):
                seen = max(0, min(m, i + m - n + 1)) if causal else m
                at = (q0 + i, slice(h * d, h * d + d))
                if seen == 0:
                    out[at] = 0.0
                    continue
                x, keys, values = q[at], k[k0 : k0 + seen, g * d : g * d + d], v[k0 : k0 + seen, g * d : g * d + d]
                z = scale * (keys @ x)
                p = np.exp(z - z.max())
                p /= p.sum()
                out[at] = p @ values
                # Each score: d products summed in fp32, scaled, an exponent of powers of two (its argument and the exponential a few
                # steps): an error of e in a score is a factor 1 +- e, in the sum below the line as well.  Each probability is
                # rounded to fp16 for the product with v, times 2^7 of the largest at least (below fp16's normal numbers half a
                # step is 2^-25, 2^-32 of the largest).  The sums are fp32, a matrix instruction's 16 keys or a tile's 32 and more at a time.
                e = scale * (d + 4) * F * (np.abs(keys) @ np.abs(x)).max() + 8 * F * (np.abs(z).max() + 4)
                spread = p @ np.abs(values)
                bound[at] = H * np.abs(out[at]) + spread * (H + 2 * e + 2 * (seen / 16 + 64) * F) + 2.0 ** -32 * p.max() * np.abs(values).sum(0) + TINY
    return out, bound


def qk_norm_rope(x, gamma, eps, inv_freq, positions, head_dim, interleaved):
    """x [M, heads * d].  Returns (y, bound)."""
    d, rot = head_dim, 2 * len(inv_freq)
    y = np.asarray(x, dtype=np.float64).reshape(len(x), -1, d).copy()
    steps = 4 * F
    if gamma is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + float(np.float32(eps))) * np.asarray(gamma, dtype=np.float64)
        steps = (d / 2 + 12) * F      # the sum of d squares counts half through the root
    t = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)
    cs, sn = np.cos(t)[:, None], np.sin(t)[:, None]
    a = np.arange(rot // 2) * (2 if interleaved else 1)
    b = a + (1 if interleaved else rot // 2)
    y1, y2 = y[..., a], y[..., b]
    size = np.abs(y)
    size[..., a] = size[..., b] = np.abs(y1) + np.abs(y2)
    y[..., a], y[..., b] = y1 * cs - y2 * sn, y2 * cs + y1 * sn
    # cosine and sine: the angle's remainder rounded to fp32 (2 pi * 2^-25) and a few steps of their own; the angle itself is a
    # product in double, 2^-52 of it
    turn = 16 * F + 2.0 ** -52 * np.abs(t).max(initial=0.0) * 4
    bound = H * np.abs(y) + size * (steps + turn) + TINY
    return y.reshape(len(x), -1), bound.reshape(len(x), -1)


def lora_add(x, a, b, row_adapter, base, scales, ranks):
    """x [M, K], a [E, R, K], b [E, N, R], base [M, N].  Returns (out, bound)."""
    x, out = np.asarray(x, dtype=np.float64), np.array(base, dtype=np.float64)
    bound = np.zeros_like(out)
    k = x.shape[1]
    for m, e in enumerate(row_adapter):
        if not 0 <= e < len(a):
            continue
        r = ranks[e]
        ae, be = np.asarray(a[e][:r], dtype=np.float64), np.asarray(b[e][:, :r], dtype=np.float64)
        t = ae @ x[m]
        out[m] += scales[e] * (be @ t)
        # K products summed in fp32 (in any order), the inner product as two fp16 terms (the first to half a step or 2^-25 of a power of
        # two at the row's largest, the second likewise of 2^27 times what is left), R products summed in fp32, a factor and a sum
        size = np.abs(t)
        most = size.max(initial=0.0)
        inner = (k + 40) * F * (np.abs(ae) @ np.abs(x[m])) + H * H * size + np.minimum(H * size, 2.0 ** -35 * most) + 2.0 ** -51 * most
        outer = abs(scales[e]) * (np.abs(be) @ inner + (r + 8) * F * (np.abs(be) @ np.abs(t)))
        bound[m] = H * np.abs(out[m]) + outer + 2 * F * np.abs(out[m]) + TINY
    return out, bound
