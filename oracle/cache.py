"""The operators over the paged cache and the logits in float64, from their definitions: rotary
frequencies and rotation, 8-bit quantisation with a power-of-two scale, attention of drafted tokens
under masks, log probabilities.  Nothing here is shared with the GPU path.
"""
from __future__ import annotations

import numpy as np

F64 = np.float64
E4M3_MAX = 448.0
MIN_EXP = -100


def rope_frequencies(rot, theta, factor=1.0, orig_ctx=0, alpha=1.0, beta=32.0):
    """Radians per position of each pair; linear or by-parts interpolation (arXiv 2309.00071, Eq. 18-20)."""
    f = np.asarray(theta, F64) ** (-2.0 * np.arange(rot // 2) / rot)
    if orig_ctx == 0:
        return f / factor
    turns = orig_ctx * f / (2 * np.pi)
    keep = np.clip((turns - alpha) / (beta - alpha), 0.0, 1.0)
    return (1 - keep) * f / factor + keep * f


def rotate(x, pos, rot, freq, interleaved=False, mscale=1.0):
    """The first ``rot`` dimensions of rows [n, heads, D] turned by pos * freq."""
    y = np.array(x, F64)
    if rot == 0:
        return y
    ang = np.asarray(pos, F64)[:, None] * freq
    c, s = np.cos(ang)[:, None] * mscale, np.sin(ang)[:, None] * mscale
    a = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    b = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    ya, yb = y[..., a].copy(), y[..., b].copy()
    y[..., a] = ya * c - yb * s
    y[..., b] = yb * c + ya * s
    return y


def e4m3_round(x):
    """Nearest e4m3 number (ties to even) of values of at most 448 in magnitude."""
    x = np.asarray(x, F64)
    _, e = np.frexp(x)                                   # |x| = m 2^e, 1/2 <= m < 1
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)      # 3 mantissa bits, subnormals below 2^-6
    return np.rint(x / step) * step


def quantise(x):
    """(values an 8-bit cache stands for, exponents) of rows [..., D]; NaN and infinities become NaN.  Values are
    float32, so with the largest exponent, 120, a number is at most 240 (256 2^120 is beyond their range)."""
    x = np.asarray(x, F64)
    fine = np.isfinite(x)
    amax = np.where(fine, np.abs(x), 0.0).max(-1)
    m, e = np.frexp(amax)                                # 448 = 7/8 2^9
    e = np.where(m > 0.875, e - 8, e - 9)
    e = np.where(amax > 0, np.maximum(e, MIN_EXP), MIN_EXP)
    scale = np.ldexp(1.0, e)[..., None]
    most = np.where(e >= 120, 240.0, E4M3_MAX)[..., None]
    return np.where(fine, np.clip(e4m3_round(np.where(fine, x, 0.0) / scale), -most, most) * scale, np.nan), e


def tree_attention(q, k, v, ctx, mask, scale):
    """q [n, n_q, D]; k, v [ctx + n, n_kv, D]; mask: n whole numbers, bit i: the row sees token ctx + i.
    Returns (out [n, n_q, D], sum_t p_t |v_t| / sum_t p_t of each output)."""
    n, n_q, d = q.shape
    g = n_q // k.shape[1]
    out, size = np.zeros((n, n_q, d), F64), np.zeros((n, n_q, d), F64)
    for r in range(n):
        see = [t for t in range(k.shape[0]) if t < ctx or (int(mask[r]) >> (t - ctx)) & 1]
        if not see:
            continue
        kk, vv = np.asarray(k, F64)[see], np.asarray(v, F64)[see]
        for h in range(n_q):
            s = kk[:, h // g] @ np.asarray(q[r, h], F64) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h] = p @ vv[:, h // g]
            size[r, h] = p @ np.abs(vv[:, h // g])
    return out, size


def logprobs(x):
    """(log probabilities [rows, vocab], entropy [rows])."""
    x = np.asarray(x, F64)
    m = x.max(-1, keepdims=True)
    lp = x - m - np.log(np.exp(x - m).sum(-1, keepdims=True))
    p = np.exp(lp)
    return lp, -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(-1)


def top(x, k):
    """Ids of the k largest of each row, descending, equal ones by the lower id."""
    return np.argsort(-np.asarray(x, F64), axis=-1, kind="stable")[:, :k]
