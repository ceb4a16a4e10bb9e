"""The serving operators in 64 bits: a paged cache, attention over it, verification of drafts."""

import numpy as np

F16_MAX = 65504.0
I8_TOP = np.float32(127.0)


def quantize_i8(x):
    """(codes, scales) of vectors x [..., dim] fp32: s = fl(max|x| / 127), code = rint(fl(x / s)); the definition
    is in binary32, so the codes are exact."""
    x = np.asarray(x, dtype=np.float32)
    top = np.max(np.abs(x), axis=-1)
    with np.errstate(all="ignore"):
        scale = (top / I8_TOP).astype(np.float32)
        scale = np.where(np.isfinite(top), scale, np.float32(np.nan))
        code = np.clip(np.rint(x / scale[..., None]), -127, 127)
    code = np.where(scale[..., None] > 0, code, 0)
    return code.astype(np.int8), scale


def quantize_f16(x):
    return np.clip(np.asarray(x, dtype=np.float32), -F16_MAX, F16_MAX).astype(np.float16)


def visible(pos, length, window):
    """Keys [lo, hi) that a row at position pos of a sequence of `length` tokens sees."""
    hi = max(0, min(pos + 1, length))
    lo = max(0, pos + 1 - window) if window else 0
    return min(lo, hi), hi


def attention(q, k, v, length, group, scale, window=0):
    """Rows q [n, q_heads, dim] (the last n of `length` tokens), k, v [length, kv_heads, dim]; returns (out, mass) in 64
    bits, mass = sum_j p_j |v_j| (the size that the errors are relative to)."""
    n, q_heads, dim = q.shape
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    out, mass = np.zeros((n, q_heads, dim)), np.zeros((n, q_heads, dim))
    for i in range(n):
        lo, hi = visible(length - n + i, length, window)
        if lo == hi:
            continue
        for h in range(q_heads):
            s = scale * (k[lo:hi, h // group] @ q[i, h])
            with np.errstate(all="ignore"):
                p = np.exp(s - np.max(s))
                p /= p.sum()
            out[i, h] = p @ v[lo:hi, h // group]
            mass[i, h] = p @ np.abs(v[lo:hi, h // group])
    return out, mass


def verify(p, q, draft, u, e):
    """(accepted, token) of one sequence: p [k + 1, vocab], q [k, vocab], draft [k], u [k], e [vocab], in 64 bits."""
    p, q, u, e = (np.asarray(t, dtype=np.float64) for t in (p, q, u, e))
    k = len(draft)
    n = 0
    while n < k and 0 <= draft[n] < p.shape[1] and u[n] * q[n, draft[n]] < p[n, draft[n]]:
        n += 1
    w = p[n]
    if n < k:
        rest = np.maximum(p[n] - q[n], 0.0)
        w = rest if (rest > 0).any() else p[n]
    return n, int(np.argmax(w / e))
