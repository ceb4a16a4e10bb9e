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


def tree_keys(mask, context, length, window):
    """Keys that a row with this mask (an int's bits) sees, in order: those before `context`, and context + j for bit j."""
    keys = [j for j in range(max(0, min(context, length)))]
    keys += [j for j in range(max(0, context), length) if mask >> (j - context) & 1]
    return np.array(keys[-window:] if window else keys, dtype=np.int64)


def tree_attention(q, k, v, masks, context, group, scale, window=0):
    """Rows q [n, q_heads, dim] with masks of the rows behind `context`; (out, mass) in 64 bits as in attention."""
    n, q_heads, dim = q.shape
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    out, mass = np.zeros((n, q_heads, dim)), np.zeros((n, q_heads, dim))
    for i in range(n):
        keys = tree_keys(masks[i], context, len(k), window)
        for h in range(q_heads if len(keys) else 0):
            s = scale * (k[keys, h // group] @ q[i, h])
            p = np.exp(s - np.max(s))
            p /= p.sum()
            out[i, h] = p @ v[keys, h // group]
            mass[i, h] = p @ np.abs(v[keys, h // group])
    return out, mass


def weights(q, k, length, group, scale, window=0):
    """[kv_heads, length]: the attention weight that rows q (the last n of `length` tokens) give each token, in 64 bits."""
    n, q_heads, _ = q.shape
    q, k = (np.asarray(t, dtype=np.float64) for t in (q, k))
    out = np.zeros((k.shape[1], length))
    for i in range(n):
        lo, hi = visible(length - n + i, length, window)
        for h in range(q_heads if lo < hi else 0):
            s = scale * (k[lo:hi, h // group] @ q[i, h])
            with np.errstate(all="ignore"):
                p = np.exp(s - np.max(s))
                out[h // group, lo:hi] += p / p.sum()
    return out


def evict(score, keep, recent):
    """Positions, in order, that one head keeps of the tokens with these scores."""
    n = len(score)
    if n <= keep:
        return list(range(n))
    early = n - recent
    order = sorted(range(early), key=lambda j: (-np.inf if np.isnan(score[j]) else float(score[j]), not np.isnan(score[j])),
                   reverse=True)  # stable: the earliest of equal ones
    return sorted(order[:keep - recent]) + list(range(early, n))


def verify_tree(p, x, parent, e):
    """(path, token) of one sequence: p [nodes, vocab], x and parent [nodes], e [levels, vocab], in 64 bits."""
    path, at = [], 0
    while True:
        token = int(np.argmax(np.asarray(p[at], dtype=np.float64) / np.asarray(e[len(path)], dtype=np.float64)))
        child = [i for i in range(1, len(x)) if parent[i] == at and x[i] == token]
        if not child or len(path) + 1 == len(e):
            return path, token
        at = child[0]
        path.append(at)
