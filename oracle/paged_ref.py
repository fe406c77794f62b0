"""Plain reference of the operators over a paged key/value cache (test infrastructure: it imports nothing from the GPU package).

Pools are [pages, kv_heads, page, 128]; a sequence of S positions has its rows in the pages its table names, and its last n
positions are the tokens of the call.  Everything is numpy in fp64, position by position as the definitions read; results are
not rounded."""
import numpy as np

D = 128


def _f64(a):
    return np.asarray(a).astype(np.float64)


def rows_of(pool, table, length):
    """[kv_heads, length, 128]: the rows of one sequence."""
    page = pool.shape[2]
    out = np.empty((pool.shape[1], length, D), dtype=pool.dtype)
    for t in range(length):
        out[:, t] = pool[table[t // page], :, t % page]
    return out


def norm_rope(x, positions, table, gain=None, eps=1e-5):
    """x [tokens, 128 heads] -> fp64; table [positions, 64, 2] of (cos, sin)."""
    x = _f64(x).reshape(len(x), x.shape[1] // D, D)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * _f64(gain)
    c, s = (_f64(table)[positions][:, None, :, i] for i in (0, 1))
    y = np.empty_like(x)
    y[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    y[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return y.reshape(len(x), x.shape[1] * D)


def attention(q, keys, values, n, scale):
    """One sequence: q [n, 128 heads], keys and values [kv_heads, S, 128].  Returns (out, lse [n, heads], column sums
    [kv_heads, S], sum of p |V| as out, largest scale * sum |q| |K| of a pair)."""
    keys, values = _f64(keys), _f64(values)
    kv, S, _ = keys.shape
    heads = q.shape[1] // D
    q = _f64(q).reshape(n, heads, D)
    out, mass, lse = np.zeros_like(q), np.zeros_like(q), np.full((n, heads), -np.inf)
    sums, size = np.zeros((kv, S)), 0.0
    first = max(n - S, 0)  # tokens ahead of it see nothing
    if S == 0 or first >= n:
        return out.reshape(n, heads * D), lse, sums, mass.reshape(n, heads * D), size
    hidden = np.arange(S)[None, :] > S - n + np.arange(first, n)[:, None]
    for h in range(heads):
        g = h // (heads // kv)
        s = np.where(hidden, -np.inf, scale * (q[first:, h] @ keys[g].T))
        top = s.max(1, keepdims=True)
        e = np.exp(s - top)
        norm = e.sum(1, keepdims=True)
        lse[first:, h] = (top + np.log(norm))[:, 0]
        p = e / norm
        out[first:, h], mass[first:, h] = p @ values[g], p @ np.abs(values[g])
        sums[g] += p.sum(0)
        size = max(size, scale * (np.abs(q[first:, h]) @ np.abs(keys[g]).T).max())
    return out.reshape(n, heads * D), lse, sums, mass.reshape(n, heads * D), size


def evict(weights, keep, recent):
    """Positions of one head that stay, in order: the last `recent`, and of the others the largest weights (ties: the lower)."""
    S = len(weights)
    m = min(S, keep)
    recent = min(recent, m)
    old = list(range(S - recent))
    old.sort(key=lambda t: (0 if np.isnan(weights[t]) else 1, -weights[t] if not np.isnan(weights[t]) else 0.0, t))
    return np.array(sorted(old[:m - recent]) + list(range(S - recent, S)), dtype=np.int64)
