"""Attention of one sequence in 64 bits, a head at a time: what oracle.decoder.attention says query by query."""
import numpy as np


def attention(q, k, v, there, length, scale, causal, window):
    """q [n, q_heads, D] at the last positions; k, v [length, kv_heads, D] -> out, lse, sum of p |v|.  NaN where a query sees one."""
    n, heads, D = q.shape
    group = heads // k.shape[1]
    at, pos = np.arange(length)[None, :], np.arange(length - n, length)[:, None]
    see = np.broadcast_to(there[None, :], (n, length)).copy()
    if causal:
        see &= at <= pos
    if window:
        see &= at > pos - window
    some = see.any(1)
    out, size, lse = np.zeros((n, heads, D)), np.zeros((n, heads, D)), np.full((n, heads), -np.inf)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for g in range(k.shape[1]):
            bad = see.astype(np.float64) @ np.isnan(v[:, g]).astype(np.float64) > 0
            values, keys = np.where(np.isnan(v[:, g]), 0.0, v[:, g]), k[:, g]
            for h in range(g * group, (g + 1) * group):
                x = np.where(see, scale * (q[:, h].astype(np.float64) @ keys.T), -np.inf)
                m = np.where(some, x.max(1, initial=-np.inf), 0.0)
                w = np.exp(x - m[:, None])
                total = w.sum(1)
                w = w / np.where(total == 0, 1.0, total)[:, None]
                lse[:, h] = m + np.log(total)
                nan = np.isnan(total)[:, None] | bad
                out[:, h] = np.where(nan, np.nan, np.nan_to_num(w) @ values)
                size[:, h] = np.nan_to_num(w) @ np.abs(values)
    return out, lse, size
