"""What stands between a decoder block's linear layers and behind its head, in 64 bits and from the formulas: norms of queries and keys
with the position rotation (and gradients), norms around a block with its gate and the residual stream (and gradients), the 8-bit key/value cache, attention
over it, token log probabilities (and gradients), from logits or from final states.
numpy only, plain loops over blocks and sequences; nothing here is fast."""
import numpy as np

BLOCK = 32
EXP_MIN, EXP_MAX = -32, 120


# ---- norms and rotation --------------------------------------------------------------------------
def _partners(rot, interleaved):
    return (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2, rot))


def rotate(x, cos, sin, interleaved, back=False):
    """x [tokens, heads, D]; cos, sin [tokens, rot / 2]."""
    a, b = _partners(2 * cos.shape[1], interleaved)
    c, s = cos[:, None, :], (-sin if back else sin)[:, None, :]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def qk_norm_rope(x, w, eps, cos, sin, interleaved=False, norm=True):
    x = x.astype(np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else w.astype(np.float64))
    return rotate(x, cos.astype(np.float64), sin.astype(np.float64), interleaved)


def qk_norm_rope_bwd(x, w, eps, cos, sin, dout, interleaved=False, norm=True):
    """(gradient by x, gradient by w)"""
    x, g = x.astype(np.float64), rotate(dout.astype(np.float64), cos.astype(np.float64), sin.astype(np.float64), interleaved, back=True)
    if not norm:
        return g, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h, u = x * r, g * (1.0 if w is None else w.astype(np.float64))
    return r * (u - h * (u * h).mean(-1, keepdims=True)), (g * h).sum((0, 1))


# ---- norms around a block -------------------------------------------------------------------------
def _unit(v, eps, layer):
    """(normed rows, what they were multiplied by)"""
    v = v - v.mean(-1, keepdims=True) if layer else v
    r = 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    return v * r, r


def _one(w, otherwise):
    return otherwise if w is None else np.asarray(w, dtype=np.float64)


def block_norm(y, h, eps, layer=False, post=False, post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None, y_scale=1.0, h_scale=1.0):
    """(residual stream behind the block, next block's input); y or h may be None."""
    stream = h_scale * h.astype(np.float64) if h is not None else 0.0
    if y is not None:
        a = y.astype(np.float64)
        if post:
            a = _unit(a, eps, layer)[0] * _one(post_weight, 1.0) + _one(post_bias, 0.0)
        stream = stream + y_scale * _one(gate, 1.0) * a
    return stream, _unit(stream, eps, layer)[0] * _one(pre_weight, 1.0) + _one(pre_bias, 0.0)


def _unit_bwd(u, unit, r, layer):
    d = u - unit * (u * unit).mean(-1, keepdims=True)
    return r * (d - u.mean(-1, keepdims=True) if layer else d)


def block_norm_bwd(y, h, eps, gx, gh, layer=False, post=False, post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None, y_scale=1.0, h_scale=1.0):
    """Gradients by every input, as a dict; gx, gh: by the two outputs (None: 0)."""
    stream, _ = block_norm(y, h, eps, layer, post, post_weight, post_bias, gate, pre_weight, pre_bias, y_scale, h_scale)
    g, out = np.zeros_like(stream) if gh is None else gh.astype(np.float64), {}
    if gx is not None:
        gx = gx.astype(np.float64)
        unit, r = _unit(stream, eps, layer)
        out["pre_weight"], out["pre_bias"] = (gx * unit).sum(0), gx.sum(0)
        g = g + _unit_bwd(gx * _one(pre_weight, 1.0), unit, r, layer)
    out["h"] = h_scale * g
    if y is None:
        return out
    a = y.astype(np.float64)
    if post:
        unit, r = _unit(a, eps, layer)
        a = unit * _one(post_weight, 1.0) + _one(post_bias, 0.0)
    into = y_scale * g * a
    out["gate"] = into.sum(0) if gate is not None and gate.ndim == 1 else into
    g = y_scale * g * _one(gate, 1.0)
    if post:
        out["post_weight"], out["post_bias"] = (g * unit).sum(0), g.sum(0)
        g = _unit_bwd(g * _one(post_weight, 1.0), unit, r, layer)
    out["y"] = g
    return out


# ---- 8-bit cache -----------------------------------------------------------------------------------
def e4m3_values():
    """The 256 codes: sign, 4 bits of exponent (bias 7), 3 of fraction; no infinities, NaN where all seven lower bits are set."""
    out = np.empty(256)
    for b in range(256):
        e, f = (b >> 3) & 15, b & 7
        v = np.nan if b & 127 == 127 else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out[b] = -v if b & 128 else v
    return out


_POSITIVE = e4m3_values()[:127]


def e4m3_encode(x):
    """Nearest code, ties to the even one; |x| <= 448; NaN and infinities -> NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    d_lo, d_hi = a - _POSITIVE[lo], _POSITIVE[hi] - a
    up = (d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0))
    code = np.where(up, hi, lo)
    code = np.where(np.isfinite(x), code, 127)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def exponent(most):
    """Smallest e with most <= 448 * 2^e, within the limits."""
    e = EXP_MIN
    while e < EXP_MAX and most > 448 * 2.0 ** e:
        e += 1
    return e


def place(token, feature, values):
    """Byte of an element in its block."""
    if not values:
        return (feature // 32) * 1024 + token * 32 + feature % 32
    a, b, c, r = token >> 4, (token >> 3) & 1, (token >> 2) & 1, token & 3
    return feature * 32 + 16 * c + 8 * a + 4 * b + r


def places(D, values):
    t, f = np.meshgrid(np.arange(BLOCK), np.arange(D), indexing="ij")
    return place(t, f, values)


def _where(table, page_tokens, pages, sequence, position):
    at = position // page_tokens
    if at >= table.shape[1] or not 0 <= table[sequence, at] < pages:
        return None
    return table[sequence, at], position % page_tokens // BLOCK


def cache_write(codes, exps, values, table, lengths, token_start, new):
    """Writes new [tokens, heads, D] into codes [pages, heads, blocks, 32 D] (keys, or values) and exps, in place."""
    pages, heads, blocks, size = codes.shape
    D, table_of, off = size // BLOCK, e4m3_values(), places(size // BLOCK, values)
    for b in range(len(lengths)):
        n = int(token_start[b + 1] - token_start[b])
        had = int(lengths[b]) - n
        by_block = {}
        for i in range(n):
            if had + i >= 0:
                by_block.setdefault((had + i) // BLOCK, []).append(((had + i) % BLOCK, int(token_start[b]) + i))
        for j, tokens in by_block.items():
            at = _where(table, blocks * BLOCK, pages, b, j * BLOCK)
            if at is None:
                continue
            page, sub = at
            fresh = tokens[0][0] == 0
            for h in range(heads):
                x = np.stack([new[row, h] for _, row in tokens]).astype(np.float64)
                e = exponent(np.where(np.isfinite(x), np.abs(x), 0).max())
                block = np.zeros((BLOCK, D), dtype=np.uint8)
                if not fresh:
                    old = int(exps[page, h, sub]) - 127
                    e = max(e, old)
                    block = e4m3_encode(table_of[codes[page, h, sub][off]] * 2.0 ** (old - e))
                for (slot, _), v in zip(tokens, x):
                    block[slot] = e4m3_encode(v * 2.0 ** -e)
                codes[page, h, sub][off] = block
                exps[page, h, sub] = e + 127


def cache_dense(codes, exps, values, table, lengths, sequence):
    """([length, heads, D], [length] there) of a sequence."""
    pages, heads, blocks, size = codes.shape
    D, n, off, table_of = size // BLOCK, int(lengths[sequence]), places(size // BLOCK, values), e4m3_values()
    x, there = np.zeros((n, heads, D)), np.zeros(n, dtype=bool)
    for j in range((n + BLOCK - 1) // BLOCK):
        at = _where(table, blocks * BLOCK, pages, sequence, j * BLOCK)
        if at is None:
            continue
        page, sub = at
        m = min(BLOCK, n - j * BLOCK)
        for h in range(heads):
            x[j * BLOCK:j * BLOCK + m, h] = (table_of[codes[page, h, sub][off]] * 2.0 ** (int(exps[page, h, sub]) - 127))[:m]
        there[j * BLOCK:j * BLOCK + m] = True
    return x, there


# ---- attention ---------------------------------------------------------------------------------------
def attention(q, k, v, there, length, scale, causal, window):
    """One sequence: q [n, q_heads, D] stand at its last positions; k, v [length, kv_heads, D].
    -> out, lse, sum of p |v| (what roundings of the weights scale with)."""
    n, heads, D = q.shape
    group = heads // k.shape[1]
    out, size, lse = np.zeros((n, heads, D)), np.zeros((n, heads, D)), np.full((n, heads), -np.inf)
    keys = np.arange(length)
    for i in range(n):
        p = length - n + i
        see = there.copy()
        if causal:
            see &= keys <= p
        if window:
            see &= keys > p - window
        if not see.any():
            continue
        for h in range(heads):
            s = scale * (k[see, h // group] @ q[i, h].astype(np.float64))
            m = s.max()
            w = np.exp(s - m)
            lse[i, h] = m + np.log(w.sum())
            out[i, h] = (w / w.sum()) @ v[see, h // group]
            size[i, h] = (w / w.sum()) @ np.abs(v[see, h // group])
    return out, lse, size


# ---- log probabilities -----------------------------------------------------------------------------
def log_probs(x, scale=1.0):
    """log p of every row, -inf for a row of -inf alone."""
    with np.errstate(invalid="ignore", divide="ignore"):
        u = x.astype(np.float64) * scale
        m = u.max(-1, keepdims=True)
        nothing = m[:, 0] == -np.inf
        u = np.where(nothing[:, None], 0, u - np.where(nothing[:, None], 0, m))
        lp = u - np.log(np.exp(u).sum(-1, keepdims=True))
        lp[nothing] = -np.inf
    return lp


def entropy(lp):
    p = np.exp(lp)
    with np.errstate(invalid="ignore"):
        return -np.where(p == 0, 0, p * lp).sum(-1)


def alternatives(x, top):
    """Indices of the largest logits, ties to the lower index, NaN before everything."""
    key = np.where(np.isnan(x), np.inf, x.astype(np.float64))
    order = np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -key, ~np.isnan(x)), axis=-1)
    return order[:, :top]


def log_probs_grad(x, targets, g_logp, g_entropy, scale=1.0):
    lp = log_probs(x, scale)
    p = np.exp(lp)
    h = entropy(lp)[:, None]
    with np.errstate(invalid="ignore"):
        d = -g_entropy[:, None] * np.where(p == 0, 0, p * (lp + h))
    for r, t in enumerate(targets):
        if 0 <= t < x.shape[1]:
            d[r] -= g_logp[r] * p[r]
            d[r, t] += g_logp[r]
    d[np.isneginf(lp).all(-1)] = 0
    return d * scale
