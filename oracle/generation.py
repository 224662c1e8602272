"""The paged cache, attention over it, and log-probabilities of tokens, from their definitions, in fp64 NumPy.

A cache is a dict: k, v [n_pages, n_kv_heads, page_size, head_dim] fp64 (the values that are held), page_table [batch, max_pages] int.
"""
import numpy as np


# ------------------------------------------------------------------ e4m3 with a power of two for each vector
def e4m3_values():
    """The 256 values of e4m3 by their code (4 bits of exponent with a bias of 7, 3 of mantissa; codes 127 and 255 are NaN)."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    x = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    x = np.where((code & 127) == 127, np.nan, x)
    return np.where(code >= 128, -x, x)


def quantise(x):
    """(codes uint8, exponents int) of vectors along the last axis: 2^-e x to the nearest of e4m3's values (ties to the even code), with the
    smallest e >= -110 that brings the largest finite magnitude within 448; e = 0 for zeros.  What is not finite becomes NaN."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    amax = np.max(np.where(fine, np.abs(x), 0.0), axis=-1)
    with np.errstate(divide="ignore"):
        m, e = np.frexp(amax / 448.0)                # amax / 448 = m 2^e with m in [1/2, 1)
    e = np.where(amax == 0, 0, np.maximum(np.where(m == 0.5, e - 1, e), -110))
    y = np.where(fine, x, 0.0) * 2.0 ** -e[..., None]
    grid = e4m3_values()[:127]                        # 0 .. 448, ascending with the code
    top = np.where(e == 120, 240.0, 448.0)[..., None]  # 256 * 2^120 is outside the range of bf16
    a = np.minimum(np.abs(y), top)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(fine, code, 127) | np.where(np.signbit(np.where(np.isnan(x), 1.0, x)), 128, 0)
    return code.astype(np.uint8), e


def dequantise(code, e):
    return e4m3_values()[code] * 2.0 ** np.asarray(e, np.float64)[..., None]


# ------------------------------------------------------------------ the cache
def place(cache, b, p):
    """(page, slot) of position p of batch row b, or None."""
    size, table = cache["k"].shape[2], cache["page_table"]
    if p < 0 or p >= size * table.shape[1]:
        return None
    page = int(table[b, p // size])
    return (page, p % size) if 0 <= page < cache["k"].shape[0] else None


def rotate(x, p, base, layout):
    """A head's vector(s) [..., head_dim] rotated to position p."""
    dh = x.shape[-1]
    phi = float(p) * base ** (-2.0 * np.arange(dh // 2) / dh)
    c, s, y = np.cos(phi), np.sin(phi), np.empty_like(x)
    i, j = (np.arange(0, dh, 2), np.arange(1, dh, 2)) if layout else (np.arange(dh // 2), np.arange(dh // 2, dh))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def row_lengths(lengths, batch, seq):
    return [seq] * batch if lengths is None else [int(np.clip(n, 0, seq)) for n in lengths]


def row_starts(start, batch):
    return [0] * batch if start is None else [int(p) for p in start]


# ------------------------------------------------------------------ attention
def attention(cache, q, start, lengths, scale):
    """(o [batch, seq, heads, head_dim], lse [batch, heads, seq], sum of weight * |v| like o, largest sum of |q_d k_d| * scale over the keys a token
    sees [batch, heads, seq]): the last two are what errors are measured by."""
    b, s, hq, dh = q.shape
    hkv = cache["k"].shape[1]
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, big = np.full((b, hq, s), -np.inf), np.zeros((b, hq, s))
    for i, (a, n) in enumerate(zip(row_starts(start, b), row_lengths(lengths, b, s))):
        at = [(p, place(cache, i, p)) for p in range(0, max(0, a + n))]
        pos = np.array([p for p, x in at if x], dtype=np.int64)
        where = [x for _, x in at if x]
        if not where:
            continue
        pages, slots = np.array([x[0] for x in where]), np.array([x[1] for x in where])
        k, v = cache["k"][pages, :, slots], cache["v"][pages, :, slots]       # [keys, kv heads, head_dim]
        for t in range(n):
            seen = pos <= a + t
            if not seen.any():
                continue
            for h in range(hq):
                j = h // (hq // hkv)
                kk, vv = k[seen, j], v[seen, j]
                x = scale * (kk @ q[i, t, h])
                m = x.max()
                w = np.exp(x - m)
                lse[i, h, t] = m + np.log(w.sum())
                w = w / w.sum()
                o[i, t, h], mag[i, t, h] = w @ vv, w @ np.abs(vv)
                big[i, h, t] = scale * (np.abs(kk) @ np.abs(q[i, t, h])).max()
    return o, lse, mag, big


# ------------------------------------------------------------------ log-probabilities
def logprobs(logits, targets, inverse_temperature, n_top):
    """(logprobs, entropy, lse [T], top_ids, top_logprobs [T, n_top]); rows whose target is no token: 0, and ids -1.  targets None: every row counts."""
    z = np.asarray(logits, np.float64) * inverse_temperature
    T, V = z.shape
    chosen, entropy, lse = np.zeros(T), np.zeros(T), np.zeros(T)
    ids, tops = np.full((T, n_top), -1), np.zeros((T, n_top))
    for r in range(T):
        if targets is not None and not 0 <= targets[r] < V:
            continue
        m = z[r].max()
        if m == -np.inf:
            lse[r], logp = -np.inf, np.full(V, -np.inf)
        else:
            e = np.exp(z[r] - m)
            logp = (z[r] - m) - np.log(e.sum())
            lse[r] = m + np.log(e.sum())
            entropy[r] = -np.sum(np.where(e > 0, np.exp(logp) * np.where(e > 0, logp, 0.0), 0.0))
        if targets is not None:
            chosen[r] = logp[targets[r]]
        order = np.lexsort((np.arange(V), -z[r]))[:n_top]
        ids[r], tops[r] = order, logp[order]
    return chosen, entropy, lse, ids, tops


def logprobs_gradient(logits, targets, inverse_temperature, d_logprobs, d_entropy):
    """Gradient of sum d_logprobs * logprobs + d_entropy * entropy with respect to the logits (either weight None: 0)."""
    z = np.asarray(logits, np.float64) * inverse_temperature
    T, V = z.shape
    d = np.zeros((T, V))
    for r in range(T):
        if (targets is not None and not 0 <= targets[r] < V) or z[r].max() <= -1e30:    # not scored, or masked altogether
            continue
        e = np.exp(z[r] - z[r].max())
        p = e / e.sum()
        logp = (z[r] - z[r].max()) - np.log(e.sum())
        if d_logprobs is not None:
            d[r] -= p * d_logprobs[r]
            d[r, targets[r]] += d_logprobs[r]
        if d_entropy is not None:
            h = -np.sum(np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0))
            d[r] -= d_entropy[r] * np.where(p > 0, p * (np.where(p > 0, logp, 0.0) + h), 0.0)
    return d * inverse_temperature
