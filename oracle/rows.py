"""Rows that are no tree, in 64 bits: rotation and appending, causal attention under a window with first tokens that stay
visible, and sampling under filters.  Written from the definitions; numpy only."""
import math

import numpy as np

PAGE = 16


def bf16(bits):
    """bf16 bit patterns (uint16) -> float64."""
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def rope_frequencies(rotary_dim, theta, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0):
    out = []
    first = last = 0
    if scaling == "pairs":
        where = lambda turns: rotary_dim * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
        first, last = max(math.floor(where(high)), 0), min(math.ceil(where(low)), rotary_dim - 1)
    for i in range(rotary_dim // 2):
        f = theta ** (-2.0 * i / rotary_dim)
        if scaling == "none":
            w = 1.0
        elif scaling == "linear":
            w = 0.0
        elif scaling == "turns":
            w = min(max((original_len * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
        else:
            w = 1.0 - min(max((i - first) / max(last - first, 0.001), 0.0), 1.0)
        out.append(w * f + (1 - w) * f / factor)
    return np.array(out)


def turn(x, pos, freq, interleaved, amplitude=1.0):
    """x [n, heads, d] at positions pos [n] -> turned, in 64 bits."""
    y = np.array(x, np.float64)
    r = 2 * len(freq)
    a = np.asarray(pos, np.float64)[:, None] * freq
    c, s = np.cos(a)[:, None] * amplitude, np.sin(a)[:, None] * amplitude
    i, j = (np.arange(0, r, 2), np.arange(1, r, 2)) if interleaved else (np.arange(r // 2), np.arange(r // 2, r))
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def row_places(row_start, prefix):
    """[(row, request, position)] of all rows that belong to a request."""
    return [(r, b, int(prefix[b]) + r - int(row_start[b])) for b in range(len(prefix)) for r in range(int(row_start[b]), int(row_start[b + 1]))]


def gather(pool, table, length):
    """pool [pages, Hkv, 16, d], a request's table -> [Hkv, length, d]."""
    n = -(-length // PAGE)
    return np.concatenate([pool[p] for p in table[:n]], axis=1)[:, :length] if n else np.zeros((pool.shape[1], 0, pool.shape[3]))


def causal_attention(q, k_pool, v_pool, table, prefix, row_start, window, sinks, scale):
    """One layer: q [R, Hq, d], pools [pages, Hkv, 16, d], all float64 -> out [R, Hq, d], lse [R, Hq] (NaN where no row is)."""
    out, lse = np.full(q.shape, np.nan), np.full(q.shape[:2], np.nan)
    hkv = k_pool.shape[1]
    g = q.shape[1] // hkv
    for b in range(len(prefix)):
        r0, r1 = int(row_start[b]), int(row_start[b + 1])
        if r0 == r1:
            continue
        total = int(prefix[b]) + r1 - r0
        pos = np.arange(int(prefix[b]), total)[:, None]
        key = np.arange(total)[None]
        seen = key <= pos
        if window:
            seen &= (key > pos - window) | (key < sinks)
        used = seen.any(0)                                       # (what no row sees is not even read)
        pages = np.unique(np.nonzero(used)[0] // PAGE)
        keys = np.nonzero(used)[0]
        k = np.zeros((hkv, total, q.shape[2]))
        v = np.zeros_like(k)
        for p in pages:
            sl = slice(p * PAGE, min((p + 1) * PAGE, total))
            k[:, sl], v[:, sl] = k_pool[table[b, p]][:, :sl.stop - sl.start], v_pool[table[b, p]][:, :sl.stop - sl.start]
        for h in range(hkv):
            x = np.einsum("rgd,td->rgt", q[r0:r1, h * g:(h + 1) * g], k[h][keys]) * scale
            x = np.where(seen[:, None, keys], x, -np.inf)
            m = x.max(-1, keepdims=True)
            e = np.exp(x - m)
            s = e.sum(-1, keepdims=True)
            out[r0:r1, h * g:(h + 1) * g] = np.einsum("rgt,td->rgd", e / s, v[h][keys])
            lse[r0:r1, h * g:(h + 1) * g] = (m + np.log(s))[..., 0]
    return out, lse


def sample_row(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """-> (token, n_kept, kept ids by rank, their probabilities by rank)."""
    x = np.asarray(logits, np.float64)
    ids = np.nonzero(~np.isnan(x) & (x > -np.inf))[0]
    if not len(ids):
        return -1, 0, ids, np.zeros(0)
    ids = ids[np.lexsort((ids, -x[ids]))]
    if x[ids[0]] == np.inf:
        ids = ids[x[ids] == np.inf]
        z = np.zeros(len(ids))
    else:
        z = x[ids] - x[ids[0]]
    if not temperature > 0:
        return int(ids[0]), 1, ids[:1], np.ones(1)
    w = np.exp(z / temperature)
    n = len(ids)
    if 0 < top_k < len(x):
        n = min(n, top_k)
    before = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]])
    stays = np.ones(n, bool)
    if top_p < 1:
        stays &= before < top_p * w[:n].sum()
    if min_p > 0:
        stays &= w[:n] >= min_p
    n = max(1, int(stays.sum()))
    p = w[:n] / w[:n].sum()
    order = np.argsort(ids[:n])
    cdf = np.cumsum(p[order])
    at = min(int((cdf <= u * cdf[-1]).sum()), n - 1)
    while p[order][at] == 0.0:                                   # (what has no mass is never drawn)
        at -= 1
    return int(ids[:n][order][at]), n, ids[:n], p
