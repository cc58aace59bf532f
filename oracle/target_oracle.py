"""CPU oracle for the target's side of an iteration.  TEST INFRASTRUCTURE ONLY.

Plain numpy restatements in 64 bits, written from the definitions; shares no code with the CUDA library and is never imported by
the product path.

  chunk_rope       norm and rotary positions on several axes of a ragged chunk's heads
  chunk_places     (request, cache position) of every row of a ragged chunk
  chunk_attention  attention of a ragged chunk over the paged cache that holds its keys and values
  verify           how many drafted tokens stand, and the token behind them

What pins each function (tests/test_oracle_target.py):
  chunk_rope       position 0 leaves a head as it is, the rotation keeps every pair's length, one axis repeated on all axes is the
                   one-axis rotation, relative-position law on every axis
  chunk_attention  explicit Python loops, a window of one copies the row's own value, a chunk in one piece equals its rows one by one
  verify           the distribution of the first emitted token is the target's (enumerated over a grid of uniform numbers), greedy
                   requests copy the target's arg-max chain, p = q accepts everything
"""
import numpy as np


def chunk_places(cu_q, kv_lens):
    """[(request, cache position)] of rows 0 .. cu_q[-1] - 1."""
    out = []
    for b in range(len(kv_lens)):
        n = int(cu_q[b + 1]) - int(cu_q[b])
        out += [(b, int(kv_lens[b]) - n + i) for i in range(n)]
    return out


def chunk_rope(x, pos, pair_axis, theta, norm_w=None, eps=1e-6):
    """x [T, heads, dh], pos [axes, T], pair_axis [pairs] -> float64 [T, heads, dh]."""
    x = np.asarray(x, dtype=np.float64).copy()
    pairs = len(pair_axis)
    if norm_w is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(norm_w, dtype=np.float64)
    angle = np.stack([np.asarray(pos[a], dtype=np.float64) * float(theta) ** (-j / pairs) for j, a in enumerate(pair_axis)], axis=1)
    c, s = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :]
    a, b = x[..., :pairs].copy(), x[..., pairs:2 * pairs].copy()
    x[..., :pairs] = a * c - b * s
    x[..., pairs:2 * pairs] = b * c + a * s
    return x


def chunk_attention(q, k_pool, v_pool, table, cu_q, kv_lens, window=0, scale=None, pages=None):
    """q [T, Hq, dh], pools [pages, page, Hkv, dh] -> float64 [cu_q[-1], Hq, dh]; a page id outside the pools reads as zeros."""
    q = np.asarray(q, dtype=np.float64)
    n_pages, page, Hkv, dh = k_pool.shape
    rep = q.shape[1] // Hkv
    scale = dh ** -0.5 if scale is None else scale
    out = np.zeros((int(cu_q[-1]), q.shape[1], dh))
    for t, (b, p) in enumerate(chunk_places(cu_q, kv_lens)):
        lo = max(0, p - window + 1) if window else 0
        if p < lo:
            continue
        at = np.arange(lo, p + 1)
        ids = np.asarray(table)[b, at // page].astype(np.int64)
        ok = (ids >= 0) & (ids < n_pages)
        K = np.where(ok[:, None, None], k_pool[np.where(ok, ids, 0), at % page].astype(np.float64), 0.0)
        V = np.where(ok[:, None, None], v_pool[np.where(ok, ids, 0), at % page].astype(np.float64), 0.0)
        for h in range(q.shape[1]):
            z = K[:, h // rep] @ q[t, h] * scale
            e = np.exp(z - z.max())
            out[t, h] = (e / e.sum()) @ V[:, h // rep]
    return out


def _shares(z, temperature):
    """softmax(z / temperature); NaN counts as -infinity, +infinity as float32's largest; None where no token has any weight."""
    z = np.asarray(z, dtype=np.float64).copy()
    z[np.isnan(z)] = -np.inf
    z = np.minimum(z, float(np.finfo(np.float32).max))
    top = z.max()
    if top == -np.inf:
        return None
    if not temperature > 0:
        p = np.zeros_like(z)
        p[int(np.argmax(z))] = 1.0
        return p
    with np.errstate(invalid="ignore"):
        e = np.where(np.isneginf(z), 0.0, np.exp((z - top) / float(temperature)))
    return e / e.sum()


def verify(target, draft, ids, alpha, u, cu_q=None, vocab_map=None, temperature=None):
    """target [T, V], draft [B, k, Vd] or None, ids [B, k], alpha [B, k], u [B] -> (n_accept [B], tokens [B, k + 1])."""
    B, k = ids.shape
    V = target.shape[1]
    cu_q = np.arange(B + 1) * (k + 1) if cu_q is None else np.asarray(cu_q)
    temperature = np.ones(B) if temperature is None else np.asarray(temperature, dtype=np.float64)
    counts, tokens = np.zeros(B, dtype=np.int32), np.full((B, k + 1), -1, dtype=np.int32)
    for b in range(B):
        rows = int(cu_q[b + 1]) - int(cu_q[b])
        if rows < 1:
            continue
        n, rest = min(k, rows - 1), None
        for i in range(n):
            p, x = _shares(target[cu_q[b] + i], temperature[b]), int(ids[b, i])
            p = np.zeros(V) if p is None else p
            q = np.zeros(V)
            if draft is None or not temperature[b] > 0:
                if 0 <= x < V:
                    q[x] = 1.0
            else:
                d = _shares(draft[b, i], temperature[b])
                if d is not None:
                    q[np.arange(V) if vocab_map is None else np.asarray(vocab_map)] = d
            px, qx = (p[x], q[x]) if 0 <= x < V else (0.0, 1.0)
            if px > 0 and min(1.0, px / qx if qx > 0 else np.inf) >= float(alpha[b, i]):
                tokens[b, i] = x
                counts[b] += 1
                continue
            rest = p if not temperature[b] > 0 else np.maximum(0.0, p - q)
            if not rest.sum() > 0:
                rest = p
            break
        if rest is None:
            rest = _shares(target[cu_q[b] + n], temperature[b])
            rest = np.zeros(V) if rest is None else rest
        upto = np.cumsum(rest)
        if upto[-1] > 0:
            v = int(np.searchsorted(upto, float(u[b]) * upto[-1], side="right"))
            tokens[b, counts[b]] = min(v, int(np.flatnonzero(rest > 0)[-1]))
        else:
            tokens[b, counts[b]] = 0
    return counts, tokens
