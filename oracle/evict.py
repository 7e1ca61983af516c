"""CPU oracle of eviction by accumulated attention weight (include/ssa_evict.h).

TEST INFRASTRUCTURE ONLY: imported by ``tests/``, never by the library.  Plain
numpy in float64 over one request and kv head at a time; it imports nothing from
the library package.

* A key's score: decay times what it had (keys of earlier iterations only) plus the
  softmax weights that the counted new rows' query heads of its kv head give it.
  Row j of c, on u cached keys, sees keys 0 .. u + j; the last min(c, window) rows
  count (window 0: all).
* What stays of n keys: the first ``sink``, the last ``recent`` and, of the others,
  the highest scores, equal ones by index; NaN is -infinity.
* The move: kept key r takes the r-th slot of the request's new pages.
"""
from __future__ import annotations

import numpy as np

PAGE = 16


def _f64(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(
        np.float64)


def weights(q, k, u, scale):
    """q [c, G, D], k [u + c, D] (float64): softmax weights [c, G, u + c], zero for the
    keys that a row does not see (also where its others are NaN)."""
    s = np.einsum("cgd,td->cgt", q, k) * float(np.float32(scale))
    seen = np.arange(k.shape[0])[None, :] <= u + np.arange(q.shape[0])[:, None]
    s = np.where(seen[:, None, :], s, -np.inf)
    w = np.exp(s - s.max(axis=2, keepdims=True))
    return np.where(seen[:, None, :], w / w.sum(axis=2, keepdims=True), 0.0)


def key_scores(b, k_cache, window=0, old=None, decay=1.0):
    """New scores float64 [num_pages, Hkv, 16] of a batch whose keys are in k_cache
    (bits); slots that the operator leaves alone are NaN.  Also, per slot, the largest
    sum of |scale q_i k_i| over the counted (row, head) pairs of the request."""
    s = b.shape
    g = s.hq // s.hkv
    out = np.full((b.num_pages, s.hkv, PAGE), np.nan)
    size = np.zeros_like(out)
    row = 0
    for i in range(b.num_reqs):
        c, u = int(b.q_len[i]), int(b.ctx_len[i])
        if c == 0:
            continue
        t = np.arange(u + c)
        page, slot = b.block_table[i, t // PAGE], t % PAGE
        first = c - min(c, window) if window else 0
        for h in range(s.hkv):
            k = _f64(k_cache[page, h, slot])
            q = _f64(b.q[row:row + c, h * g:(h + 1) * g])
            w = weights(q, k, u, s.softmax_scale)[first:].sum(axis=(0, 1))
            if old is not None:
                w[:u] += decay * old[page[:u], h, slot[:u]]
            out[page, h, slot] = w
            size[page, h, slot] = s.softmax_scale * np.einsum(
                "cgd,td->cgt", np.abs(q[first:]), np.abs(k)).max()
        row += c
    return out, size


def select(score, kept, sink, recent):
    """Ascending indexes of the kept ones of score [n]."""
    n = len(score)
    if kept >= n:
        return np.arange(n, dtype=np.int32)
    x = np.where(np.isnan(score), -np.inf, score.astype(np.float64))
    middle = list(range(sink, n - recent))
    middle.sort(key=lambda t: (-x[t], t))
    return np.sort(np.concatenate([np.arange(sink), middle[:kept - sink - recent],
                                   np.arange(n - recent, n)])).astype(np.int32)


def compact(k_cache, v_cache, scores, block_table, new_table, lens, keeps):
    """Copies of the pools after the move; keeps[i][h]: kept indexes of request i."""
    k, v, s = k_cache.copy(), v_cache.copy(), scores.copy()
    for i, n in enumerate(lens):
        for h, keep in enumerate(keeps[i]):
            if len(keep) == n:
                continue
            for r, t in enumerate(keep):
                src, dst = block_table[i, t // PAGE], new_table[i, r // PAGE]
                k[dst, h, r % PAGE] = k_cache[src, h, t % PAGE]
                v[dst, h, :, r % PAGE] = v_cache[src, h, :, t % PAGE]
                s[dst, h, r % PAGE] = scores[src, h, t % PAGE]
    return k, v, s
