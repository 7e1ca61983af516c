"""CPU oracle of attention over selected blocks (include/ssa_sparse.h), of the block
tables kept from lengths (include/ssa_pages.h) and of the rotary forms
(ssa_rope_append_as, ssa_rope_table_scaled in include/ssa_layer.h).

TEST INFRASTRUCTURE ONLY: imported by ``tests/``, never by the library.  Plain numpy
in float64 over one request, row and kv head at a time; it imports nothing from the
library package.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def _f64(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(
        np.float64)


def _order(bits):
    """bf16 bits as integers in the order of their values: -0 below +0, NaN outermost."""
    x = np.asarray(bits, np.uint16).astype(np.int32)
    return np.where(x & 0x8000, -(x & 0x7FFF) - 1, x)


def cached(b, cache, i, h, n, values=False):
    """Bits [n, D] of request i's first n cached rows of kv head h."""
    t = np.arange(n)
    page, slot = b.block_table[i, t // PAGE], t % PAGE
    return cache[page, h, :, slot] if values else cache[page, h, slot]


def summary(b, k_cache, block):
    """{(page, head): [2, D] bits} of the blocks that hold new tokens of the batch."""
    out = {}
    for i in range(b.num_reqs):
        c, u = int(b.q_len[i]), int(b.ctx_len[i])
        if c == 0:
            continue
        for h in range(b.shape.hkv):
            k = cached(b, k_cache, i, h, u + c)
            for n in range(u // block, -(-(u + c) // block)):
                part = k[n * block:(n + 1) * block]
                key = _order(part)
                d = np.arange(part.shape[1])
                out[int(b.block_table[i, n * block // PAGE]), h] = np.stack(
                    [part[key.argmax(axis=0), d], part[key.argmin(axis=0), d]])
    return out


def bounds(q, high, low):
    """q [G, D], high and low [blocks, D] (float64): the highest bound over the heads, and
    the largest sum of the terms' magnitudes."""
    terms = (np.maximum(q, 0)[:, None] * high[None], np.minimum(q, 0)[:, None] * low[None])
    x = terms[0].sum(axis=2) + terms[1].sum(axis=2)
    size = (np.abs(terms[0]) + np.abs(terms[1])).sum(axis=2)
    return x.max(axis=0), size.max(axis=0)


def select(score, top, sink, recent):
    """Ascending blocks that a row of len(score) blocks looks at, -1 behind them."""
    n = len(score)
    out = np.full(top, -1, dtype=np.int32)
    if n <= top:
        out[:n] = np.arange(n)
        return out
    x = np.where(np.isnan(score), np.inf, score.astype(np.float64))
    middle = list(range(sink, n - recent))
    middle.sort(key=lambda t: (-x[t], t))
    out[:] = np.sort(np.concatenate([np.arange(sink), middle[:top - sink - recent],
                                     np.arange(n - recent, n)]))
    return out


def keys_of(blocks, block, pos):
    """The key indexes that a list names for a row at `pos`, as often as it does."""
    n = np.asarray(blocks, dtype=np.int64)
    n = n[(n >= 0) & (n <= pos // block)]
    t = (n[:, None] * block + np.arange(block)).reshape(-1)
    return t[t <= pos]


def attention(b, k_cache, v_cache, blocks, block):
    """out [T, Hq, D], sum of |w v| of each, and the largest sum of |scale q_i k_i|."""
    s = b.shape
    g = s.hq // s.hkv
    scale = float(np.float32(s.softmax_scale))
    out = np.zeros((b.num_tokens, s.hq, s.d))
    mass = np.zeros_like(out)
    most, row = 0.0, 0
    for i in range(b.num_reqs):
        c, u = int(b.q_len[i]), int(b.ctx_len[i])
        for h in range(s.hkv):
            k, v = (_f64(cached(b, p, i, h, u + c, values=p is v_cache)) for p in (k_cache, v_cache))
            for j in range(c):
                t = keys_of(blocks[row + j, h], block, u + j)
                if len(t) == 0:
                    continue
                q = _f64(b.q[row + j, h * g:(h + 1) * g])
                x = q @ k[t].T * scale
                w = np.exp(x - x.max(axis=1, keepdims=True))
                w /= w.sum(axis=1, keepdims=True)
                out[row + j, h * g:(h + 1) * g] = w @ v[t]
                mass[row + j, h * g:(h + 1) * g] = w @ np.abs(v[t])
                most = max(most, float((np.abs(q) @ np.abs(k[t]).T).max()) * scale)
        row += c
    return out, mass, most


def pages(table, ring, state, old, new, num_pages):
    """(table, ring, state, row_start, slots) after requests went from old to new tokens."""
    table, ring = table.copy(), ring.copy()
    head, count = int(state[0]), int(state[1])
    at, end = head, head + count
    row_start, slots = [0], []
    for i, (o, n) in enumerate(zip(old, new)):
        p, q = -(-int(o) // PAGE), -(-int(n) // PAGE)
        for k in range(p, q):
            table[i, k] = ring[at % num_pages]
            at += 1
        for k in range(q, p):
            ring[end % num_pages] = table[i, k]
            end += 1
        for t in range(int(o), int(n)):
            slots.append(int(table[i, t // PAGE]) * PAGE + t % PAGE)
        row_start.append(len(slots))
    return (table, ring, np.array([at % num_pages, end - at, 0, 0]), np.array(row_start),
            np.array(slots, dtype=np.int64))


def angles(d, base, kind="none", factor=1.0, trained=0, low=0.0, high=0.0):
    """Angle per position of each pair."""
    out = []
    for i in range(d // 2):
        t = base ** (-2 * i / d)
        if kind == "linear":
            t /= factor
        elif kind == "base":
            t = (base * factor ** (d / (d - 2))) ** (-2 * i / d)
        elif kind == "parts":
            turns = trained / (2 * math.pi / t)
            if turns <= low:
                t /= factor
            elif turns < high:
                w = (turns - low) / (high - low)
                t = (1 - w) * t / factor + w * t
        out.append(t)
    return np.array(out)


def rotate(x, cos, sin, layout, rotary):
    """x [rows, heads, D] float64; cos, sin [rows, rotary / 2]."""
    out = x.copy()
    for i in range(rotary // 2):
        a, b = (i, i + rotary // 2) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = cos[:, None, i], sin[:, None, i]
        out[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        out[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return out
