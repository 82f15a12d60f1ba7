"""CPU oracle for the int8 cache of keys and values, the attention over it, and the verification of drafted tokens -- TEST
INFRASTRUCTURE ONLY.

Plain numpy in float64, straight from the definitions; it shares no code with the CUDA library.  Only the tests may
import it.  The paper fixes none of these operators (its Section 4.1 names attention among the continuous transformations, its
Algorithm 3 repeats discrete decisions from committed random numbers); these readings are this build's:

  * append: per page and head s' = max(s, float32(max |x| / 127)), s = 0 where the page begins with the new rows;
    q = round-half-even(x / s') clamped to -127..127, 0 for s' = 0; where s' > s, earlier entries become
    round-half-even(q s / s').  Rows that are not finite leave scale NaN and zeros.
  * attention: row i of a sequence stands at t = length - rows + i and sees s <= t with t - s < window or s < sinks.
  * verify: d_i is taken while u_i q_i(d_i) < p_i(d_i); then the lowest index at which the running sum of max(p - q, 0)
    passes u' times the whole.
"""
from __future__ import annotations

import math

import numpy as np

ERR = -1


def append(x, cache, scale, table, offsets, lengths):
    """One of keys and values: ``cache`` int8 [pages, heads, page, dim] and ``scale`` float32 [pages, heads], changed in place."""
    pages, heads, page, dim = cache.shape
    status = np.zeros(len(lengths), dtype=np.int32)
    for b, length in enumerate(int(v) for v in lengths):
        first, end = int(offsets[b]), int(offsets[b + 1])
        rows = end - first
        if first < 0 or rows < 0 or end > len(x) or length < rows or length > table.shape[1] * page:
            status[b] = ERR
            continue
        at = length - rows
        while at < length:
            stop = min(length, (at // page + 1) * page)
            number, slot = int(table[b, at // page]), at % page
            part = np.asarray(x[first + at - (length - rows):first + stop - (length - rows)], dtype=np.float64)
            if 0 <= number < pages:
                for h in range(heads):
                    new = part[:, h]
                    old = np.float32(scale[number, h]) if slot else np.float32(0)
                    if not np.isfinite(new).all() or np.isnan(old):
                        s = np.float32(np.nan)
                    else:
                        s = max(old, np.float32(np.abs(new).max() / 127.0))
                    if slot and s > old and old > 0:
                        cache[number, h, :slot] = np.rint(cache[number, h, :slot].astype(np.float64) * float(old) / float(s)).astype(np.int8)
                    q = np.clip(np.rint(new / float(s)), -127, 127) if s > 0 else np.zeros_like(new)
                    cache[number, h, slot:slot + len(new)] = q.astype(np.int8)
                    scale[number, h] = s
            else:
                status[b] = ERR
            at = stop
    return status


def attention(q, cache, table, offsets, lengths, scale, window=0, sinks=0):
    """(out, lse, largest sum |q k|, sum of weight * |v|) in float64; rows of no sequence are NaN."""
    k_cache, v_cache, k_scale, v_scale = (np.asarray(t) for t in cache)
    pages, kv_heads, page, dim = k_cache.shape
    tokens, heads, _ = q.shape
    group = heads // kv_heads
    out, lse = np.full((tokens, heads, dim), np.nan), np.full((tokens, heads), np.nan)
    reach, size = np.zeros((tokens, heads)), np.zeros((tokens, heads, dim))
    for b, length in enumerate(int(v) for v in lengths):
        rows = int(offsets[b + 1]) - int(offsets[b])
        for i in range(rows):
            row, t = int(offsets[b]) + i, length - rows + i
            if length < 0 or length > table.shape[1] * page:
                continue
            keys = np.arange(max(t + 1, 0))
            if window:
                keys = keys[(t - keys < window) | (keys < sinks)]
            if len(keys) == 0:
                out[row], lse[row] = 0.0, -math.inf
                continue
            number = table[b, keys // page]
            if (number < 0).any() or (number >= pages).any():
                continue
            for kv in range(kv_heads):
                ks, vs = k_scale[number, kv].astype(np.float64), v_scale[number, kv].astype(np.float64)
                if not (np.isfinite(ks).all() and np.isfinite(vs).all() and (ks >= 0).all() and (vs >= 0).all()):
                    continue
                k = k_cache[number, kv, keys % page].astype(np.float64) * ks[:, None]
                v = v_cache[number, kv, keys % page].astype(np.float64) * vs[:, None]
                for h in range(kv * group, (kv + 1) * group):
                    row_q = np.asarray(q[row, h], dtype=np.float64)
                    if not np.isfinite(row_q).all():
                        continue
                    x = scale * (k @ row_q)
                    top = x.max()
                    p = np.exp(x - top)
                    lse[row, h] = top + math.log(p.sum())
                    p /= p.sum()
                    out[row, h] = p @ v
                    reach[row, h] = scale * (np.abs(k) @ np.abs(row_q)).max()
                    size[row, h] = p @ np.abs(v)
    return out, lse, reach, size


def distribution(x, temperature):
    x = np.asarray(x, dtype=np.float64)
    if temperature == 0:
        p = np.zeros_like(x)
        p[int(np.argmax(x))] = 1.0
        return p
    gap = (x - x.max()) / temperature
    w = np.where(gap < -690.0, 0.0, np.exp(np.maximum(gap, -690.0)))
    return w / w.sum()


def verify(target, draft, tokens, u, temperature):
    """(accepted, token, logprob, status) of one request: k + 1 target rows, k draft rows (None: no distribution)."""
    target = np.asarray(target, dtype=np.float64)
    temperature, k, n = float(np.float32(temperature)), len(target) - 1, target.shape[1] if len(target) else 0
    none = (0, -1, math.nan, ERR)
    if k < 0 or not (0 <= temperature < math.inf) or not all(0.0 <= v < 1.0 for v in u) or not all(0 <= d < n for d in tokens[1:]):
        return none

    def usable(x):
        return not np.isnan(x).any() and x.max() > -math.inf and x.max() < math.inf

    for i in range(k + 1):
        if not usable(target[i]):
            return none
        p = distribution(target[i], temperature)
        if i == k:
            left = p
            break
        d = int(tokens[i + 1])
        q = np.zeros(n)
        q[d] = 1.0
        if draft is not None and temperature > 0:
            if not usable(np.asarray(draft[i], dtype=np.float64)):
                return none
            q = distribution(draft[i], temperature)
        if not u[i] * q[d] < p[d]:
            left = np.maximum(p - q, 0.0)
            break
    if left.sum() == 0:
        left = p
    reached = np.cumsum(left)
    passed = reached > u[k] * reached[-1]
    token = int(np.argmax(passed)) if passed.any() else int(np.flatnonzero(left)[-1])
    return i, token, math.log(p[token]), 0
