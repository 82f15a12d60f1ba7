"""CPU oracle for the steps of the audited execution between its products, and for the draw that ends a
step -- TEST INFRASTRUCTURE ONLY.

Plain numpy in float64, one row at a time, straight from the definitions; it shares no code with the CUDA
library.  Only the tests may import it.

What it follows.  The paper splits a step into continuous transformations and discrete decisions (Section
4.1); the checks of Algorithm 3 repeat the decisions from committed logits and committed random numbers.  The
paper does not fix the operators themselves; these readings are this build's:

  * sample: weights w = exp((x - max) / T).  Entries in the order (x descending, index ascending); top-k keeps
    the first k, top-p the shortest prefix of those that holds at least p of their mass, min-p of those the
    entries with w >= min_p, compared as x - max >= T log(min_p) (exp would round weights next to 1 to it).  The token is the lowest index at which the running sum of kept weights, in index
    order, passes u times their sum.  T = 0: the lowest index of the maximum.  -inf entries are never kept.
  * rmsnorm_quant: h = x + residual rounded to their type; t = h * weight; a = max |t| over the group;
    q = round-half-even(127 t / a), scale = a / (127 sqrt(mean h^2 + eps)); a = 0 gives zeros.
  * dispatch: the routed (token, slot) pairs sorted by (expert, pair number), stable.
  * combine: out[t] = sum_j weight[t, j] * row_scale[r] * y[r], r = position[t, j] >= 0.
"""
from __future__ import annotations

import math

import numpy as np

ERR = -1


def kept_prefix(x, temperature, top_k, top_p, min_p):
    """Indices that the filters keep, best first, and their weights (float64)."""
    x = np.asarray(x, dtype=np.float64)
    order = np.argsort(-x, kind="stable")                   # (x descending, index ascending); -inf last
    order = order[x[order] > -math.inf]
    if temperature == 0:
        return order[:1], np.ones(1)
    w = np.exp((x[order] - x[order[0]]) / float(temperature))
    if 0 < top_k < len(order):
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        reached = np.cumsum(w)
        held = int(np.argmax(reached >= float(top_p) * reached[-1])) + 1
        order, w = order[:held], w[:held]
    if min_p > 0:
        ok = x[order] - x[order[0]] >= float(temperature) * math.log(float(min_p))
        order, w = order[ok], w[ok]
    return order, w


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, kept, status) of one row; parameters as float32 / int32 values."""
    x = np.asarray(x, dtype=np.float64)
    temperature, top_p, min_p = (float(np.float32(v)) for v in (temperature, top_p, min_p))
    bad = np.isnan(x).any() or (x == math.inf).any() or not (x > -math.inf).any()
    bad = bad or not (0.0 <= u < 1.0) or not (0.0 <= temperature < math.inf) or not top_p > 0 or not 0.0 <= min_p <= 1.0
    if bad:
        return -1, math.nan, 0, ERR
    order, w = kept_prefix(x, temperature, top_k, top_p, min_p)
    back = np.argsort(order)
    order, w = order[back], w[back]
    reached = np.cumsum(w)
    passed = reached > u * reached[-1]
    at = int(np.argmax(passed)) if passed.any() else len(w) - 1
    return int(order[at]), math.log(w[at] / reached[-1]), len(w), 0


def rmsnorm_quant(h, weight, eps, group=0):
    """(q int8, scale float64) of the rows h (already the rounded sum of x and residual)."""
    h, weight = np.asarray(h, dtype=np.float64), np.asarray(weight, dtype=np.float64)
    rows, cols = h.shape
    width = group or cols
    q = np.zeros((rows, cols), dtype=np.int8)
    scale = np.zeros((rows, cols // width), dtype=np.float64)
    with np.errstate(all="ignore"):
        for i in range(rows):
            mean = float(np.mean(h[i] ** 2))
            for g in range(cols // width):
                part = slice(g * width, (g + 1) * width)
                t = h[i, part] * weight[part]
                a = float(np.max(np.abs(t)))
                if not math.isfinite(mean) or not math.isfinite(a):      # np.max returns NaN where one is
                    scale[i, g] = math.nan
                elif a > 0:
                    q[i, part] = np.rint(t * 127.0 / a).astype(np.int8)
                    scale[i, g] = a / (127.0 * math.sqrt(mean + eps)) if mean + eps > 0 else math.inf
    return q, scale


def dispatch(expert, experts):
    """(offsets, position, source pair of every output row) of an int array tokens x top."""
    flat = np.asarray(expert).reshape(-1)
    source = sorted((p for p in range(len(flat)) if 0 <= flat[p] < experts), key=lambda p: (flat[p], p))
    position = np.full(len(flat), -1, dtype=np.int32)
    for r, p in enumerate(source):
        position[p] = r
    offsets = np.cumsum([0] + [int((flat == e).sum()) for e in range(experts)])
    return offsets, position.reshape(np.asarray(expert).shape), np.array(source, dtype=np.int64)


def combine(y, position, weights=None, row_scale=None):
    y = np.asarray(y, dtype=np.float64)
    tokens, top = position.shape
    out = np.zeros((tokens, y.shape[1]))
    for t in range(tokens):
        for j in range(top):
            r = position[t, j]
            if 0 <= r < y.shape[0]:
                f = 1.0 if weights is None else float(weights[t, j])
                out[t] += f * (1.0 if row_scale is None else float(row_scale[r])) * y[r]
    return out
