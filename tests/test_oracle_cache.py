"""Pins of the oracle for the int8 cache, the attention over it and the verification of drafted tokens (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import cache as o


def test_append_rounds_and_rescales_by_hand():
    cache, scale = np.full((2, 1, 16, 16), 9, dtype=np.int8), np.full((2, 1), 5.0, dtype=np.float32)
    table = np.array([[1, 0]])
    x = np.zeros((2, 1, 16)); x[0, 0, 0] = 254.0; x[1, 0, 1] = -127.0; x[1, 0, 2] = 3.0
    assert o.append(x, cache, scale, table, [0, 2], [2]).tolist() == [0]           # a page that begins here: its old scale does not count
    assert scale[1, 0] == 2.0 and scale[0, 0] == 5.0
    assert cache[1, 0, 0, 0] == 127 and cache[1, 0, 1, 1] == -64 and cache[1, 0, 1, 2] == 2      # -63.5 and 1.5, half to even
    assert (cache[1, 0, 2:] == 9).all() and (cache[0] == 9).all()
    y = np.zeros((1, 1, 16)); y[0, 0, 0] = 508.0
    o.append(y, cache, scale, table, [0, 1], [3])                                   # the scale doubles: what is there halves
    assert scale[1, 0] == 4.0 and cache[1, 0, 0, 0] == 64 and cache[1, 0, 1, 1] == -32 and cache[1, 0, 2, 0] == 127
    y[0, 0, 0] = 4.0
    o.append(y, cache, scale, table, [0, 1], [2])                                   # cut back: written over, the scale stays
    assert scale[1, 0] == 4.0 and cache[1, 0, 1, 0] == 1 and cache[1, 0, 1, 1] == 0 and cache[1, 0, 2, 0] == 127
    y[0, 0, 0] = math.nan
    o.append(y, cache, scale, table, [0, 1], [17])
    assert math.isnan(scale[0, 0]) and (cache[0, 0, 0] == 0).all()
    assert o.append(y, cache, scale, table, [0, 1], [33]).tolist() == [o.ERR]
    assert o.append(y, cache, scale, np.array([[7, 0]]), [0, 1], [1]).tolist() == [o.ERR]


@pytest.mark.parametrize("window,sinks", [(0, 0), (5, 0), (5, 3), (1, 40)])
def test_attention_is_softmax_with_a_mask(window, sinks):
    rng = np.random.default_rng(1)
    cache = [rng.integers(-127, 128, (4, 2, 16, 16)).astype(np.int8) for _ in range(2)]
    scales = [rng.uniform(0.01, 0.1, (4, 2)).astype(np.float32) for _ in range(2)]
    table, length, rows = np.array([[2, 0, 3]]), 37, 6
    q = rng.normal(size=(rows, 4, 16))
    out, lse, _, _ = o.attention(q, cache + scales, table, [0, rows], [length], 0.3, window, sinks)
    k, v = (torch.from_numpy((c[table[0]].astype(np.float64) * s[table[0]][:, :, None, None]).transpose(1, 0, 2, 3).reshape(2, 48, 16)[:, :length])
            for c, s in zip(cache, scales))
    at, key = torch.arange(length - rows, length).view(-1, 1), torch.arange(length).view(1, -1)
    seen = key <= at
    if window:
        seen &= (at - key < window) | (key < sinks)
    for h in range(4):
        x = 0.3 * torch.from_numpy(q[:, h]) @ k[h // 2].T
        x[~seen] = -math.inf
        assert np.allclose(out[:, h], (torch.softmax(x, 1) @ v[h // 2]).numpy(), atol=1e-12)
        assert np.allclose(lse[:, h], torch.logsumexp(x, 1).numpy(), atol=1e-12)


def test_attention_rows_without_an_answer():
    cache = (np.ones((2, 1, 16, 16), np.int8), np.ones((2, 1, 16, 16), np.int8), np.ones((2, 1), np.float32), np.array([[1], [np.nan]], np.float32))
    q = np.ones((3, 1, 16))
    out, lse, _, _ = o.attention(q, cache, np.array([[0, 1]]), [0, 3], [2], 1.0)
    assert (out[0] == 0).all() and lse[0, 0] == -math.inf and (out[1:] == 1).all()              # a row in front of the first position
    out, lse, _, _ = o.attention(q, cache, np.array([[0, 1]]), [0, 3], [17], 1.0)
    assert (out[:2] == 1).all() and np.isnan(out[2]).all()                                      # only the last row sees the second page
    out, _, _, _ = o.attention(q, cache, np.array([[0, -1]]), [0, 3], [17], 1.0)
    assert (out[:2] == 1).all() and np.isnan(out[2]).all()


@pytest.mark.parametrize("with_draft", [True, False])
def test_taken_tokens_and_answers_have_the_targets_distribution(with_draft):
    """Over a grid of u and u', and all drafted tokens by their probability, the first token is distributed as the target's."""
    target = np.log(np.array([[0.5, 0.3, 0.2, 0.0], [0.25, 0.25, 0.25, 0.25]]) + 1e-300)
    draft = np.log(np.array([[0.2, 0.2, 0.1, 0.5]]))
    steps = 200
    grid = (np.arange(steps) + 0.5) / steps
    got = np.zeros(4)
    for d in range(4):
        weight = 0.0
        proposal = math.exp(draft[0, d]) if with_draft else 0.25
        for u in grid:
            for v in grid[::10]:
                a, token, _, status = o.verify(target, draft if with_draft else None, [0, d], [u, v], 1.0)
                assert status == 0
                first = d if a else token
                weight += 1
                got[first] += proposal / (steps * len(grid[::10]))
    if with_draft:
        assert np.allclose(got, [0.5, 0.3, 0.2, 0.0], atol=0.02)
    else:                                             # a proposal without a distribution is taken with p(d), else any other token
        p = np.array([0.5, 0.3, 0.2, 0.0])
        want = sum(0.25 * (p[d] * np.eye(4)[d] + (1 - p[d]) * (p * (np.arange(4) != d)) / max(1e-30, 1 - p[d])) for d in range(4))
        assert np.allclose(got, want, atol=0.02)


def test_verify_greedy_masks_and_refusals():
    t = np.array([[1.0, 3.0, 3.0], [-math.inf, 0.0, 1.0]])
    assert o.verify(t, None, [0, 1], [0.9, 0.5], 0.0)[:2] == (1, 2)
    assert o.verify(t, None, [0, 2], [0.0, 0.5], 0.0)[:2] == (0, 1)
    assert o.verify(t[::-1], t[:1], [0, 0], [0.0, 0.0], 1.0)[:2] == (0, 2)         # masked: never taken, nor drawn; p - q = (-0.06, -0.20, 0.26)
    assert o.verify(t, t[:1], [0, 1], [0.999, 0.0], 1.0)[:2] == (1, 1)             # p = q: always taken
    for bad in (dict(u=[1.0, 0]), dict(u=[0, -0.1]), dict(u=[0, math.nan]), dict(tokens=[0, 3]), dict(temperature=-1.0), dict(temperature=math.inf)):
        args = dict(target=t, draft=None, tokens=[0, 1], u=[0.5, 0.5], temperature=1.0)
        args.update(bad)
        assert o.verify(**args)[3] == o.ERR
    assert o.verify(np.full((1, 3), -math.inf), None, [0], [0.5], 1.0)[3] == o.ERR
    assert o.verify(np.array([[0.0, math.nan]]), None, [0], [0.5], 1.0)[3] == o.ERR
