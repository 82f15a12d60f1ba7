"""Pins of the step oracle (sampling, norm with int8 output, dispatch and combine) on hand-worked cases."""
import math

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def step():
    from oracle import step as o
    return o


def test_sample_filters_on_a_worked_row(step):
    # weights 1/2, 1/4, 1/8, 1/16, 1/16 of 16 in the order of indices 3, 0, 2, 1, 4 (1 and 4 equal)
    p = {3: 8, 0: 4, 2: 2, 1: 1, 4: 1}
    x = np.array([math.log(p[i]) for i in range(5)])
    keep = lambda **k: sorted(step.kept_prefix(x, 1.0, k.get("top_k", 0), k.get("top_p", 1.0), k.get("min_p", 0.0))[0])
    assert keep() == [0, 1, 2, 3, 4]
    assert keep(top_k=4) == [0, 1, 2, 3]                    # the tie goes to the lower index
    assert keep(top_p=0.74) == [0, 3] and keep(top_p=0.76) == [0, 2, 3] and keep(top_p=1e-6) == [3]
    assert keep(top_k=2, top_p=0.6) == [3] and keep(top_k=2, top_p=0.7) == [0, 3]      # of the first two's mass, 12
    assert keep(min_p=0.2) == [0, 2, 3] and keep(min_p=1.0) == [3]
    # cumulative in index order: 4, 5, 7, 15, 16 of 16
    for u, want in ((0.0, 0), (0.249, 0), (0.26, 1), (0.32, 2), (0.5, 3), (0.93, 3), (0.95, 4), (0.999, 4)):
        token, lp, kept, status = step.sample(x, u)
        assert (token, kept, status) == (want, 5, 0) and abs(lp - math.log(p[want] / 16)) < 1e-12
    assert step.sample(x, 0.9, temperature=0.0) == (3, 0.0, 1, 0)
    assert step.sample(x, 0.9, top_k=1)[:1] + step.sample(x, 0.9, top_k=1)[2:] == (3, 1, 0)
    hot = step.sample(x, 0.999, temperature=2.0)            # weights go to their square roots
    assert abs(hot[1] - math.log(1 / (math.sqrt(8) + 2 + math.sqrt(2) + 2))) < 1e-12
    x[3] = -math.inf
    assert step.sample(x, 0.6)[0] == 1 and step.sample(x, 0.7)[0] == 2 and step.sample(x, 0.6)[2] == 4      # 4, 5, 7, 8 of 8
    for bad in (dict(u=1.0), dict(u=-0.1), dict(u=math.nan), dict(u=0.5, temperature=-1.0), dict(u=0.5, top_p=0.0), dict(u=0.5, min_p=1.5)):
        assert step.sample(x, **bad)[3] == step.ERR
    assert step.sample(np.full(4, -math.inf), 0.5)[0] == -1
    assert step.sample(np.array([0.0, math.nan]), 0.5)[3] == step.ERR


def test_norm_on_worked_rows(step):
    q, s = step.rmsnorm_quant(np.array([[3.0, -4.0, 0.0]]), np.ones(3), 0.0)
    assert q.tolist() == [[95, -127, 0]] and abs(s[0, 0] - 4 / (127 * math.sqrt(25 / 3))) < 1e-15
    # 127 t / a = 0.5, 1.5, 2.5: half to even
    q, _ = step.rmsnorm_quant(np.array([[127.0, 0.5, 1.5, 2.5, -2.5]]), np.ones(5), 1e-6)
    assert q.tolist() == [[127, 0, 2, 2, -2]]
    q, s = step.rmsnorm_quant(np.zeros((1, 4)), np.ones(4), 0.0)
    assert q.tolist() == [[0] * 4] and s.tolist() == [[0.0]]
    q, s = step.rmsnorm_quant(np.array([[1.0, math.inf]]), np.ones(2), 1e-6)
    assert q.tolist() == [[0, 0]] and math.isnan(s[0, 0])
    # against the ordinary formula: q * scale is the normalised row to within half a step
    h = np.random.default_rng(0).normal(size=(3, 256)); w = np.random.default_rng(1).normal(size=256)
    want = torch.nn.functional.rms_norm(torch.from_numpy(h), (256,), torch.from_numpy(w), 1e-5).numpy()
    for group in (0, 128):
        q, s = step.rmsnorm_quant(h, w, 1e-5, group)
        wide = np.repeat(s, group or 256, axis=1)
        assert np.all(np.abs(q * wide - want) <= 0.5 * wide * (1 + 1e-9))


def test_dispatch_and_combine_on_a_worked_routing(step):
    expert = np.array([[2, 0], [0, -1], [2, 2], [1, 0]])
    offsets, position, source = step.dispatch(expert, 4)
    assert offsets.tolist() == [0, 3, 4, 7, 7] and source.tolist() == [1, 2, 7, 6, 0, 4, 5]
    assert position.tolist() == [[4, 0], [1, -1], [5, 6], [3, 2]]
    y = np.arange(7.0).reshape(7, 1)
    assert step.combine(y, position).ravel().tolist() == [4.0, 1.0, 11.0, 5.0]
    assert step.combine(y, position, np.array([[1, 2], [3, 4], [0, 1], [1, 1]]), np.full(7, 0.5)).ravel().tolist() == [2.0, 1.5, 3.0, 2.5]
