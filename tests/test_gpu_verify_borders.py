"""Verification of drafted tokens next to its borders, against the float64 oracle (run with -m gpu).

Taken tokens, answers and status are equal; every test's numbers stay further from the borders than the 1e-12 within which a
comparison may be answered either way, or lie on them exactly.  logprob: one float32 rounding of a float64 logarithm.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def imm():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    from paper_2602_22700_b200 import imm as binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def orc():
    from oracle import cache
    return cache


def offsets_of(rows):
    return torch.tensor(np.cumsum([0] + list(rows)), dtype=torch.int64)


def check(imm, orc, target, draft, tokens, offsets, u, temperature=1.0):
    """The call on host tensors against the oracle; returns its outputs."""
    got = [t.cpu() for t in imm.verify_draft(target.cuda(), None if draft is None else draft.cuda(), tokens.cuda(), offsets.cuda(), u.cuda(), temperature)]
    x, y = target.double().numpy(), None if draft is None else draft.double().numpy()
    at, tok, v = offsets.tolist(), tokens.tolist(), u.tolist()
    for b in range(len(at) - 1):
        want = orc.verify(x[at[b]:at[b + 1]], None if y is None else y[at[b] - b:at[b + 1] - b - 1], tok[at[b]:at[b + 1]], v[at[b]:at[b + 1]], temperature)
        mine = [t[b].item() for t in got]
        assert (mine[0], mine[1], mine[3]) == (want[0], want[1], want[3]), (b, mine, want)
        assert abs(mine[2] - want[2]) <= abs(want[2]) * 2.0 ** -24 + 1e-12, (b, mine, want)
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [4001, 12000, 50001])
@pytest.mark.parametrize("kind", ["bonus", "copied", "drafted"])
def test_the_largest_u_before_a_masked_tail(imm, orc, dtype, n, kind):
    """u just below 1 where what follows the last kept entry has no mass (filters leave such rows): the answer is that entry, which
    holds a good part of the mass."""
    requests, g = 48, torch.Generator().manual_seed(n)
    rows = requests * (1 if kind == "bonus" else 2)
    last = n // 3 - 1
    x = torch.randn((rows, n), generator=g)
    x[:, last] = math.log(n / 10)
    x[:, last + 1:] = -math.inf
    draft = torch.randn((requests, n), generator=g)
    draft[:, last] = -5.0
    tokens = torch.full((rows,), last + 7, dtype=torch.int32)                    # masked in the target: never taken
    u = torch.full((rows,), 0.5, dtype=torch.float64)
    offsets = offsets_of([rows // requests] * requests)
    u[offsets[1:] - 1] = 1.0 - 2.0 ** -53
    got = check(imm, orc, x.to(dtype), draft.to(dtype) if kind == "drafted" else None, tokens, offsets, u)
    assert got[0].tolist() == [0] * requests and got[1].tolist() == [last] * requests


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [2, 300, 5000])
def test_probabilities_below_the_smallest_float32(imm, orc, dtype, n):
    """Drafted tokens whose probabilities float32 does not hold: p(d) = e^-88, q(d) = e^-87 and numbers around their quotient; the
    same at a low temperature; copied tokens with numbers u around p(d)."""
    for temperature, p_gap, q_gap in ((1.0, 88.0, 87.0), (1.0, 91.0, 90.5), (0.125, 11.0, 10.875), (1.0, 240.0, 239.0)):
        us = [0.1, 0.3, 0.36, 0.37, 0.45, 0.6, 0.61, 0.9]
        rows = 2 * len(us)
        target, draft = torch.full((rows, n), -math.inf), torch.full((len(us), n), -math.inf)
        target[:, 0], target[:, 1], draft[:, 0], draft[:, 1] = 0.0, p_gap, 0.0, q_gap
        tokens, u = torch.zeros(rows, dtype=torch.int32), torch.full((rows,), 0.5, dtype=torch.float64)
        u[0::2] = torch.tensor(us, dtype=torch.float64)
        offsets = offsets_of([2] * len(us))
        got = check(imm, orc, target.to(dtype), draft.to(dtype), tokens, offsets, u, temperature)
        assert 0 < sum(got[0].tolist()) < len(us)
        u[0::2] = math.exp(-p_gap / temperature) * torch.tensor([1e-9, 0.1, 0.5, 0.999, 1.001, 2.0, 50.0, 1e9], dtype=torch.float64)
        got = check(imm, orc, target.to(dtype), None, tokens, offsets, u, temperature)
        assert got[0].tolist() == [1] * 4 + [0] * 4


@pytest.mark.parametrize("requests", [1, 3, 20, 60, 200])
@pytest.mark.parametrize("temperature", [0.1, 1.0])
@pytest.mark.parametrize("with_draft", [True, False])
def test_two_maxima_far_above_the_rest(imm, orc, requests, temperature, with_draft):
    """Two entries of about the same weight, anywhere in the row, 100 to 170 binary orders above the others: whatever part of the
    row each is summed with, both count."""
    n, rng = (128256 if requests < 60 else 20000), np.random.default_rng(requests)
    rows = 2 * requests
    target, draft = torch.zeros((rows, n)), torch.zeros((requests, n))
    tokens = torch.zeros(rows, dtype=torch.int32)
    places = rng.integers(0, n, (requests, 2))
    places[0] = 0, n * 12192 // 128256
    for r in range(requests):
        for x in (target[2 * r], target[2 * r + 1], draft[r]):
            top = temperature * math.log(2) * (126.3 if r == 0 else rng.uniform(100, 170))
            x[places[r, 0]], x[places[r, 1]] = top, top + temperature * rng.uniform(-2, 2)
        tokens[2 * r + 1] = int(places[r, 0])
    target[0, places[0, 1]] = target[0, places[0, 0]] + 0.5 * temperature         # (p = 0.3775 for the drafted one)
    u = torch.from_numpy(rng.uniform(0.0, 1.0, rows))
    u[0] = 0.7
    check(imm, orc, target, draft if with_draft else None, tokens, offsets_of([2] * requests), u, temperature)


def test_sums_whose_reference_lies_far_below_the_maximum(imm, orc):
    """Float32 sums against references 120 binary orders below their largest entries, which the roundings of all steps put off
    in one direction: u lies 2e-6 of itself beside p / q, more than float64 needs and less than these sums tell."""
    n, temperature, d = 128256, 1.5320754051208496, 2100
    p = [125.55919647216797, 126.97391510009766, -7.3632965087890625, -7.256195068359375, 61.290096282958984]
    q = [126.88074493408203, 127.91703033447266, -7.2881317138671875, -7.1419219970703125, 58.73971939086914]
    target, draft = torch.full((2, n), -60.0), torch.full((1, n), -60.0)
    for x, (h1, h2, r1, r2, top) in ((target[0], p), (draft[0], q)):
        x[0], x[16389], x[49157] = r1, r2, top                                     # what the parts of the row are summed against
        x[d], x[18484] = h1, h2
    tokens = torch.tensor([0, d], dtype=torch.int32)
    wide = [torch.softmax(x.double() / float(np.float32(temperature)), 0)[d].item() for x in (target[0], draft[0])]
    for beside in (2e-6, 1e-6, -1e-6, -2e-6):
        u = torch.tensor([wide[0] / wide[1] * (1.0 + beside), 0.3], dtype=torch.float64)
        got = check(imm, orc, target, draft, tokens, offsets_of([2]), u, temperature)
        assert got[0].tolist() == [int(beside < 0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("requests", [1, 5, 40])
@pytest.mark.parametrize("kept", ["scattered", "together"])
@pytest.mark.parametrize("with_draft", [True, False])
def test_filtered_rows(imm, orc, dtype, requests, kept, with_draft):
    """Filters leave 40 of many entries: most parts of a row have none.  Drafted tokens inside and outside what the target keeps."""
    n, rng = (128256 if requests < 40 else 30011), np.random.default_rng(requests)
    held = [(i % 4) + (requests == 1) for i in range(requests)]
    offsets, rows = offsets_of([k + 1 for k in held]), sum(held) + requests
    target, draft = torch.full((rows, n), -math.inf), torch.full((sum(held), n), -math.inf)
    tokens = torch.zeros(rows, dtype=torch.int32)
    at = 0
    for b in range(requests):
        for i in range(held[b] + 1):
            row = int(offsets[b]) + i
            places = rng.choice(n, 40, replace=False) if kept == "scattered" else int(rng.integers(0, n - 50)) + rng.choice(50, 40, replace=False)
            target[row, torch.from_numpy(places)] = torch.from_numpy(rng.normal(0, 2, 40)).float()
            if i < held[b]:
                others = np.where(rng.random(40) < 0.8, places, rng.integers(0, n, 40))
                draft[at, torch.from_numpy(others)] = torch.from_numpy(rng.normal(0, 2, 40)).float()
                tokens[row + 1] = int(rng.choice(others))
                at += 1
    u = torch.from_numpy(rng.random(rows))
    for temperature in (0.7, 0.0):
        check(imm, orc, target.to(dtype), draft.to(dtype) if with_draft else None, tokens, offsets, u, temperature)
