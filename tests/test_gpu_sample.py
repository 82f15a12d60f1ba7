"""GPU parity of token sampling with the float64 oracle (run with -m gpu).

Tolerances.  The token, the number of kept entries and the status are whole numbers: equal.  The log of the
token's share is computed in float64 from sums of at most 2^20 float64 weights (relative error below 2^20 *
2^-53 < 2e-10) and rounded once to float32 (half a step, 2^-24 of its value): 2^-24 |lp| + 1e-9.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
LOWEST = {torch.float32: -3.402823466e+38, torch.bfloat16: -3.3895313892515355e+38, torch.float16: -65504.0}

# (temperature, top_k, top_p, min_p): each filter alone, together, and at its ends
FILTERS = [(1.0, 0, 1.0, 0.0), (0.8, 20, 0.95, 0.0), (1.0, 0, 0.9, 0.0), (0.7, 0, 1.0, 0.05), (1.3, 1000, 0.98, 0.01),
           (0.0, 5, 0.5, 0.5), (1.0, 1, 1.0, 0.0), (2.0, 0, 0.999, 0.0), (1.0, 700, 1.0, 0.0), (0.05, 0, 0.5, 0.0),
           (100.0, 0, 0.3, 0.0), (1.0, 64, 0.5, 0.2), (1.0, 0, 1e-6, 0.0), (1e-3, 0, 1.0, 1.0), (1e6, 50, 0.7, 0.9)]


@pytest.fixture(scope="module")
def imm():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    from paper_2602_22700_b200 import imm as binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def synth():
    from paper_2602_22700_b200 import synth as s
    return s


@pytest.fixture(scope="module")
def step():
    from oracle import step as o
    return o


def numbers(rows, seed):
    return torch.rand(rows, dtype=torch.float64, generator=torch.Generator().manual_seed(seed)).cuda()


def at(v, i):
    return v[i].item() if isinstance(v, torch.Tensor) else v


def check(step, got, x, u, temperature, top_k, top_p, min_p):
    token, lp, kept, status = (t.cpu().numpy() for t in got)
    xs, us = x.detach().cpu().double().numpy(), u.cpu().numpy()
    for i in range(xs.shape[0]):
        want = step.sample(xs[i], us[i], at(temperature, i), at(top_k, i), at(top_p, i), at(min_p, i))
        assert (int(token[i]), int(kept[i]), int(status[i])) == (want[0], want[2], want[3]), (i, token[i], kept[i], status[i], want)
        if math.isnan(want[1]):
            assert math.isnan(lp[i])
        else:
            assert abs(lp[i] - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-9, (i, lp[i], want[1])


def run(imm, step, x, u, f):
    check(step, imm.sample(x, u, temperature=f[0], top_k=f[1], top_p=f[2], min_p=f[3]), x, u, *f)


@pytest.mark.parametrize("rows,n", [(5, 1), (6, 2), (4, 7), (3, 31), (3, 512), (2, 1000), (3, 4099), (2, 16384), (3, 40003)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_matches_oracle(imm, step, synth, rows, n, dtype):
    """Rows of the logit generator (a grid of values: many ties) and of continuous values."""
    grid = synth.reference_logits(3, rows, n, device="cuda").to(dtype)
    smooth = (torch.randn((rows, n), generator=torch.Generator().manual_seed(n)) * 3).cuda().to(dtype)
    for k, f in enumerate(FILTERS):
        run(imm, step, grid, numbers(rows, 10 * n + k), f)
        run(imm, step, smooth, numbers(rows, 10 * n + k + 5), f)


@pytest.mark.parametrize("n,dtype", [(128256, torch.float32), (151936, torch.bfloat16), (300000, torch.float16), (500001, torch.float32),
                                     (1 << 20, torch.bfloat16), (1 << 20, torch.float32)])
def test_long_rows(imm, step, synth, n, dtype):
    """Whole vocabularies, the longest rows, and rows too long for shared memory."""
    x = synth.reference_logits(8, 2, n, device="cuda")
    x[1] = (torch.randn(n, generator=torch.Generator().manual_seed(n)) * 2).cuda()
    x = x.to(dtype)
    for k, f in enumerate(FILTERS):
        run(imm, step, x, numbers(2, n + k), f)


@pytest.mark.parametrize("n", [9, 700, 40003, 128256])
@pytest.mark.parametrize("dtype", DTYPES)
def test_masks_ties_and_extremes(imm, step, synth, n, dtype):
    g = torch.Generator().manual_seed(n)
    base = synth.reference_logits(4, 12, n, device="cuda")
    x = base.clone()
    many = (torch.rand(n, generator=g) < 0.9).cuda()
    x[0, many] = -math.inf                                   # most of the vocabulary masked
    x[0, n // 3] = 1.0
    x[1, many] = LOWEST[dtype]                               # ... by the type's lowest value
    x[1, n // 3] = 1.0
    x[2, :] = -math.inf                                      # nothing left
    x[3, :] = -math.inf; x[3, n - 1] = -5.0                  # one entry left
    x[4, :] = 2.5                                            # all equal
    x[5, :] = torch.where(many, 0.0, 1.0).cuda()             # two values
    x[6, :] = LOWEST[dtype]                                  # all at the lowest value
    x[7] = torch.where(many, -0.0, 0.0).cuda()               # both zeros are one value
    x[8] = base[8] * 1e-3                                    # nearly flat
    x[9] = base[9] * 300.0                                   # far apart
    x[10, many] = -1e4                                       # a finite mask far below
    x[11, : n // 2] = -math.inf                              # a whole half
    x = x.to(dtype)
    for k, f in enumerate(FILTERS):
        run(imm, step, x, numbers(12, 7 * n + k), f)


def test_exponentially_spread_values(imm, step):
    """Values over the whole range of float32, so that no linear cut separates them."""
    n = 20000
    e = torch.linspace(-126, 126, n, dtype=torch.float64)
    x = torch.stack([2.0 ** e, -(2.0 ** e), torch.where(torch.arange(n) % 2 == 0, 2.0 ** (e / 40), -(2.0 ** (e / 40)))])
    x = x[:, torch.randperm(n, generator=torch.Generator().manual_seed(1))].float().cuda()
    for k, f in enumerate(FILTERS + [(1e30, 0, 0.5, 0.0), (3e38, 6000, 0.9, 0.1), (1e-30, 0, 0.5, 0.0), (1e-40, 0, 0.9, 0.5)]):
        run(imm, step, x, numbers(3, k), f)


def test_numbers_at_the_ends(imm, step):
    n = 3001
    x = torch.randn((6, n), generator=torch.Generator().manual_seed(5)).cuda()
    u = torch.tensor([0.0, 5e-324, 0.5, 1 - 2.0 ** -53, 1 - 2.0 ** -24, 1e-17], dtype=torch.float64).cuda()
    for f in FILTERS:
        run(imm, step, x, u, f)


def test_rows_without_an_answer_say_so(imm, step):
    n = 5000
    x = torch.randn((8, n), generator=torch.Generator().manual_seed(6)).cuda()
    x[0, 17] = math.nan; x[1, n - 1] = math.inf; x[2] = -math.inf; x[3, 4000] = -math.nan
    u = numbers(8, 6)
    u[4] = 1.0; u[5] = -1e-9; u[6] = math.nan
    got = imm.sample(x, u, 0.9, 40, 0.9, 0.01)
    check(step, got, x, u, 0.9, 40, 0.9, 0.01)
    assert got[3].tolist() == [-1] * 7 + [0] and got[0].tolist()[:7] == [-1] * 7
    u = numbers(8, 7)
    bad = {"temperature": [-1.0, math.inf, math.nan], "top_p": [0.0, -0.5, math.nan], "min_p": [-0.1, 1.01, math.nan]}
    y = torch.randn((8, n), generator=torch.Generator().manual_seed(7)).cuda()
    for name, values in bad.items():
        for v in values:
            got = imm.sample(y, u, **{name: v})
            assert got[3].tolist() == [-1] * 8 and got[0].tolist() == [-1] * 8 and got[2].tolist() == [0] * 8
            assert bool(torch.isnan(got[1]).all())


@pytest.mark.parametrize("n", [300, 40003, 128256])
@pytest.mark.parametrize("dtype", DTYPES)
def test_parameters_of_every_row(imm, step, synth, n, dtype):
    rows = len(FILTERS)
    x = synth.reference_logits(12, rows, n, device="cuda").to(dtype)
    cols = list(zip(*FILTERS))
    t, p, m = (torch.tensor(cols[i], dtype=torch.float32, device="cuda") for i in (0, 2, 3))
    k = torch.tensor(cols[1], dtype=torch.int32, device="cuda")
    u = numbers(rows, n)
    check(step, imm.sample(x, u, t, k, p, m), x, u, t, k, p, m)
    check(step, imm.sample(x, u, t, 30, 0.9, m), x, u, t, 30, 0.9, m)


@pytest.mark.parametrize("offset,pad", [(0, 3), (1, 0), (3, 5), (7, 1), (8, 8)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_unaligned_rows(imm, step, dtype, offset, pad):
    """Rows at odd addresses; what lies around a row must not be taken for it."""
    rows, n = 4, 33001
    buf = torch.full((rows * (n + pad) + offset + 16,), 60.0, dtype=dtype, device="cuda")
    x = buf[offset:offset + rows * (n + pad)].view(rows, n + pad)[:, :n]
    x.copy_(torch.randn((rows, n), generator=torch.Generator().manual_seed(offset)) * 3)
    for k, f in enumerate(FILTERS[:6]):
        run(imm, step, x, numbers(rows, k), f)
    run(imm, step, x[:, 100:2000], numbers(rows, 77), FILTERS[1])
    run(imm, step, x[1:2], numbers(1, 78), FILTERS[2])


def test_same_row_same_answer_in_any_batch(imm):
    """A row's answer does not depend on the rows beside it."""
    n = 128256
    x = (torch.randn((64, n), generator=torch.Generator().manual_seed(3)) * 2.5).cuda()
    u = numbers(64, 3)
    for f in ((1.0, 0, 1.0, 0.0), (1.0, 0, 0.95, 0.0), (0.9, 50, 0.9, 0.02)):
        whole = imm.sample(x, u, *f)
        for i in (0, 13, 63):
            one = imm.sample(x[i:i + 1], u[i:i + 1], *f)
            assert [int(one[k]) for k in (0, 2, 3)] == [int(whole[k][i]) for k in (0, 2, 3)]
            assert abs(float(one[1]) - float(whole[1][i])) <= 2.0 ** -23 * abs(float(one[1]))


def test_many_short_rows(imm, step):
    x = torch.randn((3001, 65), generator=torch.Generator().manual_seed(9)).cuda()
    for f in FILTERS[:5]:
        run(imm, step, x, numbers(3001, 9), f)


def test_capture_replay_streams_and_buffers(imm, step, synth):
    """A captured call replayed on new inputs, a call on another stream, two at once; neighbours of the outputs stay."""
    n, rows, f = 40003, 6, (0.9, 50, 0.9, 0.01)
    x, u = synth.reference_logits(1, rows, n, device="cuda"), numbers(rows, 1)
    guard = [torch.full((rows + 2,), 7, dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.int32, torch.int32)]
    out = tuple(g[1:-1] for g in guard)
    imm.sample(x, u, *f, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        imm.sample(x, u, *f, out=out)
    for seed in (2, 3):
        x.copy_(synth.reference_logits(seed, rows, n, device="cuda")); u.copy_(numbers(rows, seed))
        graph.replay()
        check(step, out, x, u, *f)
    assert all(float(g[0]) == 7 and float(g[-1]) == 7 for g in guard)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    y, v = synth.reference_logits(4, rows, n, device="cuda"), numbers(rows, 4)
    torch.cuda.synchronize()
    with torch.cuda.stream(s1):
        a = imm.sample(x, u, *f)
    with torch.cuda.stream(s2):
        b = imm.sample(y, v, 1.0, 0, 0.95, 0.0)
    torch.cuda.synchronize()
    check(step, a, x, u, *f)
    check(step, b, y, v, 1.0, 0, 0.95, 0.0)


@pytest.mark.parametrize("n", [1023, 1025, 2047, 12000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_without_usable_bins(imm, step, dtype, n):
    """Spreads that a sample does not show: a cluster of equal maxima, two far clusters, far outliers, large values
    that lie close together, a list that ends inside ties."""
    g = torch.Generator().manual_seed(n)
    base = torch.randn((8, n), generator=g)
    base[0, ::7] = 9.0                                       # many equal maxima
    base[1, : n // 2] -= 500.0
    base[2, 5] = 1e4                                         # one far above
    base[3] = 3e4 + torch.round(base[3] * 8) * (32.0 if dtype == torch.float16 else 256.0)
    base[4] = torch.round(base[4])                           # a few values
    base[5] = torch.where(torch.rand(n, generator=g) < 0.5, -1e4, base[5])
    base[6, :40] += 20.0
    base[7] *= 0.01
    x = base.cuda().to(dtype)
    for k, f in enumerate(FILTERS + [(1.0, n // 2, 0.9, 0.0), (1.0, n - 1, 1.0, 0.0), (50.0, 0, 0.999, 0.0), (0.3, 1100, 0.9999, 1e-6)]):
        run(imm, step, x, numbers(8, 3 * n + k), f)


def test_no_rows(imm):
    got = imm.sample(torch.empty((0, 100), device="cuda"), torch.empty(0, dtype=torch.float64, device="cuda"))
    assert [t.numel() for t in got] == [0, 0, 0, 0]
