"""GPU parity of token sampling with the float64 oracle on masked rows and at the ends of its parameters (run with -m gpu).

Every call gets output tensors filled with another call's values, so that a row without an answer shows.
Tolerances: whole numbers equal; the log of the token's share as in test_gpu_sample.py (float64 sums of at most 2^20
weights, one rounding to float32): 2^-24 |lp| + 1e-9.  Numbers u next to 1 are used where the last entry that
counts holds at least 1e-9 of the kept mass: sums of 2^20 float64 terms are off by less than 2^20 2^-53 = 1.2e-10 of it,
so every order of summation draws that entry.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
LOWEST = {torch.float32: -3.402823466e+38, torch.bfloat16: -3.3895313892515355e+38, torch.float16: -65504.0}
ENDS = [0.0, 5e-324, 1e-300, 0.37, 1 - 2.0 ** -52, 1 - 2.0 ** -53]


@pytest.fixture(scope="module")
def imm():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    from paper_2602_22700_b200 import imm as binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def step():
    from oracle import step as o
    return o


def normal(n, seed, scale=1.0):
    return torch.randn(n, generator=torch.Generator().manual_seed(seed)) * scale


def numbers(values):
    return torch.tensor(values, dtype=torch.float64).cuda()


def run(imm, step, x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Rows x against the oracle; outputs begin as something that no row answers."""
    rows = x.shape[0]
    out = tuple(torch.full((rows,), 77, dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.int32, torch.int32))
    imm.sample(x, u, temperature, top_k, top_p, min_p, out=out)
    token, lp, kept, status = (t.cpu().numpy() for t in out)
    xs, us = x.cpu().double().numpy(), u.cpu().numpy()
    for i in range(rows):
        want = step.sample(xs[i], us[i], temperature, top_k, top_p, min_p)
        assert (int(token[i]), int(kept[i]), int(status[i])) == (want[0], want[2], want[3]), (i, us[i], token[i], kept[i], status[i], want)
        assert abs(lp[i] - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-9, (i, us[i], lp[i], want[1])


# ------------------------------------------------------------------ whole stretches masked

def stretches(n):
    """(first, end) of the entries that stay: the head, the middle, the tail masked, all but a few entries, every other stretch."""
    keep = torch.zeros((6, n), dtype=torch.bool)
    keep[0, n // 3:] = True
    keep[1, : n // 4] = True; keep[1, 3 * n // 4:] = True
    keep[2, : n // 2] = True
    keep[3, n // 2: n // 2 + 7] = True
    keep[4] = (torch.arange(n) // 3000) % 2 == 1
    keep[5, n - 5:] = True
    return keep


@pytest.mark.parametrize("n", [9001, 40003, 128256])
@pytest.mark.parametrize("dtype", DTYPES)
def test_stretches_masked_as_a_whole(imm, step, n, dtype):
    """Unfiltered, min-p alone, and a nucleus of thousands of entries, drawn from the ends of [0, 1)."""
    keep = stretches(n)
    for scale, filters in ((2.0, [(1.0, 0, 1.0, 0.0), (0.7, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.02)]), (0.2, [(1.0, 0, 0.9, 0.0), (1.0, 0, 0.999, 0.1)])):
        x = torch.full(keep.shape, -math.inf)
        for i in range(keep.shape[0]):
            row = normal(n, n + i, scale)
            last = int(keep[i].nonzero().max())
            row[last] = 1.5 * scale                          # the last kept entry counts
            x[i] = torch.where(keep[i], row, x[i])
        x = x.repeat_interleave(len(ENDS), 0).to(dtype).cuda()
        u = numbers(ENDS * keep.shape[0])
        for f in filters:
            run(imm, step, x, u, *f)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows_end_in_a_masked_tail(imm, step, dtype):
    """The largest numbers below 1, where sums in two orders may disagree on whether the last entry passes."""
    rows, n = 96, 20011
    for end in (n - 1, 12000, 4097):
        x = torch.full((rows, n), -math.inf)
        x[:, :end] = normal((rows, end), end, 2.0)
        x[:, end - 1] = 3.0
        u = numbers([1 - 2.0 ** -53, 1 - 2.0 ** -52] * (rows // 2))
        run(imm, step, x.to(dtype).cuda(), u)
        run(imm, step, x.to(dtype).cuda(), u, 1.0, 0, 1.0, 0.01)
        run(imm, step, (x * 0.1).to(dtype).cuda(), u, 1.0, 0, 0.95, 0.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_stretch_visited_but_not_kept(imm, step, dtype):
    """The first stretch is finite and low, but for the best entry that a nucleus of thousands leaves out."""
    n, head, p = 40003, 4096, 0.8
    x = normal(n, 11, 0.3).to(dtype)
    x[:head] = -40.0
    _, w = step.kept_prefix(x.double().numpy(), 1.0, 0, p, 0.0)
    order = np.argsort(-x.double().numpy(), kind="stable")
    out = int(order[len(w) + 20])                            # some places behind the border
    x[7] = x[out]
    rows = x.repeat(len(ENDS), 1).cuda()
    run(imm, step, rows, numbers(ENDS), 1.0, 0, p, 0.0)


# ------------------------------------------------------------------ masks that leave a few entries

@pytest.mark.parametrize("n,dtype", [(128256, torch.float32), (40003, torch.float32), (128256, torch.bfloat16), (40003, torch.float16)])
@pytest.mark.parametrize("value", [-5.0, -100.0, -1000.0, -60000.0, 200.0])
def test_a_few_entries_left(imm, step, n, dtype, value):
    """One to three finite entries anywhere in the row, so that no sample of it need see one."""
    g = torch.Generator().manual_seed(n)
    rows = 24
    x = torch.full((rows, n), -math.inf)
    for i in range(rows):
        at = torch.randint(n, (1 + i % 3,), generator=g)
        x[i, at] = value * (1 + torch.arange(len(at)) * 2.0 ** -6)
    x = x.to(dtype).cuda()
    u = torch.rand(rows, generator=g, dtype=torch.float64)
    u[:2] = 0.0
    for t in (0.01, 0.1, 1.0, 30.0):
        for f in ((0, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.3), (5, 0.9, 0.0), (1000, 1.0, 0.0)):
            run(imm, step, x, u.cuda(), t, *f)


# ------------------------------------------------------------------ the largest temperatures

@pytest.mark.parametrize("n", [700, 5003, 40003])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temperature", [1e36, 2e37, 3e38])
def test_temperatures_near_the_type_s_end(imm, step, n, dtype, temperature):
    """All entries weigh the same, masked ones and the ones behind the row's end nothing."""
    rows = 12
    x = normal((rows, n), n, 2.0)
    x[4:8, : n // 2] = -math.inf
    x[8:, n // 3:] = -math.inf
    x = x.to(dtype).cuda()
    u = torch.rand(rows, generator=torch.Generator().manual_seed(n), dtype=torch.float64)
    u[0], u[4], u[8] = 0.0, 0.0, 1 - 2.0 ** -53
    for f in ((0, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.5), (0, 0.3, 1.0), (50, 0.7, 0.0)):
        run(imm, step, x, u.cuda(), temperature, *f)


# ------------------------------------------------------------------ weights at the end of float64

@pytest.mark.parametrize("n", [90, 700, 9001, 40003])
@pytest.mark.parametrize("dtype", DTYPES)
def test_the_smallest_numbers_and_finite_masks(imm, step, n, dtype):
    """Entries masked by a finite value weigh exp((x - max) / T) in float64, zero where that vanishes: u = 0 draws the first
    entry with a weight, however small (e^-700 is one, e^-800 is none)."""
    masks = [LOWEST[dtype], -1e4, -800.0, -700.0]
    x = normal((len(masks), n), n, 1.0)
    x[:, n // 2] = 6.0
    for i, v in enumerate(masks):
        x[i, : n // 3] = v
        x[i, 2 * n // 3: n - 3] = v
    for i in range(len(masks)):                              # the row's maximum is 0: -700 is e^-700
        x[i] -= torch.where(x[i] > -100, 6.0, 0.0)
    us = [0.0, 5e-324, 1e-300, 1e-295, 1e-280, 0.5]
    rows = x.repeat_interleave(len(us), 0).to(dtype).cuda()
    u = numbers(us * len(masks))
    for f in ((1.0, 0, 1.0, 0.0), (1.0, 0, 0.99999, 0.0), (1.0, n - 5, 1.0, 0.0), (1.0, 0, 1.0, 1e-6)):
        run(imm, step, rows, u, *f)


def test_small_sums_before_a_large_entry(imm, step):
    """The running sum keeps entries of e^-50 in front of the maximum: u between two of their sums draws the entry between."""
    for n in (40, 200, 1100, 40003):
        x = torch.full((3, n), -math.inf)
        x[:, 8], x[:, 12], x[:, 13], x[:, 20] = -50.0, -50.5, 0.0, -1.0
        w = [math.exp(-50.0), math.exp(-50.5), 1.0, math.exp(-1.0)]
        u = numbers([0.5 * w[0] / sum(w), (w[0] + 0.5 * w[1]) / sum(w), 2 * w[0] / sum(w)])
        for f in ((1.0, 0, 1.0, 0.0), (1.0, 4, 1.0, 0.0)):
            run(imm, step, x.cuda(), u, *f)


# ------------------------------------------------------------------ entries of no weight behind the last one that counts

@pytest.mark.parametrize("n,top_k", [(60, 40), (120, 100), (700, 650), (1000, 1000), (9001, 1200), (9001, 3000), (40003, 30000), (9001, 0)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_the_last_entry_with_a_weight(imm, step, n, top_k, dtype):
    """Kept entries of no weight (a finite mask) at the end of the row are never drawn, whatever u is."""
    rows, live = 64, max(8, min(n, top_k or n) // 3)
    x = torch.full((rows, n), -9000.0)
    x[:, :live] = normal((rows, live), n + top_k, 2.0)
    x[:, live - 1] = 2.0
    x = x.to(dtype).cuda()
    u = numbers([1 - 2.0 ** -53, 1 - 2.0 ** -52, 0.0, 0.99] * (rows // 4))
    run(imm, step, x, u, 1.0, top_k, 1.0, 0.0)
    run(imm, step, x, u, 0.9, top_k, 0.99999, 0.0)


def test_a_sum_that_grows_by_many_entries_together(imm):
    """The last stretches weigh less than half a unit of the sum's last place each, and more together: an order of summation
    may draw from them or not, but an answer there is, and it is an entry with a weight."""
    n = 128256
    x = torch.full((n,), -math.inf)
    x[5], x[77] = 0.0, math.log(0.5)
    x[121 * 1024:] = math.log(0.6e-16 / 1024)
    us = [1 - 2.0 ** -53, 1 - 2.0 ** -52, 1 - 2.0 ** -51]
    for top_k, t in ((0, 1.0), (120000, 1.0)):
        out = tuple(torch.full((len(us),), 77, dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.int32, torch.int32))
        for rows in (x.repeat(len(us), 1), x.repeat(len(us), 1).bfloat16()):
            rows = rows.cuda()
            for i, u in enumerate(us):
                part = tuple(o[i:i + 1] for o in out)
                imm.sample(rows[i:i + 1], numbers([u]), t, top_k, out=part)
                assert int(part[3]) == 0 and int(part[2]) == n - 121 * 1024 + 2
                assert bool(rows[i, int(part[0])] > -math.inf) and -60.0 < float(part[1]) < 0.0


@pytest.mark.parametrize("n,dtype", [(12721, torch.float32), (40003, torch.bfloat16), (128256, torch.float16)])
def test_the_smallest_numbers_where_the_maximum_stands_alone(imm, step, n, dtype):
    """A few entries 640 above the bulk, at places that a sample of the row misses, and the head 300 below the bulk: e^-940 of the
    maximum is no weight, e^-640 is one."""
    g = torch.Generator().manual_seed(n)
    rows = 16
    x = torch.full((rows, n), -700.0)
    x[:, : n // 3] = -1000.0
    for i in range(rows):
        x[i, n // 2 + torch.randint(n // 2, (3,), generator=g)] = -60.0
    x = x.to(dtype).cuda()
    for us in ([0.0, 5e-324, 1e-300, 1e-285], [0.0, 0.3, 1e-265, 0.9]):
        for f in ((1.0, 0, 1.0, 0.0), (1.0, 0, 0.99999, 0.0), (1.0, 0, 1.0, 1e-6)):
            run(imm, step, x, numbers(us * (rows // 4)), *f)
