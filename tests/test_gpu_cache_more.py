"""The int8 cache and the attention over it: limits, ends of the numbers, and sizes where the choice of a kernel changes (run with
-m gpu).  Inputs, oracle and tolerances are those of test_gpu_cache.py."""
import math

import numpy as np
import pytest
import torch

from test_gpu_cache import check_attention, host, i32, make_cache, make_table, offsets_of, randn, same

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


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.float16, 64)])
def test_rows_of_a_wait_that_ran_out_are_nan(imm, monkeypatch, dtype, dim):
    """Where a block's products end early and its other warps' waits run out, every row is what it is otherwise, or NaN throughout:
    items that end in other blocks, items that were still to come, rows that two groups of warps share.  Nothing stays as it was, and
    the next call is whole."""
    heads, kv_heads, rows, lengths = 16, 4, [900, 20, 70, 333, 1], [1500, 3000, 70, 400, 2000]
    table, pages = make_table(51, lengths, 64)
    cache, q = make_cache(52, pages, kv_heads, 64, dim), randn((sum(rows), heads, dim), 53, dtype, 1.5)
    offsets, lengths = offsets_of(rows), i32(lengths)
    want, ws = imm.kv_attention(q, cache, table, offsets, lengths), imm.kv_attention_workspace(q, cache, table, offsets)
    lib, lost = imm.lib(), []
    for cycles, steps in ((20000, 0), (20000, 1), (20000, 3), (20000, 8), (20000, 13), (20000, 21), (0, 30), (0, 1 << 30), (20000, 1 << 30)):
        out = (torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda"))
        ws.zero_()                             # (what an earlier call left there would hide a part that is missing)
        with monkeypatch.context() as m:
            m.setattr(lib, "imm_kv_attention", lambda desc, stream: lib.imm_kv_attention_limited(desc, cycles, steps, stream))
            imm.kv_attention(q, cache, table, offsets, lengths, out=out, workspace=ws)
        nan = out[1].isnan()
        assert torch.equal(out[0].isnan().all(2), nan) and torch.equal(out[0].isnan().any(2), nan)
        assert torch.equal(out[0][~nan], want[0][~nan]) and torch.equal(out[1][~nan], want[1][~nan])
        lost.append(int(nan.sum()))
    assert lost[0] == sum(rows) * heads and 0 < lost[4] < lost[0], lost
    again = imm.kv_attention(q, cache, table, offsets, lengths, workspace=ws)
    assert same(again[0], want[0]) and same(again[1], want[1])


# Scores carry the exponent of their page's value scale: up to 128 in size, so a rounding of one is 2^-18 of a binary order; four of
# them (the score, the maximum, their difference, the way back), 2^-16 ln(2) = 1.06e-5, beside what test_gpu_cache.py allows for.
CARRIED = 1.1e-5


def check_far(orc, q, cache, table, offsets, lengths, got):
    out, lse, reach, size = orc.attention(host(q), [host(t) for t in cache], host(table), host(offsets), host(lengths), 0.125)
    dim, n, dtype = q.shape[2], int(lengths.max()), q.dtype
    e_x = (4 * dim / 16 + 8) * 2.0 ** -23 * reach + 2.0 ** -22 + CARRIED
    assert np.all(np.abs(host(got[1]) - lse) <= e_x + (n / 64 + 16) * 2.0 ** -23 + np.abs(lse) * 2.0 ** -23)
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    largest = 127.0 * float(host(cache[3]).max())
    y = host(got[0])
    tol = (2 * e_x[..., None] + 2.0 ** -11 + (n / 8 + 64) * 2.0 ** -23) * size + n * 2.0 ** -31 * largest + half * np.abs(out) + 1e-30
    if dtype == torch.float16:
        tol, y, out = tol + 2.0 ** -25, np.clip(y, -65504, 65504), np.clip(out, -65504, 65504)
    assert np.all(np.abs(y - out) <= tol)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 3, 40])
@pytest.mark.parametrize("large,small", [(30, None), (60, None), (40, -95), (110, -20), (100, 30), (-60, None)])
def test_keys_count_however_far_their_value_scales_lie_apart(imm, orc, dtype, rows, large, small):
    """A few pages of values 2^large beside others of 2^small or 0: the others' keys are in the sum of the weights although their values
    do not show.  In any order of the pages, and where parts are joined."""
    dim, page, lengths = 64, 16, [1600, 200, 64]
    table, pages = make_table(61, lengths, page)
    cache = make_cache(62, pages, 1, page, dim)
    cache[2].fill_(0.002)
    q = randn((rows * 3, 2, dim), 63, dtype, 0.5)
    offsets, n = offsets_of([rows] * 3), i32(lengths)
    for places in ((0,), (99, 12, 3), (40, 41, 6, 1)):
        cache[3].fill_(0.0 if small is None else 2.0 ** small)
        for b in range(3):
            for p in places:
                if p < -(-lengths[b] // page):
                    cache[3][int(table[b, p])] = 1.5 * 2.0 ** large
        check_far(orc, q, cache, table, offsets, n, imm.kv_attention(q, cache, table, offsets, n, 0.125))


def check_scores(imm, orc, dtype, rows, size):
    """Scores around -size, all of them below 0, and around size, whose roundings are many binary orders where size is large."""
    dim, page, lengths = 64, 16, [100, 333, 40]
    table, pages = make_table(71, lengths, page)
    cache = make_cache(72, pages, 1, page, dim)
    cache[0].abs_().clamp_(min=50)
    q = randn((rows * 3, 2, dim), 73).abs() + 0.5
    cache[2].fill_(size / (0.125 * 127 * dim * 4.0))                               # (4: the largest entries of q)
    for sign in (-1.0, 1.0):
        check_attention(imm, orc, (sign * q).to(dtype), cache, table, offsets_of([rows] * 3), i32(lengths), 0.125)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 4, 40])
@pytest.mark.parametrize("size", [1e4, 3e5, 1e7, 1e8, 3e12, 1e29])
def test_scores_whose_roundings_are_large(imm, orc, dtype, rows, size):
    check_scores(imm, orc, dtype, rows, size)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 4, 40])
@pytest.mark.parametrize("size", [1e31, 3e37])
def test_scores_near_the_ends_of_float32(imm, orc, dtype, rows, size):
    check_scores(imm, orc, dtype, rows, size)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [48, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 20), (300, 200)])
def test_prompts_over_pages_of_128(imm, orc, dtype, dim, window, sinks):
    """Many rows per key where a page is a whole tile of keys, and ends inside one."""
    rows, lengths = [300, 129, 64, 1], [700, 130, 257, 128]
    table, pages = make_table(81, lengths, 128)
    cache = make_cache(82, pages, 2, 128, dim)
    q = randn((sum(rows), 8, dim), 83, dtype, 1.5)
    check_attention(imm, orc, q, cache, table, offsets_of(rows), i32(lengths), 0.1, window, sinks)


@pytest.mark.parametrize("batch", [1024, 1025, 1100])
@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 2)])
def test_many_rows_of_more_sequences_than_a_plan_holds(imm, orc, batch, window, sinks):
    """36 rows per key on average: up to 1024 sequences the tensor memory path, beyond it the other one."""
    rows = [9 + (i % 5) - 2 for i in range(batch)]
    lengths = [r + (i * 7) % 40 for i, r in enumerate(rows)]
    table, pages = make_table(84, lengths, 16)
    cache = make_cache(85, pages, 1, 16, 64)
    q = randn((sum(rows), 4, 64), 86, torch.bfloat16, 1.5)
    check_attention(imm, orc, q, cache, table, offsets_of(rows), i32(lengths), 0.125, window, sinks)


@pytest.mark.parametrize("heads,kv_heads,dim,rows", [(8, 8, 64, 1), (8, 1, 128, 1), (32, 8, 128, 4), (20, 1, 96, 1), (12, 2, 256, 5)])
def test_float16_weights_of_few_rows_have_two_terms(imm, orc, monkeypatch, heads, kv_heads, dim, rows):
    """Float16 rows where a key meets few of them: weights of 22 bits, like float32's."""
    import test_gpu_cache
    monkeypatch.setitem(test_gpu_cache.WEIGHT, torch.float16, 2.0 ** -22)
    lengths = [2000, 77, 512]
    table, pages = make_table(87, lengths, 32)
    cache = make_cache(88, pages, kv_heads, 32, dim, spread=0.1)
    q = randn((3 * rows, heads, dim), 89, torch.float16, 0.7)
    check_attention(imm, orc, q, cache, table, offsets_of([rows] * 3), i32(lengths), dim ** -0.5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 12, 40])
@pytest.mark.parametrize("size", [1e3, 1e7, 3e8, 3e9, 4.5e9, 6e9, 1e11])
def test_large_scores_over_far_value_scales(imm, orc, dtype, rows, size):
    """Scores whose roundings are large and rise with the position, where value scales lie far apart: every sum stays finite."""
    dim, page, lengths = 64, 16, [180, 350]
    table, pages = make_table(91, lengths, page)
    cache = make_cache(92, pages, 2, page, dim)
    cache[0].abs_().clamp_(min=50)
    q = (randn((rows * 2, 8, dim), 93).abs() + 0.5).to(dtype)
    cache[2].fill_(size / (0.125 * 127 * dim * 4.0))
    rise = torch.linspace(0.5, 1.0, max(len(table[0]), 1), device="cuda")
    g = torch.Generator().manual_seed(94)
    for b in range(2):
        for p in range(-(-lengths[b] // page)):
            cache[2][int(table[b, p])] *= rise[p]
    offsets, n = offsets_of([rows] * 2), i32(lengths)
    for _ in range(6):
        cache[3].copy_(torch.exp2(torch.round((torch.rand(cache[3].shape, generator=g) * 2 - 1) * 108)))
        cache[3][torch.rand(cache[3].shape, generator=g).cuda() < 0.3] = 0.0
        out, lse = imm.kv_attention(q, cache, table, offsets, n, 0.125)
        _, want, reach, _ = orc.attention(host(q), [host(t) for t in cache], host(table), host(offsets), host(n), 0.125)
        assert torch.isfinite(lse).all() and not out.isnan().any()
        e_x = (4 * dim / 16 + 8) * 2.0 ** -23 * reach + 2.0 ** -22 + CARRIED
        assert np.all(np.abs(host(lse) - want) <= e_x + 30 * 2.0 ** -23 + np.abs(want) * 2.0 ** -23)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 12, 40])
@pytest.mark.parametrize("size", [2e7, 4e7, 8e7, 1.6e8, 3.2e8])
def test_scores_a_few_rounding_steps_apart(imm, orc, dtype, rows, size):
    """Scores of +-size that differ by tens, where a rounding step is 2 to 32: no weight passes float16's range by the rounding of its
    limit."""
    dim, page, lengths = 64, 16, [300, 700]
    table, pages = make_table(95, lengths, page)
    cache = make_cache(96, pages, 2, page, dim)
    cache[0][..., 0] = 127
    scale = size / (0.125 * math.log2(math.e) * 127 * 60000)
    cache[2].fill_(scale)
    offsets, n, g = offsets_of([rows] * 2), i32(lengths), torch.Generator().manual_seed(97)
    for sign in (1.0, -1.0):
        q = torch.zeros((rows * 2, 8, dim))
        q[..., 0] = sign * 60000 * (1 - 0.02 * torch.rand(q.shape[:2], generator=g))
        q[..., 1] = (0.2 + torch.rand(q.shape[:2], generator=g)) * 30 / (0.125 * math.log2(math.e) * 127 * scale)
        q = q.to(dtype).cuda()
        out, lse = imm.kv_attention(q, cache, table, offsets, n, 0.125)
        _, want, reach, _ = orc.attention(host(q), [host(t) for t in cache], host(table), host(offsets), host(n), 0.125)
        assert torch.isfinite(lse).all() and torch.isfinite(out).all()
        e_x = (4 * dim / 16 + 8) * 2.0 ** -23 * reach + 2.0 ** -22
        assert np.all(np.abs(host(lse) - want) <= e_x + 30 * 2.0 ** -23 + np.abs(want) * 2.0 ** -23)
