"""GPU parity of the int8 cache of keys and values and the attention over it with the float64 oracle (run with -m gpu).

Tolerances.  append: entries, scales and status are equal (a scale is one float32 division, an entry a float64 quotient
rounded to an integer).  Attention, per row: let R = scale * sum |q k| (the largest over the keys) and S = sum of weight * |v|.
  x = scale q k: products exact; at most 2 dim / 16 additions into a float32 sum that a matrix instruction may cut off instead of
  rounding, so 2^-23 of the magnitudes each, the same again inside an instruction; three factors, the subtraction of the
  maximum and its result's rounding: (4 dim / 16 + 8) 2^-23 R absolutely, plus 2^-22 for the exponential of 2: e_x.
  The logarithm of the sum: e_x + n / 64 additions of 2^-23 per lane, 16 for the reductions, and two half-steps of its own size.
  The output: e_x in the weights and in their sum (2 e_x), a weight's rounding (2^-11, in float32 2^-22), n / 16 cut-off
  additions of 2^-23 twice over, 64 for joins: relative to S.  Weights below float16's range: an absolute 2^-31 of the largest
  per key (2^-25 under the 2^6 that the largest is held at), relative to S at most n 2^-31 max |v| / S.  Then half a
  step of the output's type: of float16's smallest values that is 2^-25 absolutely, and what lies beyond its largest value
  (65504, and half a step of 32) rounds to infinity, so both sides are compared as clamped to 65504.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
WEIGHT = {torch.float32: 2.0 ** -22, torch.bfloat16: 2.0 ** -11, torch.float16: 2.0 ** -11}


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


def make_cache(seed, pages, heads, page, dim, spread=0.7):
    g = torch.Generator().manual_seed(seed)
    cache = [torch.randint(-127, 128, (pages, heads, page, dim), generator=g, dtype=torch.int8).cuda() for _ in range(2)]
    return tuple(cache + [(torch.exp(spread * torch.randn((pages, heads), generator=g)) * 0.02).cuda() for _ in range(2)])


def make_table(seed, lengths, page, width=None, shuffle=True):
    """A page table over pages of its own for every sequence, -1 where there is none; (table, pages)."""
    need = [-(-n // page) for n in lengths]
    order = np.random.default_rng(seed).permutation(sum(need) + 2) if shuffle else np.arange(sum(need) + 2)
    table = np.full((len(lengths), width or max(max(need), 1)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table).cuda(), sum(need) + 2


def offsets_of(rows):
    return torch.tensor(np.cumsum([0] + list(rows)), dtype=torch.int64).cuda()


def i32(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def randn(shape, seed, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).cuda().to(dtype)


def host(t):
    return t.cpu().double().numpy() if t.is_floating_point() else t.cpu().numpy()


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=123.0), torch.nan_to_num(b.float(), nan=123.0))


# ------------------------------------------------------------------ append


def check_append(imm, orc, k, v, cache, table, offsets, lengths):
    want = [host(cache[0]).copy(), host(cache[1]).copy(), cache[2].cpu().numpy().copy(), cache[3].cpu().numpy().copy()]
    status = orc.append(host(k), want[0], want[2], host(table), host(offsets), host(lengths))
    orc.append(host(v), want[1], want[3], host(table), host(offsets), host(lengths))
    got = imm.kv_append(k, v, cache, table, offsets, lengths)
    assert got.tolist() == status.tolist()
    for t, w in zip(cache, want):
        assert np.array_equal(t.cpu().numpy(), w, equal_nan=t.is_floating_point())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,dim,page", [(1, 16, 16), (2, 128, 16), (3, 80, 32), (8, 64, 64), (2, 256, 128)])
def test_append_matches_oracle(imm, orc, dtype, heads, dim, page):
    """Single tokens, rows that end inside a page, whole pages, empty sequences, rows behind the last sequence."""
    rows = [1, 0, 1, page, 3 * page + 5, 7, 1, 2]
    lengths = [1, 40, page, page, 3 * page + 5, page + 3, 2 * page + 1, page + 1]
    table, pages = make_table(dim, lengths, page)
    cache = make_cache(page, pages, heads, page, dim)
    tokens = sum(rows) + 3
    both = randn((tokens, 2 * heads, dim), 5, dtype) * torch.exp(randn((tokens, 2 * heads, 1), 6)).to(dtype) * 4
    check_append(imm, orc, both[:, :heads], both[:, heads:], cache, table, offsets_of(rows), i32(lengths))
    # again, one token each: pages that grow, pages that begin
    rows, lengths = [1] * 8, [2, 40, page, page, 3 * page + 6, page + 4, 2 * page + 2, page + 2]
    check_append(imm, orc, both[:8, :heads].contiguous() * 3, both[8:16, :heads].contiguous(), cache, table, offsets_of(rows), i32(lengths))


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_quotients_on_the_borders(imm, orc, dtype):
    """Half-integers, zeros, the smallest and the largest magnitudes, rows that are not finite."""
    dim, page = 32, 16
    x = torch.zeros((6 * page, 1, dim))
    x[:page] = (torch.arange(page * dim).view(page, 1, dim) % 254 - 126.5); x[0, 0, 0] = 127.0
    x[page:2 * page] = x[:page] * 2.0 ** -14
    x[3 * page:4 * page] = torch.randn((page, 1, dim), generator=torch.Generator().manual_seed(1)) * 6e4
    x[4 * page:5 * page] = torch.randn((page, 1, dim), generator=torch.Generator().manual_seed(2)) * 1e-7
    x[5 * page] = math.inf
    if dtype != torch.float16:
        x[3 * page:4 * page] *= 1e33
        x[4 * page:5 * page] *= 1e-35
    x = x.cuda().to(dtype)
    table, pages = make_table(3, [6 * page, 6 * page], page)
    cache = make_cache(4, pages, 1, page, dim)
    check_append(imm, orc, x, x.flip(0).contiguous(), cache, table[:1].contiguous(), offsets_of([6 * page]), i32([6 * page]))
    # token by token: every page's scale grows several times
    cache = make_cache(4, pages, 1, page, dim)
    for i in range(5, 5 + 2 * page):
        check_append(imm, orc, x[i:i + 1], x[-i:][:1], cache, table[1:].contiguous(), offsets_of([1]), i32([i]))


def test_append_unaligned_rows_strided_pages_and_tables(imm, orc):
    for dtype in DTYPES:
        heads, dim, page, rows, lengths = 2, 48, 16, [5, 33], [20, 40]
        buffer = randn((38 * 3 * 53 + 1,), 7, dtype)[1:].view(38, 3, 53)          # rows and heads at odd addresses
        k, v = buffer[:, :2, :48], buffer[:, 1:, 3:51]
        table, pages = make_table(8, lengths, page, width=5)
        wide = torch.full((2, 9), 77, dtype=torch.int32, device="cuda")
        wide[:, :5] = table
        both = torch.randint(-127, 128, (pages, 2, heads, page, dim), dtype=torch.int8, device="cuda")      # keys and values page by page
        cache = (both[:, 0], both[:, 1], torch.rand((pages, heads), device="cuda"), torch.rand((pages, heads), device="cuda"))
        check_append(imm, orc, k, v, cache, wide[:, :5], offsets_of(rows), i32(lengths))


def test_append_leaves_out_what_it_cannot_place(imm, orc):
    heads, dim, page = 2, 64, 16
    rows, lengths = [3, 3, 20, 2, 1], [2, 4 * page + 1, 30, 2, 5]                  # too short, too long, a bad page, fine, a page too far
    table = torch.tensor([[0, 1, 2, 3], [4, 5, 6, 7], [8, 99, 9, 9], [10, -1, -1, -1], [12, 0, 0, 0]], dtype=torch.int32, device="cuda")
    cache = make_cache(1, 12, heads, page, dim)
    k, v = randn((29, heads, dim), 2, torch.bfloat16), randn((29, heads, dim), 3, torch.bfloat16)
    check_append(imm, orc, k, v, cache, table, offsets_of(rows), i32(lengths))
    # offsets that lie outside the call, or decrease
    before = [t.clone() for t in cache]
    bad = torch.tensor([0, 40, 3, -1, 5, 5], dtype=torch.int64, device="cuda")
    assert imm.kv_append(k, v, cache, table, bad, i32([50, 20, 20, 20, 20])).tolist()[:3] == [imm.ERR_ARG] * 3
    assert same(cache[2], before[2]) and torch.equal(cache[0], before[0])
    # no rows at all
    assert imm.kv_append(k[:0], v[:0], cache, table, offsets_of([0] * 5), i32([0, 1, 16, 64, 65])).tolist() == [0, 0, 0, 0, imm.ERR_ARG]


# ------------------------------------------------------------------ attention


def check_attention(imm, orc, q, cache, table, offsets, lengths, scale, window=0, sinks=0, got=None):
    """Rows of every sequence against the oracle; returns (out, lse)."""
    dim, dtype = q.shape[2], q.dtype
    if got is None:
        got = imm.kv_attention(q, cache, table, offsets, lengths, scale, window, sinks)
    scale = float(np.float32(scale))
    out, lse, reach, size = orc.attention(host(q), [host(t) for t in cache], host(table), host(offsets), host(lengths), scale, window, sinks)
    rows = slice(0, int(offsets[-1]))
    n = max(1, int(lengths.max()))
    y, z = host(got[0])[rows], host(got[1])[rows]
    out, lse, reach, size = out[rows], lse[rows], reach[rows], size[rows]
    assert np.array_equal(np.isnan(y), np.isnan(out)) and np.array_equal(np.isnan(z), np.isnan(lse))
    assert np.array_equal(z == -math.inf, lse == -math.inf)
    e_x = (4 * dim / 16 + 8) * 2.0 ** -23 * reach + 2.0 ** -22
    good = np.isfinite(lse)
    assert np.all(np.abs(z[good] - lse[good]) <= e_x[good] + (n / 64 + 16) * 2.0 ** -23 + np.abs(lse[good]) * 2.0 ** -23)
    largest = float(np.max([host(t).max(initial=0) for t in cache[3:]])) * 127 if bool(torch.isfinite(cache[3]).all()) else 0.0
    tol = (2 * e_x[..., None] + WEIGHT[dtype] + (n / 8 + 64) * 2.0 ** -23) * size + n * 2.0 ** -31 * largest + HALF_STEP[dtype] * np.abs(out) + 1e-30
    if dtype == torch.float16:
        tol = tol + 2.0 ** -25
        y, out = np.clip(y, -65504, 65504), np.clip(out, -65504, 65504)
    bad = np.argwhere(~((np.abs(y - out) <= tol) | np.isnan(out)))
    assert len(bad) == 0, (bad[:4], y[tuple(bad[0])], out[tuple(bad[0])], tol[tuple(bad[0])])
    return got


HEADS = [(1, 1, 16, 16), (4, 1, 64, 16), (8, 8, 80, 32), (32, 8, 128, 16), (5, 1, 48, 64), (6, 2, 256, 128), (24, 2, 96, 64), (40, 2, 128, 32)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,dim,page", HEADS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 0), (33, 5)])
def test_attention_of_single_tokens(imm, orc, dtype, heads, kv_heads, dim, page, window, sinks):
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 200, 1000]
    table, pages = make_table(dim, lengths, page)
    cache = make_cache(heads, pages, kv_heads, page, dim)
    q = randn((10, heads, dim), 3, dtype, 1.5)
    check_attention(imm, orc, q, cache, table, offsets_of([1] * 10), i32(lengths), dim ** -0.5, window, sinks)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,dim,page", HEADS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3), (1, 0), (70, 200)])
def test_attention_of_several_rows(imm, orc, dtype, heads, kv_heads, dim, page, window, sinks):
    """Drafts, prompts and histories in one call; sequences without rows, without tokens, and shorter than their rows."""
    rows, lengths = [5, 0, 3, 70, 1, 4, 2, 9], [300, 50, 3, 70, 129, 0, 1, 150]
    table, pages = make_table(dim + 1, lengths, page)
    cache = make_cache(heads + 1, pages, kv_heads, page, dim)
    tokens = sum(rows) + 2
    q = randn((tokens, heads, dim), 4, dtype, 1.5)
    out = (torch.full_like(q, 7.0), torch.full((tokens, heads), 7.0, device="cuda"))
    got = imm.kv_attention(q, cache, table, offsets_of(rows), i32(lengths), dim ** -0.5, window, sinks, out=out)
    check_attention(imm, orc, q, cache, table, offsets_of(rows), i32(lengths), dim ** -0.5, window, sinks, got)
    assert (got[0][-2:] == 7.0).all() and (got[1][-2:] == 7.0).all()               # rows of no sequence


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("most,heads,kv_heads,dim", [(1, 4, 2, 64), (4, 4, 1, 96), (9, 4, 1, 64), (9, 8, 2, 128), (13, 4, 1, 128), (19, 4, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 5)])
def test_attention_of_many_short_sequences(imm, orc, dtype, most, heads, kv_heads, dim, window, sinks):
    """More sequences than a block has threads, shares of several items each, at every number of rows per key: 2, 10, 20, 28 and 40
    on average."""
    g = np.random.default_rng(most * dim)
    rows = [1 + (i * 7 + most) % most for i in range(150)]
    lengths = [r + int(g.integers(0, 260)) for r in rows]
    rows[3], rows[149], lengths[77] = 0, 0, 0
    table, pages = make_table(most, lengths, 32)
    cache = make_cache(dim, pages, kv_heads, 32, dim)
    q = randn((sum(rows), heads, dim), 5, dtype, 1.5)
    check_attention(imm, orc, q, cache, table, offsets_of(rows), i32(lengths), dim ** -0.5, window, sinks)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_of_a_prompt_with_a_history(imm, orc, dtype):
    rows, lengths = [300, 129], [420, 1000]
    table, pages = make_table(9, lengths, 64)
    cache = make_cache(10, pages, 2, 64, 64)
    q = randn((429, 4, 64), 11, dtype, 1.5)
    for window, sinks in ((0, 0), (130, 70)):
        check_attention(imm, orc, q, cache, table, offsets_of(rows), i32(lengths), 0.125, window, sinks)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_far_scales_and_logits(imm, orc, dtype):
    """Pages whose scales lie many powers of two apart, of values that matter and do not; logits beyond the range of exp; zeros."""
    dim, page, length = 64, 16, 160
    table, pages = make_table(12, [length], page, shuffle=False)
    cache = make_cache(13, pages, 1, page, dim)
    q = randn((1, 2, dim), 14, dtype)
    for ks, vs in (([0.02] * 10, [2.0 ** (-4 * i) for i in range(10)]), ([0.02] * 10, [2.0 ** (4 * i - 20) for i in range(10)]),
                   ([0.5 * 0.4 ** i for i in range(10)], [2.0 ** (3 * i - 20) for i in range(10)]), ([0.0] * 10, [0.0, 1.0] * 5),
                   ([2.0] * 10, [0.01] * 10), ([0.3 * 1.5 ** i for i in range(10)], [1e-6] * 10)):
        cache[2][:10, 0] = torch.tensor(ks, device="cuda")
        cache[3][:10, 0] = torch.tensor(vs, device="cuda")
        check_attention(imm, orc, q, cache, table, offsets_of([1]), i32([length]), 0.125)
    cache[3].zero_()
    got = imm.kv_attention(q, cache, table, offsets_of([1]), i32([length]))
    assert (got[0] == 0).all() and torch.isfinite(got[1]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_rows_of_all_magnitudes(imm, orc, dtype):
    dim = 64
    table, pages = make_table(15, [40], 16)
    cache = make_cache(16, pages, 1, 16, dim)
    q = randn((6, 1, dim), 17)
    q[0] *= 1e-6; q[1] *= 3e3; q[2, 0, 1:] *= 1e-5; q[3] = 0
    if dtype != torch.float16:
        q[4] *= 1e-36; q[0] *= 1e-25
        cache[2].fill_(1e-3); q[1] *= 1e2
    check_attention(imm, orc, q.to(dtype), cache, table, offsets_of([6]), i32([40]), 0.125)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 6, 40])
def test_attention_what_is_not_finite_stays_in_its_rows(imm, orc, dtype, rows):
    """Pages with NaN, infinite or negative scales, missing pages, rows with NaN or infinity; what is not seen does no harm."""
    dim, page, lengths = 64, 16, [100, 100, 100, 100, 100, 100]
    for window, sinks in ((0, 0), (10, 0), (20, 16)):
        table, pages = make_table(18, lengths, page)
        cache = make_cache(19, pages, 1, page, dim)
        host_table = table.cpu()
        cache[3][int(host_table[0, 6])] = math.nan           # seen by the last rows only: positions 96 .. 99
        cache[2][int(host_table[1, 2])] = math.inf
        cache[3][int(host_table[2, 5])] = -1.0
        table[3, 0] = -1; table[4, 4] = pages                # positions 0 .. 15; 64 .. 79
        q = randn((rows * 6, 2, dim), 20, dtype)
        q[rows * 5, 0, 5] = math.nan; q[rows * 6 - 1, 1, 0] = -math.inf
        got = check_attention(imm, orc, q, cache, table, offsets_of([rows] * 6), i32(lengths), 0.125, window, sinks)
        assert torch.isfinite(got[0]).any() or not window    # (without a window every sequence has one that its last row sees)
    # lengths that no table holds
    got = imm.kv_attention(q, cache, table, offsets_of([rows] * 6), i32([-1, 113, 112, 5, 1, 0]))
    assert got[0][:2 * rows].isnan().all() and got[1][:2 * rows].isnan().all() and (got[0][5 * rows:] == 0).all()


def test_attention_offsets_out_of_order_write_nothing(imm):
    table, pages = make_table(21, [50] * 4, 16)
    cache = make_cache(22, pages, 1, 16, 64)
    q = randn((4, 2, 64), 23, torch.bfloat16)
    for bad in ([0, 9, 1, 1, 1], [-3, 1, 0, 0, 0], [2, 1, 0, 0, 0]):
        out = (torch.full_like(q, 7.0), torch.full((4, 2), 7.0, device="cuda"))
        imm.kv_attention(q, cache, table, torch.tensor(bad, dtype=torch.int64, device="cuda"), i32([50] * 4), out=out)
        torch.cuda.synchronize()
        assert (out[0][2:] == 7.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_strides_and_alignment(imm, orc, dtype):
    """q as a part of a projection's output, at odd addresses too; out with strides of its own; keys and values page by page."""
    heads, kv_heads, dim, page, rows, lengths = 6, 2, 80, 32, [1, 7, 30], [40, 100, 90]
    tokens = sum(rows)
    table, pages = make_table(24, lengths, page)
    both = torch.randint(-127, 128, (pages, 2, kv_heads, page, dim), dtype=torch.int8, device="cuda")
    scales = torch.rand((2, pages, kv_heads), device="cuda") * 0.05
    cache = (both[:, 0], both[:, 1], scales[0], scales[1])
    for q in (randn((tokens, heads + 2 * kv_heads, dim), 25, dtype)[:, :heads], randn((tokens * 8 * 83 + 1,), 26, dtype)[1:].view(tokens, 8, 83)[:, 1:7, 2:82],
              randn((heads, tokens, dim), 27, dtype).transpose(0, 1)):
        whole = torch.full((tokens, heads + 1, dim + 3), 7.0, dtype=dtype, device="cuda")
        out = (whole[:, :heads, 1:dim + 1], torch.empty((tokens, heads), device="cuda"))
        got = imm.kv_attention(q, cache, table, offsets_of(rows), i32(lengths), 0.11, 60, 4, out=out)
        check_attention(imm, orc, q, cache, table, offsets_of(rows), i32(lengths), 0.11, 60, 4, got)
        assert (whole[:, heads] == 7.0).all() and (whole[:, :, 0] == 7.0).all() and (whole[:, :, dim + 1:] == 7.0).all()


@pytest.mark.parametrize("dtype,heads,kv_heads,dim", [(torch.bfloat16, 8, 2, 128), (torch.float16, 2, 2, 64), (torch.float32, 4, 1, 128)])
def test_attention_over_a_long_history(imm, dtype, heads, kv_heads, dim):
    """Keys shared out over the whole GPU; against float64 on the GPU (the oracle's formula by torch operations)."""
    page, lengths = 64, [30000, 77, 12345, 1]
    table, pages = make_table(28, lengths, page)
    cache = make_cache(29, pages, kv_heads, page, dim)
    q = randn((4, heads, dim), 30, dtype, 1.5)
    for window, sinks in ((0, 0), (10000, 100)):
        out, lse = imm.kv_attention(q, cache, table, offsets_of([1] * 4), i32(lengths), 0.08, window, sinks)
        for b, length in enumerate(lengths):
            at = table[b, :-(-length // page)].long()
            for h in range(heads):
                kv = h // (heads // kv_heads)
                k, v = ((cache[i][at, kv].double() * cache[i + 2][at, kv].double().view(-1, 1, 1)).view(-1, dim)[:length] for i in (0, 1))
                row = q[b, h].double()
                x = float(np.float32(0.08)) * (k @ row)
                key = torch.arange(length, device="cuda")
                if window:
                    x[(length - 1 - key >= window) & (key >= sinks)] = -math.inf
                p = torch.softmax(x, 0)
                e_x = (4 * dim / 16 + 8) * 2.0 ** -23 * float(0.08 * (k.abs() @ row.abs()).max()) + 2.0 ** -22
                want = torch.logsumexp(x, 0)
                assert abs(float(lse[b, h]) - float(want)) <= e_x + (length / 64 + 16) * 2.0 ** -23 + abs(float(want)) * 2.0 ** -23
                tol = (2 * e_x + WEIGHT[dtype] + (length / 8 + 64) * 2.0 ** -23) * (p @ v.abs()) + length * 2.0 ** -31 * float(v.abs().max())
                assert bool((((p @ v) - out[b, h].double()).abs() <= tol + HALF_STEP[dtype] * (p @ v).abs()).all())


def test_attention_pages_beyond_32_bits(imm, orc):
    """Entries of a cache further from its start than 2^31."""
    heads, page, dim, pages = 8, 128, 128, (1 << 31) // (8 * 128 * 128) + 40
    cache = tuple([torch.zeros((pages, heads, page, dim), dtype=torch.int8, device="cuda") for _ in range(2)] +
                  [torch.zeros((pages, heads), device="cuda") for _ in range(2)])
    table = torch.tensor([[pages - 1, pages - 9], [3, pages - 2]], dtype=torch.int32, device="cuda")
    k, v = randn((300, heads, dim), 31, torch.bfloat16), randn((300, heads, dim), 32, torch.bfloat16)
    assert imm.kv_append(k, v, cache, table, offsets_of([150, 150]), i32([150, 150])).tolist() == [0, 0]
    q = randn((2, heads, dim), 33, torch.bfloat16)
    out, _ = imm.kv_attention(q, cache, table, offsets_of([1, 1]), i32([150, 150]))
    small = tuple(t[table.view(-1).long()].contiguous() for t in cache)
    check_attention(imm, orc, q, small, i32([[0, 1], [2, 3]]), offsets_of([1, 1]), i32([150, 150]), dim ** -0.5, got=(out, _))


def test_calls_repeat_on_streams_and_in_graphs(imm):
    """The same call gives the same bits; a captured step of append and attention follows the lengths it is given; another stream's
    tensors and workspace."""
    heads, kv_heads, dim, page, batch = 8, 2, 64, 16, 5
    start = [17, 60, 1, 300, 31]
    table, pages = make_table(34, [n + 40 for n in start], page)
    steps = [randn((batch, heads + 2 * kv_heads, dim), 35 + i, torch.bfloat16, 1.5) for i in range(12)]

    def fresh():
        return tuple(t.clone() for t in make_cache(36, pages, kv_heads, page, dim))

    def step(x, cache, lengths, out=None, ws=None, status=None):
        imm.kv_append(x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], cache, table, offsets, lengths, out=status)
        return imm.kv_attention(x[:, :heads], cache, table, offsets, lengths, out=out, workspace=ws)

    offsets = offsets_of([1] * batch)
    cache, want = fresh(), []
    for i, x in enumerate(steps):
        want.append([t.clone() for t in step(x, cache, i32([n + 1 + i for n in start]))])
        again = imm.kv_attention(x[:, :heads], cache, table, offsets, i32([n + 1 + i for n in start]))
        assert torch.equal(again[0], want[-1][0]) and torch.equal(again[1], want[-1][1])
    end = [t.clone() for t in cache]
    # captured once, replayed with other rows and lengths
    x, lengths, cache = steps[0].clone(), i32([n + 1 for n in start]), fresh()
    q = x[:, :heads]
    out, ws = (torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty((batch, heads), device="cuda")), imm.kv_attention_workspace(q, cache, table, offsets)
    status = torch.empty(batch, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, cache, lengths, out, ws, status)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x, cache, lengths, out, ws, status)
    for t, c in zip(fresh(), cache):
        c.copy_(t)
    for i, s in enumerate(steps):
        x.copy_(s)
        lengths.copy_(i32([n + 1 + i for n in start]))
        graph.replay()
        assert torch.equal(out[0], want[i][0]) and torch.equal(out[1], want[i][1])
    assert all(torch.equal(a, b) for a, b in zip(cache, end))


def test_prompts_captured_and_beside_another_stream(imm):
    """Prompts: a captured call follows the lengths that it is given; two calls at once on two streams, with a workspace each."""
    rows, longest = [300, 1, 129], [900, 700, 400]
    table, pages = make_table(41, longest, 32)
    cache = make_cache(42, pages, 2, 32, 128)
    q = randn((430, 8, 128), 43, torch.bfloat16, 1.5)
    offsets, lengths = offsets_of(rows), i32(longest)
    ends = [i32(longest), i32([300, 1, 129]), i32([640, 50, 0])]
    want = [imm.kv_attention(q, cache, table, offsets, n, window=w, sinks=4) for n in ends for w in (0, 100)]
    out, ws = (torch.empty_like(q), torch.empty((430, 8), device="cuda")), imm.kv_attention_workspace(q, cache, table, offsets)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        imm.kv_attention(q, cache, table, offsets, lengths, out=out, workspace=ws)
    for i, n in enumerate(ends):
        lengths.copy_(n)
        graph.replay()
        assert same(out[0], want[2 * i][0]) and same(out[1], want[2 * i][1])
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for turn in range(6):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(imm.kv_attention(q, cache, table, offsets, ends[turn % 3], window=100 * i, sinks=4))
    torch.cuda.synchronize()
    for i in range(2):
        for turn, y in enumerate(got[i]):
            assert same(y[0], want[2 * (turn % 3) + i][0]) and same(y[1], want[2 * (turn % 3) + i][1])


def test_binding_refusals(imm):
    cache = make_cache(1, 4, 2, 16, 64)
    table, offsets, lengths = i32([[0, 1]]), offsets_of([2]), i32([20])
    x = randn((2, 2, 64), 2)
    for bad in (x[:, :1], x[:, :, :48], x.double(), x.transpose(1, 2), x[0]):
        with pytest.raises(ValueError):
            imm.kv_append(bad, x, cache, table, offsets, lengths)
        with pytest.raises(ValueError):
            imm.kv_append(x, bad, cache, table, offsets, lengths)
    for bad in (cache[:3] + (cache[3][:2],), (cache[0].float(),) + cache[1:], (cache[0].transpose(1, 2),) + cache[1:], (cache[0], cache[1][:2]) + cache[2:]):
        with pytest.raises(ValueError):
            imm.kv_append(x, x, bad, table, offsets, lengths)
        with pytest.raises(ValueError):
            imm.kv_attention(x, bad, table, offsets, lengths)
    for bad in (dict(table=table.long()), dict(offsets=offsets[:1]), dict(offsets=offsets.int()), dict(lengths=lengths.long())):
        args = dict(table=table, offsets=offsets, lengths=lengths)
        args.update(bad)
        with pytest.raises(ValueError):
            imm.kv_attention(x, cache, **args)
    with pytest.raises(ValueError):
        imm.kv_attention(x[:, :, :48], cache, table, offsets, lengths)
    with pytest.raises(ValueError):
        imm.kv_attention(x, cache, table, offsets, lengths, out=(x[:1].clone(), torch.empty((2, 2), device="cuda")))
    with pytest.raises(imm.ImmError):
        imm.kv_attention(randn((2, 3, 64), 3), cache, table, offsets, lengths)
    with pytest.raises(imm.ImmError):
        imm.kv_attention(x, cache, table, offsets, lengths, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(imm.ImmError):
        imm.kv_attention(x, cache, table, offsets, lengths, window=-1)
