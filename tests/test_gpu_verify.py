"""GPU parity of the verification of drafted tokens with the float64 oracle, and a step of a request with drafts from the
cache to the answer (run with -m gpu).

Taken tokens, answers and status are equal: the comparisons are of float64 weights that both sides have within 1e-12, and no
test's numbers lie that near to a border (the borders that are met on purpose are exact).  logprob is one float32 rounding of a
float64 logarithm: 2^-24 relative, and 1e-12 of the weights.
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


def make(seed, held, n, dtype, lift=12.0, noise=0.7, masked=0.0):
    """(target, draft, tokens, offsets, u) of requests with `held` drafted tokens each, proposed by the draft."""
    g = torch.Generator().manual_seed(seed)
    rows = sum(held) + len(held)
    x = torch.randn((rows, n), generator=g) * 2
    x.scatter_add_(1, torch.randint(n, (rows, 5), generator=g), torch.linspace(lift, lift - 5, 5).expand(rows, 5).contiguous())
    if masked:
        x[torch.rand((rows, n), generator=g) < masked] = -math.inf
        x[:, n // 2] = 0.0
    offsets = np.cumsum([0] + [k + 1 for k in held])
    tested = np.array([r for b in range(len(held)) for r in range(offsets[b], offsets[b + 1] - 1)], dtype=np.int64)
    target = x.to(dtype)
    draft = (x[tested] + noise * torch.randn((len(tested), n), generator=g)).to(dtype)
    tokens = torch.zeros(rows, dtype=torch.int32)
    if len(tested):
        tokens[torch.from_numpy(tested) + 1] = torch.multinomial(torch.softmax(draft.float(), 1), 1, generator=g).view(-1).to(torch.int32)
    u = torch.rand(rows, generator=g, dtype=torch.float64)
    return target.cuda(), draft.cuda(), tokens.cuda(), torch.from_numpy(offsets).cuda(), u.cuda()


def check(imm, orc, target, draft, tokens, offsets, u, temperature=1.0, got=None):
    if got is None:
        got = imm.verify_draft(target, draft, tokens, offsets, u, temperature)
    x, y = target.cpu().double().numpy(), None if draft is None else draft.cpu().double().numpy()
    at, tok, v = offsets.tolist(), tokens.tolist(), u.tolist()
    for b in range(len(at) - 1):
        t = float(temperature[b]) if isinstance(temperature, torch.Tensor) else temperature
        want = orc.verify(x[at[b]:at[b + 1]], None if y is None else y[at[b] - b:at[b + 1] - b - 1], tok[at[b]:at[b + 1]], v[at[b]:at[b + 1]], t)
        mine = [t[b].item() for t in got]
        assert (mine[0], mine[1], mine[3]) == (want[0], want[1], want[3]), (b, mine, want)
        if want[3] == 0:
            assert abs(mine[2] - want[2]) <= abs(want[2]) * 2.0 ** -24 + 1e-12
        else:
            assert math.isnan(mine[2])
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 2, 3, 17, 255, 256, 1000, 4099, 32001])
@pytest.mark.parametrize("with_draft", [True, False])
def test_matches_oracle(imm, orc, dtype, n, with_draft):
    held = [0, 1, 2, 5, 3, 0, 8, 4, 1]
    target, draft, tokens, offsets, u = make(n, held, n, dtype)
    check(imm, orc, target, draft if with_draft else None, tokens, offsets, u)
    temperature = torch.tensor([0.0, 0.5, 1.0, 2.0, 0.0, 0.7, 1.3, 0.9, 0.3], device="cuda")
    check(imm, orc, target, draft if with_draft else None, tokens, offsets, u, temperature)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("requests", [1, 3, 40, 200])
def test_numbers_of_requests(imm, orc, dtype, requests):
    """From sixteen blocks per request to one."""
    held = [(3 * i + 2) % 5 for i in range(requests)]
    n = 50001 if requests < 100 else 5001
    target, draft, tokens, offsets, u = make(requests, held, n, dtype, masked=0.3)
    check(imm, orc, target, draft, tokens, offsets, u, 0.8)


@pytest.mark.parametrize("dtype", DTYPES)
def test_ends_of_the_numbers(imm, orc, dtype):
    """u at 0 and just below 1; masked drafts; the same distribution twice; ties; far temperatures."""
    held, n = [3, 2, 4, 1], 700
    target, draft, tokens, offsets, u = make(5, held, n, dtype, masked=0.5)
    for value in (0.0, 1.0 - 2.0 ** -53, 5e-324):
        check(imm, orc, target, draft, tokens, offsets, torch.full_like(u, value))
        check(imm, orc, target, None, tokens, offsets, torch.full_like(u, value))
    same = target[[r for b in range(4) for r in range(int(offsets[b]), int(offsets[b + 1]) - 1)]].contiguous()
    got = check(imm, orc, target, same, torch.full_like(tokens, n // 2), offsets, torch.full_like(u, 1.0 - 2.0 ** -53))
    assert got[0].tolist() == held                            # p = q: all are taken
    flat = torch.zeros_like(target)
    check(imm, orc, flat, torch.zeros_like(draft), tokens, offsets, u)
    check(imm, orc, flat, None, tokens, offsets, u, 0.0)
    for t in (1e-3, 50.0, 1e30, 3e38):
        check(imm, orc, target, draft, tokens, offsets, u, t)
    only = torch.full_like(target, -math.inf)
    only[:, 3] = -2.0
    got = check(imm, orc, only, draft, torch.full_like(tokens, 3), offsets, u)
    assert got[0].tolist() == held and got[1].tolist() == [3] * 4
    got = check(imm, orc, only, draft, torch.full_like(tokens, 4), offsets, u)
    assert got[0].tolist() == [0] * 4 and got[1].tolist() == [3] * 4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_maxima_anywhere_and_far_apart(imm, orc, dtype):
    """Rows whose entries lie further apart than the range of a weight, rising and falling."""
    n, held = 6000, [2, 2, 2]
    target, draft, tokens, offsets, u = make(6, held, n, dtype)
    ramp = torch.linspace(-3000.0, 3000.0, n, device="cuda")
    rows, drafts = [0, 3, 6], [0, 2, 4]
    target[rows[0]] = ramp.to(dtype); target[rows[1]] = ramp.flip(0).to(dtype); target[rows[2]] = (ramp * 1e30).to(dtype)
    draft[drafts[0]] = ramp.to(dtype); draft[drafts[1]] = ramp.flip(0).to(dtype); draft[drafts[2]] = (ramp * 1e30).to(dtype)
    tokens[offsets[:-1] + 1] = torch.tensor([n - 1, 0, n - 1], dtype=torch.int32, device="cuda")
    for t in (1.0, 10.0, 0.01):
        check(imm, orc, target, draft, tokens, offsets, u, t)


@pytest.mark.parametrize("dtype", DTYPES)
def test_requests_without_an_answer(imm, orc, dtype):
    held = [2] * 9
    target, draft, tokens, offsets, u = make(7, held, 300, dtype)
    u[0] = 1.0; u[3 + 2] = math.nan
    tokens[6 + 1] = 300; tokens[9 + 2] = -1
    target[12, 7] = math.nan; target[15, 9] = math.inf; target[18] = -math.inf
    draft[7 * 2, 5] = math.nan
    temperature = torch.ones(9, device="cuda")
    temperature[8] = -0.5
    got = check(imm, orc, target, draft, tokens, offsets, u, temperature)
    assert got[3].tolist() == [imm.ERR_ARG] * 9
    temperature[8] = math.nan
    assert int(imm.verify_draft(target, draft, tokens, offsets, u, temperature)[3][8]) == imm.ERR_ARG
    for t in (-1.0, math.inf, math.nan):
        assert imm.verify_draft(target, draft, tokens, offsets, u, t)[3].tolist() == [imm.ERR_ARG] * 9
    # rows behind the token that is not taken are not looked at
    target, draft, tokens, offsets, u = make(8, [3], 300, dtype)
    target[0, int(tokens[1])] = -math.inf
    target[2:] = math.nan; draft[1:] = math.nan
    got = check(imm, orc, target, draft, tokens, offsets, u)
    assert got[0].tolist() == [0] and got[3].tolist() == [0]
    # requests without rows, rows outside the call
    odd = torch.tensor([0, 0, 4, 9, 2, -1, 1], dtype=torch.int64, device="cuda")
    got = imm.verify_draft(target, draft, tokens, odd, u)                          # (the second one's draft rows would begin at -1)
    assert got[3].tolist() == [imm.ERR_ARG] * 6 and got[1].tolist() == [-1] * 6
    got = imm.verify_draft(target, None, tokens, odd[:3], u)
    assert got[3].tolist()[0] == imm.ERR_ARG
    target, draft, tokens, offsets, u = make(8, [3, 2], 300, dtype)
    got = imm.verify_draft(target, draft[:4], tokens, torch.cat([offsets, offsets[-1:]]), u)
    assert got[3].tolist() == [0, imm.ERR_ARG, imm.ERR_ARG]                        # a draft row too few; no rows
    check(imm, orc, target, draft, tokens, offsets, u, got=[t[:2] for t in imm.verify_draft(target, draft, tokens, torch.cat([offsets, offsets[-1:]]), u)])


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_at_any_address(imm, orc, dtype):
    held, n = [2, 0, 3], 1001
    target, draft, tokens, offsets, u = make(9, held, n, dtype, masked=0.2)
    for pad, skip in ((0, 1), (7, 3), (7, 0), (23, 5)):
        wide = torch.full((len(target) * (n + pad) + skip + 8,), math.nan, dtype=dtype, device="cuda")
        x = wide[skip:skip + len(target) * (n + pad)].view(len(target), n + pad)[:, :n]
        x.copy_(target)
        check(imm, orc, x, draft, tokens, offsets, u)
        both = torch.full((len(draft) * (n + 1) + 2,), math.nan, dtype=dtype, device="cuda")
        y = both[1:1 + len(draft) * (n + 1)].view(len(draft), n + 1)[:, 1:]
        y.copy_(draft)
        check(imm, orc, x, y, tokens, offsets, u)


def test_the_largest_row_and_repeated_calls(imm, orc):
    n = 1 << 20
    target, draft, tokens, offsets, u = make(10, [2, 1], n, torch.bfloat16)
    first = check(imm, orc, target, draft, tokens, offsets, u)
    out = tuple(torch.empty_like(t) for t in first)
    graph = torch.cuda.CUDAGraph()
    imm.verify_draft(target, draft, tokens, offsets, u, out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        imm.verify_draft(target, draft, tokens, offsets, u, out=out)
    for seed in (11, 12):
        u.copy_(torch.rand(u.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64))
        graph.replay()
        check(imm, orc, target, draft, tokens, offsets, u, got=out)


def test_binding_refusals(imm):
    target, draft, tokens, offsets, u = make(13, [2, 1], 64, torch.float32)
    for bad in (dict(target=target.double()), dict(target=target[0]), dict(draft=draft.half()), dict(draft=draft[:, :60]),
                dict(tokens=tokens.long()), dict(tokens=tokens[:3]), dict(offsets=offsets.int()), dict(u=u.float()), dict(u=u[:2]),
                dict(temperature=torch.ones(3, device="cuda")), dict(temperature=torch.ones(2, device="cuda").double())):
        args = dict(target=target, draft=draft, tokens=tokens, offsets=offsets, u=u)
        args.update(bad)
        with pytest.raises(ValueError):
            imm.verify_draft(**args)


def test_a_step_with_drafted_tokens_from_the_cache_to_the_answer(imm, orc, oracle):
    """Three requests: rows into the cache, attention of a drafted step, logits, verification; the sequences are cut back to what was
    taken and the next step goes on; the cache's entries are the operand of a proved product."""
    heads, kv_heads, dim, page, n = 4, 2, 64, 16, 500
    start, held, g = [20, 37, 3], [3, 0, 2], torch.Generator().manual_seed(14)
    table = torch.arange(3 * 6, dtype=torch.int32, device="cuda").view(3, 6)
    cache = tuple([torch.zeros((18, kv_heads, page, dim), dtype=torch.int8, device="cuda") for _ in range(2)] +
                  [torch.zeros((18, kv_heads), device="cuda") for _ in range(2)])
    embed = torch.randn((n, (heads + 2 * kv_heads) * dim), generator=g).cuda()
    head = torch.randn((heads * dim, n), generator=g).cuda() * 0.6

    def rows_of(tokens):
        return embed[tokens.long()].to(torch.bfloat16).view(-1, heads + 2 * kv_heads, dim)

    def i32(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def offsets_of(v):
        return torch.tensor(np.cumsum([0] + v), dtype=torch.int64, device="cuda")

    prompt = torch.randint(n, (sum(start),), generator=g).cuda()
    x = rows_of(prompt)
    assert imm.kv_append(x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], cache, table, offsets_of(start), i32(start)).tolist() == [0] * 3
    lengths = list(start)
    last = torch.randint(n, (3,), generator=g).tolist()
    for step in range(3):
        drafted = [torch.randint(n, (k,), generator=g).tolist() for k in held]
        tokens = i32(sum(([a] + d for a, d in zip(last, drafted)), []))
        offsets = offsets_of([k + 1 for k in held])
        x = rows_of(tokens)
        after = i32([a + k + 1 for a, k in zip(lengths, held)])
        assert imm.kv_append(x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], cache, table, offsets, after).tolist() == [0] * 3
        y, _ = imm.kv_attention(x[:, :heads], cache, table, offsets, after)
        logits = y.reshape(len(tokens), -1).float() @ head
        draft = torch.randn((sum(held), n), generator=g).cuda()
        u = torch.rand(len(tokens), generator=g, dtype=torch.float64).cuda()
        got = check(imm, orc, logits, draft, tokens, offsets, u, 0.9)
        # the rows one by one: the same cache, the same masks
        for b in range(3):
            for i in range(held[b] + 1):
                row = int(offsets[b]) + i
                one, _ = imm.kv_attention(x[row:row + 1, :heads], cache, table[b:b + 1], offsets_of([1]), i32([lengths[b] + i + 1]))
                assert torch.allclose(one[0].float(), y[row].float(), atol=0.02, rtol=0.02)
        taken = got[0].tolist()
        lengths = [a + 1 + k for a, k in zip(lengths, taken)]
        last = got[1].tolist()
    # a page's keys are the right operand of a proved product, with an int8 row of queries as the left one
    q8 = torch.randint(-127, 128, (5, dim), generator=g, dtype=torch.int8).cuda()
    keys = cache[0][int(table[0, 0]), 1].t().contiguous()
    product = (q8.cpu().int() @ keys.cpu().int()).to(torch.int32).cuda()
    proof = imm.sumcheck_matmul_prove([(q8, keys, product, 3)], seed=21)[0]
    assert proof == [int(w) for w in oracle.sumcheck_matmul_prove(q8.cpu().numpy(), keys.cpu().numpy(), product.cpu().numpy(), 21, 3)]
