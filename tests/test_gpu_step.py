"""GPU parity of the steps between products (norm with int8 output, expert dispatch and combine) with the
float64 oracle, and a run of them with the proofs and the logit distances (run with -m gpu).

Tolerances.  int8 entries, the residual sum h (one rounding), offsets, positions and moved rows: equal.  Scales:
the mean of squares is added up from float32 partial sums of at most 64 squares (65 half-steps of 2^-24, halved by
the square root) and float64 above them; the scale is rounded once: (33 + 1) 2^-24 relative.  Combine: per output a
float32 sum of `top` products, every term rounded at most three times and the running sum once per term:
(top + 3) 2^-24 of the sum of magnitudes, then half a step of the output type.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SCALE_TOL = 34 * 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


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


def randn(shape, seed, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).cuda().to(dtype)


# ------------------------------------------------------------------ norm


def check_norm(step, got, x, weight, residual, eps, group):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    if residual is not None:
        assert torch.equal(torch.nan_to_num(got[2].float(), nan=123.0), torch.nan_to_num(h.float(), nan=123.0))
    q, scale = got[0].cpu().numpy(), got[1].cpu().numpy()
    want_q, want_s = step.rmsnorm_quant(h.cpu().double().numpy(), weight.cpu().double().numpy(), eps, group)
    assert np.array_equal(q, want_q), np.argwhere(q != want_q)[:5]
    assert np.array_equal(np.isnan(scale), np.isnan(want_s))
    ok = np.isfinite(want_s)
    assert np.all(np.abs(scale[ok] - want_s[ok]) <= SCALE_TOL * np.abs(want_s[ok]) + 1e-44)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (2, 31), (5, 64), (3, 129), (4, 1000), (7, 4096), (2, 4104), (3, 5001), (2, 14336),
                                       (2, 16384), (1, 40001)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("with_residual", [False, True])
def test_norm_matches_oracle(imm, step, rows, cols, dtype, with_residual):
    x, r = randn((rows, cols), cols, dtype, 2.0), randn((rows, cols), cols + 1, dtype, 3.0) if with_residual else None
    for wdtype in {dtype, torch.float32}:
        w = (1 + randn((cols,), cols + 2, scale=0.3)).to(wdtype)
        check_norm(step, imm.rmsnorm_quant(x, w, r, 1e-5), x, w, r, 1e-5, 0)


@pytest.mark.parametrize("rows,cols", [(1, 128), (3, 256), (5, 640), (2, 4096), (9, 14336), (2, 20480)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_in_groups(imm, step, rows, cols, dtype):
    x, r, w = randn((rows, cols), 1, dtype, 2.0), randn((rows, cols), 2, dtype, 3.0), 1 + randn((cols,), 3, dtype, 0.3)
    x[0, :128] = 0; r[0, :128] = 0                           # a group of zeros
    check_norm(step, imm.rmsnorm_quant(x, w, r, 1e-6, 128), x, w, r, 1e-6, 128)
    check_norm(step, imm.rmsnorm_quant(x, w, None, 1e-6, 128), x, w, None, 1e-6, 128)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [77, 512, 4096])
def test_norm_values_on_the_borders(imm, step, dtype, cols):
    """Quotients that are exactly half-integers, the largest entry alone, constant rows, rows of zeros."""
    x = torch.zeros((5, cols), device="cuda")
    half = torch.arange(cols, device="cuda") % 254 - 126.5   # .5 from -126.5 to 126.5
    x[0] = half; x[0, 0] = 127.0
    x[1] = half * 2.0 ** 3; x[1, cols - 1] = -127.0 * 2.0 ** 3
    x[2, cols // 2] = -1e-3
    x[3] = 0.75
    x = x.to(dtype)
    w = torch.ones(cols, device="cuda", dtype=dtype)
    for eps in (0.0, 1e-5):
        got = imm.rmsnorm_quant(x, w, eps=eps)
        check_norm(step, got, x, w, None, eps, 0)
    assert int(got[0][4].abs().max()) == 0 and float(got[1][4, 0]) == 0.0
    # weights that make every product land next to a border in float32
    w32 = (1 + torch.arange(cols, device="cuda") * 2.0 ** -20).float()
    check_norm(step, imm.rmsnorm_quant(x, w32, eps=1e-5), x, w32, None, 1e-5, 0)


@pytest.mark.parametrize("cols", [100, 256, 5001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_extreme_magnitudes(imm, step, dtype, cols):
    """Products beyond float32 on either side, squares beyond float32."""
    x = randn((6, cols), 5, torch.float32)
    x[0] *= 1e30; x[1] *= 1e-30; x[2] *= 1e-38; x[3, 3] = 3e38; x[4, 3] = 1e-20; x[5] *= 1e18
    x = x.to(dtype)
    for mag in (1.0, 1e30, 1e-30):
        w = (randn((cols,), 6) * mag).to(dtype)
        for group in (0, 128) if cols % 128 == 0 else (0,):
            check_norm(step, imm.rmsnorm_quant(x, w, eps=0.0, group=group), x, w, None, 0.0, group)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_rows_that_are_not_finite(imm, step, dtype):
    for cols, group in ((300, 0), (512, 0), (512, 128)):
        x, w = randn((5, cols), 8, dtype), 1 + randn((cols,), 9, dtype, 0.1)
        x[0, 7] = math.inf; x[1, 7] = math.nan; x[2, cols - 1] = -math.inf
        got = imm.rmsnorm_quant(x, w, group=group)
        check_norm(step, got, x, w, None, 1e-6, group)
        assert bool(torch.isnan(got[1][:3]).all()) and not bool(torch.isnan(got[1][3:]).any())
        w[200] = math.nan
        check_norm(step, imm.rmsnorm_quant(x, w, group=group), x, w, None, 1e-6, group)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_strides_aliases_and_neighbours(imm, step, dtype):
    rows, cols = 5, 1000
    for offset, pad in ((0, 24), (1, 7), (8, 8)):
        buf = torch.full((3, rows * (cols + pad) + 16), 9.0, dtype=dtype, device="cuda")
        view = lambda k: buf[k, offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        x, r, h = view(0), view(1), view(2)
        x.copy_(randn((rows, cols), 1)); r.copy_(randn((rows, cols), 2))
        w = 1 + randn((cols,), 3, dtype, 0.2)
        qbuf = torch.full((rows * (cols + pad) + 16,), 55, dtype=torch.int8, device="cuda")
        q = qbuf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        scale = torch.empty((rows, 1), device="cuda")
        imm.rmsnorm_quant(x, w, r, 1e-5, out=(q, scale, h))
        check_norm(step, (q, scale, h), x, w, r, 1e-5, 0)
        rest = qbuf.clone()
        rest[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 55
        assert bool((rest == 55).all())
        rest = buf[2].clone()
        rest[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 9.0
        assert bool((rest == 9.0).all())
        x0, r0 = x.clone(), r.clone()
        imm.rmsnorm_quant(x, w, r, 1e-5, out=(q, scale, r))       # the residual updated in place
        check_norm(step, (q, scale, r), x0, w, r0, 1e-5, 0)
        r.copy_(r0)
        imm.rmsnorm_quant(x, w, r, 1e-5, out=(q, scale, x))
        check_norm(step, (q, scale, x), x0, w, r0, 1e-5, 0)


def test_norm_many_rows_and_none(imm, step):
    x, w = randn((4001, 136), 4, torch.bfloat16), 1 + randn((136,), 5, torch.bfloat16, 0.1)
    check_norm(step, imm.rmsnorm_quant(x, w), x, w, None, 1e-6, 0)
    q, s = imm.rmsnorm_quant(x[:0], w)
    assert q.shape == (0, 136) and s.shape == (0, 1)


# ------------------------------------------------------------------ dispatch


def routing(tokens, top, experts, seed, dropped=0.0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(experts, (tokens, top), generator=g, dtype=torch.int32)
    if dropped:
        ids[torch.rand((tokens, top), generator=g) < dropped] = -1
    return ids.cuda()


def check_dispatch(step, got, x, ids, experts, scale):
    rows, offsets, position, row_scale, status = got
    want_o, want_p, source = step.dispatch(ids.cpu().numpy(), experts)
    assert offsets.cpu().tolist() == want_o.tolist() and np.array_equal(position.cpu().numpy(), want_p) and int(status) == 0
    token = torch.from_numpy(source // ids.shape[1]).cuda()
    assert torch.equal(rows[:len(source)].view(torch.uint8), x[token].view(torch.uint8))
    if scale is not None:
        assert torch.equal(row_scale[:len(source)], scale[token])


@pytest.mark.parametrize("tokens,top,experts,cols", [(1, 1, 1, 1), (1, 2, 8, 4096), (7, 3, 5, 33), (16, 2, 8, 4096), (100, 8, 256, 72),
                                                     (64, 64, 64, 16), (333, 6, 64, 130), (1024, 2, 8, 64), (1025, 2, 8, 20),
                                                     (3000, 4, 1024, 8), (5000, 3, 7, 16)])
@pytest.mark.parametrize("dtype", [torch.int8, torch.bfloat16, torch.float32])
def test_dispatch_matches_oracle(imm, step, tokens, top, experts, cols, dtype):
    x = randn((tokens, cols), tokens, torch.float32, 20.0).to(dtype)
    scale = torch.rand(tokens, generator=torch.Generator().manual_seed(1)).cuda()
    for dropped in (0.0, 0.3, 1.0):
        ids = routing(tokens, top, experts, tokens + top, dropped)      # an expert may be named twice by a token
        check_dispatch(step, imm.moe_dispatch(x, ids, experts, scale), x, ids, experts, scale)
    ids = torch.full((tokens, top), experts - 1, dtype=torch.int32, device="cuda")
    check_dispatch(step, imm.moe_dispatch(x, ids, experts), x, ids, experts, None)


def test_dispatch_without_tokens_and_with_very_many(imm, step):
    x, ids = torch.empty((0, 8), dtype=torch.int8, device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda")
    rows, offsets, position, _, status = imm.moe_dispatch(x, ids, 5)
    assert rows.shape == (0, 8) and offsets.tolist() == [0] * 6 and position.shape == (0, 2) and int(status) == 0
    for tokens, top, experts in ((262144, 2, 8), (300001, 2, 3), (70000, 17, 1000)):      # 256 runs, longer runs
        x = torch.arange(tokens, dtype=torch.int32, device="cuda").view(-1, 1)
        ids = routing(tokens, top, experts, tokens, 0.05)
        check_dispatch(step, imm.moe_dispatch(x, ids, experts), x, ids, experts, None)


def test_dispatch_leaves_the_rest_and_reports_bad_experts(imm, step):
    tokens, top, experts, cols = 600, 4, 9, 40
    x, ids = randn((tokens, cols), 3), routing(tokens, top, experts, 3, 0.5)
    out = (torch.full((tokens * top + 5, cols), 7.0, device="cuda"), torch.empty(experts + 1, dtype=torch.int64, device="cuda"),
           torch.empty((tokens, top), dtype=torch.int32, device="cuda"), torch.full((tokens * top + 5,), 7.0, device="cuda"),
           torch.empty(1, dtype=torch.int32, device="cuda"))
    scale = torch.rand(tokens, device="cuda")
    imm.moe_dispatch(x, ids, experts, scale, out=out)
    check_dispatch(step, out, x, ids, experts, scale)
    held = int((ids >= 0).sum())
    assert bool((out[0][held:] == 7.0).all()) and bool((out[3][held:] == 7.0).all())
    for wrong in (experts, -2, 2 ** 31 - 1, -2 ** 31):
        bad = ids.clone()
        bad[599, 3] = wrong
        as_none = ids.clone()
        as_none[599, 3] = -1
        got = imm.moe_dispatch(x, bad, experts)
        want = imm.moe_dispatch(x, as_none, experts)
        assert int(got[4]) == imm.ERR_ARG and int(want[4]) == imm.OK
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
        k = int(want[1][-1])
        assert torch.equal(got[0][:k], want[0][:k])


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3), (4, 0), (3, 2)])
def test_dispatch_strides(imm, step, offset, pad):
    tokens, top, experts = 50, 3, 6
    for dtype, cols in ((torch.int8, 1001), (torch.bfloat16, 333), (torch.float32, 100), (torch.int8, 64)):
        buf = torch.zeros(tokens * (cols + pad) + offset + 16, dtype=dtype, device="cuda")
        x = buf[offset:offset + tokens * (cols + pad)].view(tokens, cols + pad)[:, :cols]
        x.copy_(randn((tokens, cols), 1, torch.float32, 20.0))
        ids = routing(tokens, top, experts, 5, 0.1)
        obuf = torch.full((tokens * top * (cols + pad) + offset + 16,), 3, dtype=dtype, device="cuda")
        view = obuf[offset:offset + tokens * top * (cols + pad)].view(tokens * top, cols + pad)
        out = (view[:, :cols], torch.empty(experts + 1, dtype=torch.int64, device="cuda"),
               torch.empty((tokens, top), dtype=torch.int32, device="cuda"), None, torch.empty(1, dtype=torch.int32, device="cuda"))
        imm.moe_dispatch(x, ids, experts, out=out)
        held = int((ids >= 0).sum())
        want_o, want_p, source = step.dispatch(ids.cpu().numpy(), experts)
        assert torch.equal(view[:held, :cols], x[torch.from_numpy(source // top).cuda()])
        assert bool((view[:, cols:] == 3).all()) and bool((view[held:] == 3).all()) and bool((obuf[:offset] == 3).all())


# ------------------------------------------------------------------ combine


def check_combine(step, got, y, position, weights, row_scale, top):
    args = (position.cpu().numpy(), None if weights is None else weights.cpu().double().numpy(),
            None if row_scale is None else row_scale.cpu().double().numpy())
    wide = y.cpu().double().numpy()
    want, size = step.combine(wide, *args), step.combine(np.abs(wide), args[0], None if args[1] is None else np.abs(args[1]),
                                                         None if args[2] is None else np.abs(args[2]))
    tol = (top + 3) * 2.0 ** -24 * size
    tol = tol + HALF_STEP[got.dtype] * (np.abs(want) + tol) + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    assert np.all(np.abs(got.cpu().double().numpy() - want) <= tol)


@pytest.mark.parametrize("tokens,top,cols", [(1, 1, 1), (1, 2, 4096), (5, 3, 33), (16, 2, 4096), (31, 6, 2051), (9, 64, 40), (300, 8, 100),
                                             (2, 2, 20000)])
@pytest.mark.parametrize("dtype", [torch.int32] + DTYPES)
def test_combine_matches_oracle(imm, step, tokens, top, cols, dtype):
    experts = 16
    ids = routing(tokens, top, experts, tokens, 0.2)
    _, position, source = step.dispatch(ids.cpu().numpy(), experts)
    position = torch.from_numpy(position).cuda()
    rows = max(len(source), 1)
    y = randn((rows, cols), 1, torch.float32, 1e6).to(torch.int32) if dtype == torch.int32 else randn((rows, cols), 1, dtype)
    w, s = randn((tokens, top), 2), torch.rand(rows, generator=torch.Generator().manual_seed(3)).cuda() * (1e-6 if dtype == torch.int32 else 1.0)
    for weights, row_scale in ((w, s), (w, None), (None, s), (None, None)):
        for out_dtype in DTYPES:
            if out_dtype == torch.float16 and dtype == torch.int32 and row_scale is None:
                continue                                          # (beyond the range of float16)
            got = imm.moe_combine(y, position, weights, row_scale, out_dtype=out_dtype)
            assert got.dtype == out_dtype
            check_combine(step, got, y, position, weights, row_scale, top)


def test_combine_strides_empty_tokens_and_bad_positions(imm, step):
    tokens, top, cols = 40, 3, 333
    for dtype in (torch.bfloat16, torch.float32, torch.int32):
        for offset, pad in ((0, 3), (1, 0), (8, 8)):
            y = torch.zeros(120 * (cols + pad) + 16, dtype=dtype, device="cuda")[offset:offset + 120 * (cols + pad)].view(120, cols + pad)[:, :cols]
            y.copy_(randn((120, cols), 4, torch.float32, 100.0))
            position = torch.randperm(120, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(tokens, top).cuda()
            position[3] = -1
            position[5, 1] = -1
            position[6, 0] = 120                                  # a row that y does not have is left out
            position[6, 1] = 2 ** 31 - 1
            obuf = torch.full((tokens * (cols + pad) + 16,), 5.0, dtype=torch.float32, device="cuda")
            view = obuf[offset:offset + tokens * (cols + pad)].view(tokens, cols + pad)
            w = randn((tokens, top), 8)
            got = imm.moe_combine(y, position, w, out=view[:, :cols])
            check_combine(step, got, y, position, w, None, top)
            assert float(got[3].abs().max()) == 0.0 and bool((view[:, cols:] == 5.0).all()) and bool((obuf[:offset] == 5.0).all())
    assert imm.moe_combine(y, position[:0]).shape == (0, cols)


def test_combine_undoes_dispatch_and_is_its_adjoint(imm):
    """With weights that add up to one the round trip returns the tokens; without weights combine is the
    transpose of dispatch: <dispatch(x), g> = <x, combine(g)>, exactly in integers."""
    tokens, top, experts, cols = 700, 4, 12, 96
    ids = torch.stack([torch.randperm(experts, generator=torch.Generator().manual_seed(t))[:top] for t in range(tokens)]).to(torch.int32).cuda()
    x = randn((tokens, cols), 2, torch.bfloat16)
    rows, offsets, position, _, _ = imm.moe_dispatch(x, ids, experts)
    back = imm.moe_combine(rows, position, torch.full((tokens, top), 1.0 / top, device="cuda"))
    assert torch.equal(back, x)
    xi = torch.randint(-9, 10, (tokens, cols), generator=torch.Generator().manual_seed(5)).cuda()
    gi = torch.randint(-9, 10, (tokens * top, cols), generator=torch.Generator().manual_seed(6)).cuda()
    moved = imm.moe_dispatch(xi.to(torch.int32), ids, experts)[0].long()
    summed = imm.moe_combine(gi.to(torch.int32), position, out_dtype=torch.float32).long()
    assert int((moved * gi).sum()) == int((xi * summed).sum())


# ------------------------------------------------------------------ captured, on other streams, together


def test_capture_and_replay(imm, step):
    tokens, top, experts, cols = 1500, 2, 8, 256
    x, r, w = randn((tokens, cols), 1, torch.bfloat16), randn((tokens, cols), 2, torch.bfloat16), 1 + randn((cols,), 3, torch.bfloat16, 0.1)
    ids, wt = routing(tokens, top, experts, 4), torch.rand((tokens, top), device="cuda")

    def chain():
        q, s, h = imm.rmsnorm_quant(x, w, r, 1e-5)
        rows, offsets, position, row_scale, status = imm.moe_dispatch(q, ids, experts, s.view(-1))
        return q, s, h, rows, offsets, position, row_scale, status, imm.moe_combine(rows.to(torch.int32), position, wt, row_scale)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain()
    with torch.cuda.graph(other):
        got2 = chain()
    for seed in (5, 6):
        x.copy_(randn((tokens, cols), seed)); ids.copy_(routing(tokens, top, experts, seed, 0.1))
        graph.replay(); other.replay()
        for g in (got, got2):
            check_norm(step, g[:3], x, w, r, 1e-5, 0)
            check_dispatch(step, g[3:8], g[0], ids, experts, g[1].view(-1))
            check_combine(step, g[8], g[3].to(torch.int32), g[5], wt, g[6], top)


def test_a_step_of_an_expert_layer_is_proved_and_sampled(imm, step):
    """The calls as an audit uses them: the residual stream is normalised to int8, sorted by expert, every expert's
    product is proved from the sorted rows, its accumulators come back weighted, the next norm feeds the output
    projection, whose logits are sampled and compared with the reference's."""
    tokens, d, experts, top, vocab = 48, 64, 4, 2, 1500
    g = torch.Generator().manual_seed(7)
    x, r, w = randn((tokens, d), 1, torch.bfloat16), randn((tokens, d), 2, torch.bfloat16), 1 + randn((d,), 3, torch.bfloat16, 0.1)
    q, s, h = imm.rmsnorm_quant(x, w, r, 1e-5)
    ids = torch.stack([torch.randperm(experts, generator=g)[:top] for _ in range(tokens)]).to(torch.int32).cuda()
    rows, offsets, position, row_scale, status = imm.moe_dispatch(q, ids, experts, s.view(-1))
    assert int(status) == imm.OK
    W = torch.randint(-20, 21, (experts, d, d), generator=g).to(torch.int8)
    C = torch.empty((tokens * top, d), dtype=torch.int32, device="cuda")
    off = offsets.cpu().tolist()
    assert off[-1] == tokens * top
    problems = []
    for e in range(experts):
        if off[e + 1] > off[e]:
            A = rows[off[e]:off[e + 1]]
            C[off[e]:off[e + 1]] = (A.cpu().long() @ W[e].long()).to(torch.int32).cuda()
            problems.append((A, W[e].cuda(), C[off[e]:off[e + 1]], e))
    for (A, B, c, pid), t in zip(problems, imm.sumcheck_matmul_prove(problems, 11)):
        assert imm.sumcheck_verify(t, imm.ceil_log2(A.shape[1]), 11, pid) == (imm.OK, -1)
    weights = torch.softmax(randn((tokens, top), 9), 1)
    y = imm.moe_combine(C, position, weights, row_scale * 0.01)
    check_combine(step, y, C, position, weights, row_scale * 0.01, top)
    q2, s2, h2 = imm.rmsnorm_quant(y, w, h, 1e-5)
    check_norm(step, (q2, s2, h2), y, w, h, 1e-5, 0)
    logits = ((q2.float() * s2) @ randn((d, vocab), 5)).contiguous()
    u = torch.rand(tokens, generator=g, dtype=torch.float64).cuda()
    token, lp, kept, st = imm.sample(logits, u, 0.8, 20, 0.95)
    assert int(st.abs().max()) == 0 and int(kept.max()) <= 20
    lx = logits.cpu().double().numpy()
    for i in range(tokens):
        want = step.sample(lx[i], float(u[i]), 0.8, 20, 0.95)
        assert (int(token[i]), int(kept[i])) == (want[0], want[2]) and abs(float(lp[i]) - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-9
    committed = torch.topk(logits, 20, dim=1).indices.to(torch.int32).contiguous()
    dist, dstatus = imm.ldd_topk_distance(logits, committed)
    assert int(dstatus.abs().max()) == 0 and float(dist.abs().max()) == 0.0
    assert bool((committed == token.view(-1, 1)).any(1).all())
