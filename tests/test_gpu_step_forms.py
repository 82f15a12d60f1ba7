"""GPU parity of every launch form of the norm with int8 output, and of dispatch where a block moves several long rows
(run with -m gpu).  Tolerances as in test_gpu_step.py: int8 entries, h and moved rows equal; scales 34 * 2^-24 relative.

Which form a call takes depends on the number of rows (more than the GPU has multiprocessors, or not), on the columns, and
on how x, residual, h and q lie with respect to 16 bytes.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SCALE_TOL = 34 * 2.0 ** -24


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


def many():
    return torch.cuda.get_device_properties(0).multi_processor_count + 5


def randn(shape, seed, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).cuda().to(dtype)


def placed(rows, cols, dtype, offset, pad, fill):
    """(buffer, view) of rows x cols entries that begin `offset` entries into a buffer, `pad` entries between the rows."""
    buf = torch.full((rows * (cols + pad) + offset + 32,), fill, dtype=dtype, device="cuda")
    return buf, buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def check(imm, step, rows, cols, dtype, group=0, x_at=(0, 0), r_at=None, h_at=None, q_at=(0, 0), wdtype=None):
    """A call with a residual and one without, its neighbours left as they were."""
    views = {}
    for name, place in (("x", x_at), ("r", r_at or x_at), ("h", h_at or x_at)):
        views[name] = placed(rows, cols, dtype, place[0], place[1], 9.0)
    x, r, h = (views[k][1] for k in "xrh")
    x.copy_(randn((rows, cols), cols, dtype, 2.0)); r.copy_(randn((rows, cols), cols + 1, dtype, 3.0))
    x[rows // 2] = 0; r[rows // 2] = 0
    x[1] *= 64
    w = (1 + randn((cols,), cols + 2, scale=0.3)).to(wdtype or dtype)
    qbuf, q = placed(rows, cols, torch.int8, q_at[0], q_at[1], 55)
    scale = torch.full((rows, cols // group if group else 1), 7.0, device="cuda")

    def compare(rows_h):
        want_q, want_s = step.rmsnorm_quant(rows_h.cpu().double().numpy(), w.cpu().double().numpy(), 1e-5, group)
        got_q, got_s = q.cpu().numpy(), scale.cpu().numpy()
        assert np.array_equal(got_q, want_q), np.argwhere(got_q != want_q)[:5]
        assert np.all(np.abs(got_s - want_s) <= SCALE_TOL * np.abs(want_s))

    imm.rmsnorm_quant(x, w, r, 1e-5, group, out=(q, scale, h))
    want = (x.float() + r.float()).to(dtype)
    assert torch.equal(h, want)
    compare(want)
    for buf, view, fill in ((views["h"][0], h, 9.0), (qbuf, q, 55)):
        view.fill_(fill)
        assert bool((buf == fill).all())
    imm.rmsnorm_quant(x, w, None, 1e-5, group, out=(q, scale))
    compare(x)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vectors", [1, 31, 32, 33, 64, 65, 128, 129, 700, 2048])
def test_aligned_rows(imm, step, dtype, vectors):
    """A warp per row with one, two and four vectors per lane; blocks with four."""
    check(imm, step, many(), vectors * (4 if dtype == torch.float32 else 8), dtype)


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 16384), (torch.float32, 16388), (torch.bfloat16, 16392), (torch.bfloat16, 32768),
                                        (torch.float16, 24000), (torch.bfloat16, 32776)])
def test_aligned_long_rows(imm, step, dtype, cols):
    """Eight vectors per thread, and rows too long for that."""
    check(imm, step, many(), cols, dtype)
    check(imm, step, 3, cols, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cols", [64, 504, 1024, 4096, 20000])
def test_aligned_rows_with_float32_weights(imm, step, dtype, cols):
    check(imm, step, many(), cols, dtype, wdtype=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [128, 2048, 2176, 4096, 4224, 8192, 8320])
def test_groups(imm, step, dtype, cols):
    """Blocks of 64, 128 and 256 threads."""
    check(imm, step, many(), cols, dtype, group=128)
    check(imm, step, 3, cols, dtype, group=128)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cols", [1024, 6400])
def test_groups_with_float32_weights(imm, step, dtype, cols):
    check(imm, step, many(), cols, dtype, group=128, wdtype=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("grains", [1, 20, 30, 31, 62, 63, 126, 127, 500, 2046])
@pytest.mark.parametrize("x_at,q_at", [((1, 0), (0, 0)), ((3, 5), (2, 1))])
def test_rows_at_odd_addresses_alike(imm, step, dtype, grains, x_at, q_at):
    """x, residual and h at the same distance from a 16-byte boundary: their aligned granules."""
    cols = grains * (4 if dtype == torch.float32 else 8) + 1
    check(imm, step, many(), cols, dtype, x_at=x_at, q_at=q_at)


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 16379), (torch.bfloat16, 16381), (torch.bfloat16, 32751), (torch.float16, 32757),
                                        (torch.float32, 17001)])
def test_long_rows_at_odd_addresses_alike(imm, step, dtype, cols):
    check(imm, step, many(), cols, dtype, x_at=(1, 2))
    check(imm, step, 3, cols, dtype, x_at=(1, 2), wdtype=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [1, 100, 128, 129, 512, 513, 4096, 4097, 16384, 16385])
def test_rows_that_lie_unlike_one_another(imm, step, dtype, cols):
    """x, residual and h at different distances from a boundary: entry by entry."""
    for rows in (many(), 3):
        check(imm, step, rows, cols, dtype, x_at=(0, 0), r_at=(1, 0), h_at=(0, 3))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [128, 640, 4224])
def test_groups_at_odd_addresses(imm, step, dtype, cols):
    for rows in (many(), 3):
        check(imm, step, rows, cols, dtype, group=128, x_at=(1, 3), q_at=(5, 0))
        check(imm, step, rows, cols, dtype, group=128, x_at=(0, 0), r_at=(1, 0))


@pytest.mark.parametrize("dtype,cols", [(torch.int8, 8192), (torch.int8, 8208 + 16 * 512), (torch.bfloat16, 4096 + 8), (torch.float32, 2048 + 4)])
def test_dispatch_of_long_rows_several_to_a_block(imm, step, dtype, cols):
    tokens, top, experts = 8 * many() + 3, 2, 8
    x = randn((tokens, cols), 1, torch.float32, 20.0).to(dtype)
    ids = torch.randint(-1, experts, (tokens, top), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    rows, offsets, position, _, status = imm.moe_dispatch(x, ids, experts)
    want_o, want_p, source = step.dispatch(ids.cpu().numpy(), experts)
    assert offsets.cpu().tolist() == want_o.tolist() and np.array_equal(position.cpu().numpy(), want_p) and int(status) == 0
    token = torch.from_numpy(source // top).cuda()
    assert torch.equal(rows[:len(source)].view(torch.uint8), x[token].view(torch.uint8))
