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
