"""Refusals of the cache, attention and verification calls that need no GPU: the library checks its arguments before it
touches a device (the pointers here are never dereferenced)."""
import os
import subprocess

import pytest
import torch

FAKE = 0x10000


@pytest.fixture(scope="module")
def imm():
    from paper_2602_22700_b200 import build, imm as binding
    build.build()
    return binding


def append(imm, k=FAKE, v=FAKE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, table=FAKE, offsets=FAKE, length=FAKE, status=FAKE, tokens=4, ldk=128, hsk=64,
           ldv=128, hsv=64, pages=10, kps=2048, vps=2048, ldt=5, batch=2, width=5, kv_heads=2, dim=64, page=16, dtype=None, r0=0, r1=0):
    return imm.lib().imm_kv_append(imm._APPEND_DESC.pack(*[p or 0 for p in (k, v, kc, vc, ks, vs, table, offsets, length, status)], tokens, ldk, hsk,
                                                         ldv, hsv, pages, kps, vps, ldt, batch, width, kv_heads, dim, page,
                                                         imm.BF16 if dtype is None else dtype, r0, r1), None)


SHAPES = (dict(tokens=-1), dict(tokens=(1 << 24) + 1), dict(batch=-1), dict(batch=(1 << 16) + 1), dict(kv_heads=0), dict(kv_heads=2000), dict(dim=0),
          dict(dim=72), dict(dim=272), dict(page=0), dict(page=8), dict(page=48), dict(page=256), dict(pages=0), dict(pages=1 << 31), dict(width=0),
          dict(width=1 << 27, ldt=1 << 27), dict(ldt=4), dict(kps=2032), dict(vps=2032))


def test_append_refusals(imm):
    assert imm.lib().imm_kv_append(None, None) == imm.ERR_ARG
    for bad in [{name: None} for name in ("k", "v", "kc", "vc", "ks", "vs", "table", "offsets", "length", "status")] + \
            [dict(dtype=imm.I8), dict(dtype=9), dict(r0=1)]:
        assert append(imm, **bad) == imm.ERR_ARG, bad
    for bad in SHAPES + (dict(ldk=63), dict(ldv=63), dict(hsk=63), dict(hsv=63)):
        assert append(imm, **bad) == imm.ERR_SHAPE, bad
    for bad in (dict(k=FAKE + 1), dict(v=FAKE + 1), dict(kc=FAKE + 8), dict(vc=FAKE + 8), dict(ks=FAKE + 2), dict(vs=FAKE + 2), dict(table=FAKE + 2),
                dict(offsets=FAKE + 4), dict(length=FAKE + 2), dict(status=FAKE + 2), dict(kps=2056), dict(dtype=imm.F32, k=FAKE + 2)):
        assert append(imm, **bad) == imm.ERR_ALIGN, bad
    assert append(imm, batch=0) == imm.OK and append(imm, batch=0, k=None, table=None, status=None) == imm.OK


def attention(imm, q=FAKE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, table=FAKE, offsets=FAKE, length=FAKE, out=FAKE, lse=FAKE, ws=FAKE, nws=1 << 40,
              tokens=4, ldq=256, hsq=64, ldo=256, hso=64, pages=10, kps=2048, vps=2048, ldt=5, batch=2, width=5, heads=4, kv_heads=2, dim=64,
              page=16, dtype=None, window=0, sinks=0, scale=0.1, r0=0, r1=0):
    return imm.lib().imm_kv_attention(imm._ATTENTION_DESC.pack(*[p or 0 for p in (q, kc, vc, ks, vs, table, offsets, length, out, lse, ws)], nws, tokens,
                                                               ldq, hsq, ldo, hso, pages, kps, vps, ldt, batch, width, heads, kv_heads, dim, page,
                                                               imm.BF16 if dtype is None else dtype, window, sinks, scale, r0, r1), None)


def test_attention_refusals(imm):
    assert imm.lib().imm_kv_attention(None, None) == imm.ERR_ARG
    for bad in [{name: None} for name in ("q", "kc", "vc", "ks", "vs", "table", "offsets", "length", "out")] + \
            [dict(dtype=imm.I32), dict(dtype=-1), dict(r0=1), dict(r1=1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
             dict(scale=float("nan")), dict(window=-1), dict(sinks=-1)]:
        assert attention(imm, **bad) == imm.ERR_ARG, bad
    for bad in SHAPES + (dict(heads=3), dict(heads=0), dict(heads=2000, kv_heads=2), dict(ldq=63), dict(hsq=63), dict(ldo=63), dict(hso=63)):
        assert attention(imm, **bad) == imm.ERR_SHAPE, bad
    for bad in (dict(q=FAKE + 1), dict(kc=FAKE + 8), dict(vc=FAKE + 4), dict(ks=FAKE + 2), dict(vs=FAKE + 1), dict(table=FAKE + 2), dict(offsets=FAKE + 4),
                dict(length=FAKE + 2), dict(out=FAKE + 1), dict(lse=FAKE + 2), dict(ws=FAKE + 8), dict(vps=2056), dict(dtype=imm.F32, q=FAKE + 2)):
        assert attention(imm, **bad) == imm.ERR_ALIGN, bad
    need = imm.lib().imm_kv_attention_workspace(4, 2, 4, 2, 64, imm.BF16)
    assert need > 0
    assert attention(imm, ws=None) == imm.ERR_WORKSPACE and attention(imm, nws=need - 1) == imm.ERR_WORKSPACE
    assert attention(imm, batch=0, ws=None) == imm.OK and attention(imm, tokens=0, q=None, out=None, ws=None) == imm.OK
    for bad in ((-1, 2, 4, 2, 64, imm.BF16), (4, -1, 4, 2, 64, imm.BF16), (4, 2, 5, 2, 64, imm.BF16), (4, 2, 4, 2, 60, imm.BF16), (4, 2, 4, 2, 64, imm.I8)):
        assert imm.lib().imm_kv_attention_workspace(*bad) == 0


def test_attention_rows_per_key_head_are_limited(imm):
    """Rows of a key head, tokens * heads / kv_heads, are counted in 32 bits."""
    most = dict(tokens=1 << 24, heads=64, kv_heads=1, nws=0)
    assert attention(imm, **most) == imm.ERR_WORKSPACE                 # (2^30 of them are within the limit)
    assert attention(imm, **{**most, "heads": 65}) == imm.ERR_SHAPE
    assert imm.lib().imm_kv_attention_workspace(1 << 24, 1, 64, 1, 64, imm.BF16) > 0
    assert imm.lib().imm_kv_attention_workspace(1 << 24, 1, 65, 1, 64, imm.BF16) == 0


def verify(imm, target=FAKE, draft=FAKE, tokens=FAKE, offsets=FAKE, u=FAKE, temp=None, accepted=FAKE, token=FAKE, logprob=FAKE, status=FAKE, requests=2,
           rows=6, drafts=4, n=100, ldt=100, ldd=100, temperature=1.0, dtype=None, r0=0, r1=0):
    return imm.lib().imm_verify_draft(imm._VERIFY_DESC.pack(*[p or 0 for p in (target, draft, tokens, offsets, u, temp, accepted, token, logprob, status)],
                                                            requests, rows, drafts, n, ldt, ldd, temperature, imm.F32 if dtype is None else dtype, r0, r1), None)


def test_verify_refusals(imm):
    assert imm.lib().imm_verify_draft(None, None) == imm.ERR_ARG
    for bad in [{name: None} for name in ("target", "tokens", "offsets", "u", "accepted", "token", "logprob", "status")] + \
            [dict(dtype=imm.I8), dict(dtype=7), dict(r0=1), dict(r1=1)]:
        assert verify(imm, **bad) == imm.ERR_ARG, bad
    for bad in (dict(requests=-1), dict(requests=(1 << 20) + 1), dict(rows=-1), dict(rows=(1 << 27) + 1), dict(drafts=-1), dict(n=0), dict(n=(1 << 20) + 1, ldt=1 << 21),
                dict(ldt=99), dict(ldd=99)):
        assert verify(imm, **bad) == imm.ERR_SHAPE, bad
    for bad in (dict(target=FAKE + 2), dict(draft=FAKE + 1), dict(tokens=FAKE + 2), dict(offsets=FAKE + 4), dict(u=FAKE + 4), dict(temp=FAKE + 2),
                dict(accepted=FAKE + 1), dict(token=FAKE + 2), dict(logprob=FAKE + 3), dict(status=FAKE + 2), dict(dtype=imm.F16, target=FAKE + 1)):
        assert verify(imm, **bad) == imm.ERR_ALIGN, bad
    assert verify(imm, requests=0) == imm.OK and verify(imm, requests=0, target=None, offsets=None, status=None) == imm.OK


def test_packed_structs_are_the_headers(imm, tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    (tmp_path / "s.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "imm.h"\nint main(void) { printf("%zu %zu %zu %zu", '
                                  'sizeof(imm_kv_append_desc), sizeof(imm_kv_attention_desc), sizeof(imm_verify_desc), '
                                  'offsetof(imm_kv_attention_desc, scale)); return 0; }\n')
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")])
    sizes = [int(v) for v in subprocess.check_output([str(tmp_path / "s")]).split()]
    assert sizes == [imm._APPEND_DESC.size, imm._ATTENTION_DESC.size, imm._VERIFY_DESC.size, imm._ATTENTION_DESC.size - 12]


def test_binding_refuses_cpu_tensors(imm):
    x, i = torch.zeros((2, 1, 16)), torch.zeros((1, 1), dtype=torch.int32)
    cache = (torch.zeros((1, 1, 16, 16), dtype=torch.int8), torch.zeros((1, 1, 16, 16), dtype=torch.int8), torch.zeros((1, 1)), torch.zeros((1, 1)))
    offsets = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError):
        imm.kv_append(x, x, cache, i, offsets, i.view(-1))
    with pytest.raises(ValueError):
        imm.kv_attention(x, cache, i, offsets, i.view(-1))
    with pytest.raises(ValueError):
        imm.kv_attention_workspace(x, cache, i, offsets)
    with pytest.raises(ValueError):
        imm.verify_draft(torch.zeros((2, 8)), None, i.view(-1), offsets, torch.zeros(2, dtype=torch.float64))
