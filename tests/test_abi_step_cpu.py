"""Refusals of the calls between products and of token sampling that need no GPU: the library checks its
arguments before it touches a device (the pointers here are never dereferenced)."""
import pytest
import torch

FAKE = 0x10000


@pytest.fixture(scope="module")
def imm():
    from paper_2602_22700_b200 import build, imm as binding
    build.build()
    return binding


def sample(imm, logits=FAKE, dtype=None, steps=4, n=100, ld=100, u=FAKE, token=FAKE, logprob=FAKE, kept=FAKE, status=FAKE, d_temperature=0,
           d_top_p=0, d_min_p=0, d_top_k=0, reserved=0):
    return imm.lib().imm_sample(imm._SAMPLE_DESC.pack(logits or 0, u or 0, token or 0, logprob or 0, kept or 0, status or 0, d_temperature, d_top_p,
                                                      d_min_p, d_top_k, steps, n, ld, 1.0, 1.0, 0.0, 0, imm.F32 if dtype is None else dtype,
                                                      reserved), None)


def test_sample_refusals(imm):
    for name in ("logits", "u", "token", "logprob", "kept", "status"):
        assert sample(imm, **{name: None}) == imm.ERR_ARG
    assert imm.lib().imm_sample(None, None) == imm.ERR_ARG and sample(imm, reserved=1) == imm.ERR_ARG
    for dtype in (imm.I8, imm.I32, 5, -1):
        assert sample(imm, dtype=dtype) == imm.ERR_ARG
    for bad in (dict(steps=-1), dict(n=0), dict(n=-3), dict(ld=99), dict(n=(1 << 20) + 1, ld=1 << 21), dict(steps=(1 << 27) + 1)):
        assert sample(imm, **bad) == imm.ERR_SHAPE
    for name, off in (("logits", 2), ("u", 4), ("token", 2), ("logprob", 1), ("kept", 3), ("status", 2), ("d_temperature", 2), ("d_top_p", 1),
                      ("d_min_p", 2), ("d_top_k", 2)):
        assert sample(imm, **{name: FAKE + off}) == imm.ERR_ALIGN
    assert sample(imm, dtype=imm.BF16, logits=FAKE + 1) == imm.ERR_ALIGN
    assert sample(imm, steps=0) == imm.OK and sample(imm, steps=0, logits=None, u=None, token=None) == imm.OK


def norm(imm, x=FAKE, res=None, w=FAKE, dtype=None, wdtype=None, rows=4, cols=256, ldx=256, ldr=256, ldh=256, ldq=256, eps=1e-6, group=0,
         h=None, q=FAKE, scale=FAKE):
    return imm.lib().imm_rmsnorm_quant(imm._NORM_DESC.pack(x or 0, res or 0, w or 0, h or 0, q or 0, scale or 0, rows, cols, ldx, ldr, ldh, ldq, eps,
                                                           imm.BF16 if dtype is None else dtype, imm.BF16 if wdtype is None else wdtype,
                                                           group, 0), None)


def test_norm_refusals(imm):
    for bad in (dict(x=None), dict(w=None), dict(q=None), dict(scale=None), dict(res=FAKE), dict(dtype=imm.I8), dict(dtype=9), dict(wdtype=imm.F16),
                dict(wdtype=imm.I32), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(group=64), dict(group=-1)):
        assert norm(imm, **bad) == imm.ERR_ARG, bad
    for bad in (dict(rows=-1), dict(cols=0), dict(cols=(1 << 20) + 1), dict(ldx=255), dict(ldq=255), dict(res=FAKE, h=FAKE, ldr=255),
                dict(h=FAKE, ldh=255), dict(rows=(1 << 30) + 1), dict(cols=200, group=128)):
        assert norm(imm, **bad) == imm.ERR_SHAPE, bad
    for bad in (dict(x=FAKE + 1), dict(w=FAKE + 1), dict(wdtype=imm.F32, w=FAKE + 2), dict(res=FAKE + 1, h=FAKE), dict(h=FAKE + 1),
                dict(scale=FAKE + 2)):
        assert norm(imm, **bad) == imm.ERR_ALIGN, bad
    assert norm(imm, rows=0) == imm.OK and norm(imm, rows=0, x=None, q=None) == imm.OK


def dispatch(imm, x=FAKE, scale=None, expert=FAKE, tokens=4, top=2, experts=8, cols=64, es=2, ldx=64, ldo=64, out_rows=8, out=FAKE, oscale=None,
             offsets=FAKE, position=FAKE, status=FAKE, ws=None, nws=0):
    return imm.lib().imm_moe_dispatch(imm._DISPATCH_DESC.pack(x or 0, scale or 0, expert or 0, out or 0, oscale or 0, offsets or 0, position or 0,
                                                              status or 0, ws or 0, nws, tokens, cols, ldx, ldo, out_rows, top, experts, es, 0),
                                      None)


def test_dispatch_refusals(imm):
    for bad in (dict(x=None), dict(expert=None), dict(out=None), dict(offsets=None), dict(position=None), dict(status=None), dict(scale=FAKE),
                dict(oscale=FAKE), dict(es=0), dict(es=3), dict(es=8)):
        assert dispatch(imm, **bad) == imm.ERR_ARG, bad
    for bad in (dict(tokens=-1), dict(top=0), dict(top=65), dict(experts=0), dict(experts=1025), dict(cols=0), dict(cols=(1 << 20) + 1), dict(ldx=63),
                dict(ldo=63), dict(out_rows=7), dict(tokens=1 << 26, out_rows=1 << 40)):
        assert dispatch(imm, **bad) == imm.ERR_SHAPE, bad
    for bad in (dict(x=FAKE + 1), dict(out=FAKE + 1), dict(expert=FAKE + 2), dict(offsets=FAKE + 4), dict(position=FAKE + 2), dict(status=FAKE + 1),
                dict(scale=FAKE + 1, oscale=FAKE), dict(ws=FAKE + 8)):
        assert dispatch(imm, **bad) == imm.ERR_ALIGN, bad
    need = imm.moe_dispatch_workspace(100000, 8, 64)
    assert need > 0
    big = dict(tokens=100000, top=8, experts=64, out_rows=800000)
    assert dispatch(imm, **big) == imm.ERR_WORKSPACE
    assert dispatch(imm, **big, ws=FAKE, nws=need - 1) == imm.ERR_WORKSPACE
    assert imm.moe_dispatch_workspace(-1, 2, 8) == imm.moe_dispatch_workspace(4, 65, 8) == imm.moe_dispatch_workspace(4, 2, 2000) == 0


def combine(imm, y=FAKE, dtype=None, rs=None, position=FAKE, weight=None, tokens=4, top=2, cols=64, y_rows=8, ldy=64, ldo=64, odtype=None, out=FAKE):
    return imm.lib().imm_moe_combine(imm._COMBINE_DESC.pack(y or 0, rs or 0, position or 0, weight or 0, out or 0, tokens, cols, y_rows, ldy, ldo, top,
                                                            imm.I32 if dtype is None else dtype, imm.BF16 if odtype is None else odtype, 0), None)


def test_combine_refusals(imm):
    for bad in (dict(y=None), dict(position=None), dict(out=None), dict(dtype=imm.I8), dict(odtype=imm.I32), dict(odtype=7)):
        assert combine(imm, **bad) == imm.ERR_ARG, bad
    for bad in (dict(tokens=-1), dict(top=0), dict(top=65), dict(cols=0), dict(ldy=63), dict(ldo=63), dict(y_rows=-1)):
        assert combine(imm, **bad) == imm.ERR_SHAPE, bad
    for bad in (dict(y=FAKE + 2), dict(out=FAKE + 1), dict(rs=FAKE + 1), dict(position=FAKE + 2), dict(weight=FAKE + 3)):
        assert combine(imm, **bad) == imm.ERR_ALIGN, bad
    assert combine(imm, tokens=0) == imm.OK and combine(imm, tokens=0, y=None, position=None, out=None) == imm.OK


def test_packed_structs_are_the_headers(imm):
    """Sizes of the packed argument structs as a C compiler lays them out."""
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = '#include <stdio.h>\n#include "imm.h"\nint main(void) { printf("%zu %zu %zu %zu", sizeof(imm_sample_desc), sizeof(imm_norm_desc), ' \
           'sizeof(imm_dispatch_desc), sizeof(imm_combine_desc)); return 0; }\n'
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "s.c"), "w") as f:
            f.write(code)
        subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), os.path.join(d, "s.c"), "-o", os.path.join(d, "s")])
        sizes = [int(v) for v in subprocess.check_output([os.path.join(d, "s")]).split()]
    assert sizes == [imm._SAMPLE_DESC.size, imm._NORM_DESC.size, imm._DISPATCH_DESC.size, imm._COMBINE_DESC.size]
    big = 1 << 20                                    # the binding allocates a workspace from the same size on as the library
    assert imm.moe_dispatch_workspace(imm.MOE_RUN, 1, 8) == 0 and imm.moe_dispatch_workspace(imm.MOE_RUN + 1, 1, 8) > 0
    assert imm.moe_dispatch_workspace(big, 2, 8) > 0


def test_binding_refuses_cpu_tensors(imm):
    x = torch.zeros((2, 8))
    with pytest.raises(ValueError):
        imm.sample(x, torch.zeros(2, dtype=torch.float64))
    with pytest.raises(ValueError):
        imm.rmsnorm_quant(x, torch.ones(8))
    with pytest.raises(ValueError):
        imm.moe_dispatch(x, torch.zeros((2, 1), dtype=torch.int32), 4)
    with pytest.raises(ValueError):
        imm.moe_combine(x, torch.zeros((2, 1), dtype=torch.int32))
