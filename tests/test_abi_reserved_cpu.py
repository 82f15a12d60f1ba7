"""Reserved fields of the cache, attention and verification calls must be 0, each of them (no GPU: the pointers are never dereferenced)."""
import pytest

from test_abi_cache_cpu import append, attention, imm, verify  # noqa: F401


@pytest.mark.parametrize("call", [append, attention, verify])
def test_reserved_fields_are_refused(imm, call):  # noqa: F811
    for value in (1, -1, 1 << 30):
        for field in ("r0", "r1"):
            assert call(imm, **{field: value}) == imm.ERR_ARG, (field, value)
