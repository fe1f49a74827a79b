"""The rule that chooses a grouped product's kernel (host code; no GPU is used)."""

import pytest

from tests import grouped_plans as P


@pytest.mark.parametrize("k_bytes", P.DEPTHS)
@pytest.mark.parametrize("up", [False, True])
@pytest.mark.parametrize("dtype", list(P.DT))
@pytest.mark.parametrize("name", list(P.KINDS))
def test_every_kernel_has_a_case(name, dtype, up, k_bytes):
    assert P.case(name, dtype, up, k_bytes) is not None
    assert P.case(name, dtype, up, k_bytes, 30, 2) is not None


@pytest.mark.parametrize("dtype", list(P.DT))
def test_gathered_rows_past_4_gib_leave_the_large_tiles(dtype):
    """their offsets have 32 bits"""
    sizes, d_out, d_in = [2048] * 16, 4096, 2048 // P.BYTES[dtype]
    rows = 2 ** 32 // 2048
    assert P.plan(dtype, False, sizes, d_in, d_out, 1, rows - 1).kernel == P.TILES
    assert P.plan(dtype, False, sizes, d_in, d_out, 1, rows).kernel == P.RING
    assert P.plan(dtype, False, sizes, d_in, d_out, 0, 4 * rows).kernel == P.TILES
