"""No-GPU checks of the projections' limits: what one launch can hold, and when a product asks for a workspace."""
import ctypes as C

import pytest

import paper_2505_13109_amd as fkv
from test_proj_cpu import P, refused


# rows, blocks of 128: their product is the limit, 2^28 - 16, or one of the 15 above it.  A launch has 16 threads a block of 128 in blocks of 256, so
# from 2^28 - 15 on that would be 2^32 of them.
@pytest.mark.parametrize("rows,blocks", [(326167, 823), (2375535, 113), (3085465, 87)])
def test_what_one_launch_cannot_hold_is_refused(rows, blocks):
    assert rows * blocks > (1 << 28) - 16 and (rows * blocks * 16 + 255) // 256 * 256 >= 1 << 32
    L, cols = fkv.lib(), blocks * 128
    refused(L.fkv_proj_quant(0, 1, P, rows, cols, 1, P, P, None), -3, "rows x ceil")
    refused(L.fkv_proj_gate(0, 1, P, rows, cols, P, P, None), -3, "rows x ceil")


def test_what_one_launch_can_hold_is_not():
    L, need = fkv.lib(), C.c_size_t()
    for rows, blocks in ((1, 1024), ((1 << 18) - 1, 1024), (4194303, 64), (2236961, 120)):
        assert rows * blocks <= (1 << 28) - 16
        assert L.fkv_proj_workspace(rows, 16, blocks * 128, C.byref(need)) == 0, (rows, blocks)
