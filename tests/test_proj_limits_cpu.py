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


@pytest.mark.parametrize("n,cols", [(1, 16), (16, 128), (900, 640), (512, 8192), (4096, 4096), (4096, 14336), (28672, 4096), (32768, 131072), (3001, 2192), (17, 131072)])
def test_workspaces_are_of_whole_parts(n, cols):
    """None up to 32 rows (the binding relies on it), and beyond that 2 to 16 sums in fp32 of each result, columns in fours."""
    L, need = fkv.lib(), C.c_size_t()
    for rows in range(0, 33):
        assert L.fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0 and need.value == 0
    for rows in (33, 48, 64, 65, 120, 128, 200, 300, 1000, 4096, 1 << 17):
        assert L.fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0
        parts, rest = divmod(need.value, 4 * rows * (-(-n // 4) * 4))
        assert rest == 0 and (parts == 0 or 2 <= parts <= 16) and parts <= -(-cols // 128)


def test_there_are_products_in_parts():
    L, need, found = fkv.lib(), C.c_size_t(), []
    for rows, n, cols in ((200, 512, 8192), (203, 4096, 11056), (128, 4096, 14336), (300, 300, 4096), (120, 900, 8192)):
        assert L.fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0
        found.append(need.value)
    assert all(found), found
