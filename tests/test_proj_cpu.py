"""No-GPU checks of the projections in 8 bits: what they refuse before they touch a GPU, and the model's codes."""
import ctypes as C

import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M

P = 0x1000100          # an address that no call may read


def refused(rc, code, word):
    assert rc == code, rc
    assert word in fkv.lib().fkv_proj_last_error().decode()


def test_refusals_of_the_entry_points():
    L = fkv.lib()
    quant = lambda dtype=1, x=P, rows=4, cols=256, tile=1, codes=P, scales=P: L.fkv_proj_quant(0, dtype, x, rows, cols, tile, codes, scales, None)
    refused(quant(dtype=2), -1, "dtype")
    refused(quant(rows=-1), -3, "rows")
    refused(quant(rows=4194305), -3, "rows")
    for cols in (0, 8, 17, 131088, -16):
        refused(quant(cols=cols), -3, "cols")
    refused(quant(tile=2), -1, "tile")
    for bad in (dict(x=None), dict(x=P + 8), dict(codes=None), dict(codes=P + 4), dict(scales=None), dict(scales=P + 1)):
        refused(quant(**bad), -1, "aligned")
    assert quant(rows=0, x=None, codes=None, scales=None) == 0

    norm = lambda x=P, add=P, weight=P, rows=4, cols=256, eps=1e-5, res=P, codes=P, scales=P, out=P, dtype=1: L.fkv_proj_norm(
        0, dtype, x, add, weight, rows, cols, eps, res, codes, scales, out, None)
    for eps in (0.0, -1.0, 1e-39, float("inf"), float("nan")):
        refused(norm(eps=eps), -1, "eps")
    refused(norm(codes=None), -1, "together")
    refused(norm(scales=None), -1, "together")
    refused(norm(add=None), -1, "add")
    refused(norm(codes=None, scales=None, out=None, add=None, res=None), -1, "nothing")
    refused(norm(dtype=-1), -1, "dtype")
    refused(norm(cols=24), -3, "cols")
    for name in ("x", "add", "weight", "res", "codes", "scales", "out"):
        refused(norm(**{name: P + 2}), -1, "aligned")
    refused(norm(x=None), -1, "x")
    assert norm(rows=0) == 0

    gate = lambda gu=P, rows=4, cols=256, codes=P, scales=P, dtype=0: L.fkv_proj_gate(0, dtype, gu, rows, cols, codes, scales, None)
    refused(gate(gu=None), -1, "gu")
    refused(gate(cols=40), -3, "cols")
    refused(gate(scales=P + 4), -1, "aligned")
    refused(gate(dtype=7), -1, "dtype")

    axes = lambda *v: (C.c_int32 * 64)(*v)
    rope = lambda qkv=P, rows=4, n_q=4, n_kv=2, pos=P, n_axes=2, axis_of=None, freq=P, q=P, k=P, v=P, dtype=1: L.fkv_proj_rope(
        0, dtype, qkv, rows, n_q, n_kv, pos, n_axes, axis_of, freq, q, k, v, None)
    for bad in (dict(n_q=0), dict(n_kv=0), dict(n_q=4097), dict(n_kv=-1)):
        refused(rope(**bad), -1, "n_q and n_kv")
    for n in (0, 5):
        refused(rope(n_axes=n), -1, "n_axes")
    refused(rope(axis_of=axes(0, 1, 2)), -1, "axis_of")
    refused(rope(axis_of=axes(0, -1)), -1, "axis_of")
    for name in ("qkv", "q", "k", "v", "pos", "freq"):
        refused(rope(**{name: None}), -1, "null")
        refused(rope(**{name: P + 4}), -1, "aligned")

    need = C.c_size_t()
    matmul = lambda x=P, xs=P, w=P, ws=P, rows=4, n=300, cols=256, out=P, work=None, size=0, dtype=1: L.fkv_proj_matmul(
        0, dtype, x, xs, w, ws, rows, n, cols, out, work, size, None)
    for n in (0, -1, 4194305):
        refused(matmul(n=n), -3, "n must be")
        refused(L.fkv_proj_workspace(4, n, 256, C.byref(need)), -3, "n must be")
    refused(matmul(cols=100), -3, "cols")
    refused(matmul(rows=-5), -3, "rows")
    refused(L.fkv_proj_workspace(4, 4, 100, C.byref(need)), -3, "cols")
    refused(L.fkv_proj_workspace(4, 4, 128, None), -1, "null")
    for name in ("x", "xs", "w", "ws", "out"):
        refused(matmul(**{name: None}), -1, "null")
        refused(matmul(**{name: P + 8}), -1, "aligned")
    assert matmul(rows=0) == 0
    assert L.fkv_proj_workspace(0, 4, 128, C.byref(need)) == 0 and need.value == 0


def test_a_product_asks_for_the_workspace_that_it_needs():
    L = fkv.lib()
    need = C.c_size_t()
    found = 0
    for rows in (1, 16, 17, 64, 128, 203, 256, 1000, 4096, 1 << 17):
        for n, cols in ((16, 16), (4096, 4096), (4096, 14336), (28672, 4096), (32768, 131072)):
            assert L.fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0
            if need.value:
                found += 1
                call = lambda work, size: L.fkv_proj_matmul(0, 1, P, P, P, P, rows, n, cols, P, work, size, None)
                refused(call(P, need.value - 1), -4, "workspace")
                refused(call(None, need.value), -1, "work")
                refused(call(P + 8, need.value), -1, "work")
    print("sizes with a workspace:", found)


def test_the_binding_refuses_what_is_not_on_a_gpu():
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    codes, scales = fkv.empty_quant(4, 256, device="cpu")
    for call in (lambda: fkv.proj_quant(x, codes, scales), lambda: fkv.proj_norm(x, None, codes, scales), lambda: fkv.proj_gate(x, codes, scales),
                 lambda: fkv.proj_matmul(codes, scales, codes, scales, x)):
        with pytest.raises(fkv.FreeKVError, match="cpu"):
            call()
    with pytest.raises(fkv.FreeKVError, match="cpu"):
        fkv.proj_rope(torch.zeros((4, 6, 128), dtype=torch.float16), None, None, torch.zeros(4, 4, 128), torch.zeros(4, 1, 128), None)
    for bad in (x.float(), x[:, ::2], x[0], None):
        with pytest.raises(fkv.FreeKVError, match="wanted"):
            fkv.proj_quant(bad, codes, scales)


def test_sections():
    from paper_2505_13109_amd.projection import _axis_of
    assert list(_axis_of((16, 24, 24), 3)) == [0] * 16 + [1] * 24 + [2] * 24
    assert list(_axis_of([i % 3 for i in range(64)], 3)) == [i % 3 for i in range(64)]
    assert _axis_of(None, 2) is None and list(_axis_of((64,), 1)) == [0] * 64
    for bad, axes in (((16, 24), 2), ((16, 24, 24), 2), ((70, -6), 2), ([3] * 64, 3), ([-1] + [0] * 63, 2), ((), 1)):
        with pytest.raises(fkv.FreeKVError, match="sections"):
            _axis_of(bad, axes)


def test_more_sections_than_are_kept_from_several_threads():
    from concurrent.futures import ThreadPoolExecutor
    from paper_2505_13109_amd.projection import _axis_of

    def ask(first):
        return all(list(_axis_of((n, 64 - n), 2)) == [0] * n + [1] * (64 - n) for i in range(30) for n in range(first, 65))

    with ThreadPoolExecutor(8) as pool:
        assert all(pool.map(ask, range(8)))


def test_the_models_codes_are_the_types():
    """All e4m3 numbers, and what lies between them, against the type's own conversion (which rounds to even)."""
    every = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(M.nearest_e4m3(every), every) and every[-1] == 448
    between = (every[:-1] + every[1:]) / 2
    for q in (between, between * (1 - 2.0 ** -20), between * (1 + 2.0 ** -20)):
        assert torch.equal(M.nearest_e4m3(q), q.float().to(torch.float8_e4m3fn).double())
        assert torch.equal(M.nearest_e4m3(-q), -M.nearest_e4m3(q))
    x = torch.randn((130, 200), generator=torch.Generator().manual_seed(1)).double()
    for tile in (1, 128):
        codes, scales = M.quant(x, tile)
        assert ((M.values(codes, scales, tile) - x).abs() <= x.abs() * 2.0 ** -4 + M.spread(scales, 130, 200, tile) * 2.0 ** -10).all()


def test_the_binding_refuses_what_is_no_tensor():
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    for call in (lambda: fkv.proj_quant(x, None, None), lambda: fkv.proj_norm(x, 1.0, None, None, out=3), lambda: fkv.proj_gate([1], None, None),
                 lambda: fkv.proj_matmul(None, None, None, None, None), lambda: fkv.proj_matmul(x, x, x, x, "out"), lambda: fkv.proj_rope(x, 1, 2, 3, 4, 5)):
        with pytest.raises(fkv.FreeKVError):
            call()
