"""No-GPU checks of the paged cache in 4 bits: its arena's arithmetic, what it refuses before it touches a GPU, the model's codes."""
import ctypes as C

import pytest
import torch

import paper_2505_13109_amd as fkv
from paged_model import Model, kept
from paper_2505_13109_amd.binding import CacheConfig


def _cfg(**kw):
    base = dict(n_layers=2, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=32, max_seqs=16, max_ctx=4096, n_pages=1000, dtype=1)
    base.update(kw)
    return CacheConfig(**base)


def test_arena_and_config():
    L = fkv.lib()
    need = C.c_size_t()
    assert L.fkv_cache_arena_bytes(C.byref(_cfg()), C.byref(need)) == 0
    pool, opens = 2 * 1000 * 8 * 5120, 2 * 16 * 8 * 16384
    assert pool + opens <= need.value < (pool + opens) * 1.4
    big = C.c_size_t()
    assert L.fkv_cache_arena_bytes(C.byref(_cfg(n_layers=80, n_pages=80000)), C.byref(big)) == 0
    assert big.value > 80 * 80000 * 8 * 5120 > 2 ** 32                # (sizes past 32 bits)
    for bad in (dict(head_dim=64), dict(page_size=16), dict(n_q_heads=30), dict(n_q_heads=136, n_kv_heads=8), dict(n_layers=0), dict(n_kv_heads=0),
                dict(max_seqs=0), dict(max_seqs=4097), dict(max_ctx=100), dict(max_ctx=0), dict(max_ctx=1 << 23), dict(n_pages=0), dict(dtype=2)):
        assert L.fkv_cache_arena_bytes(C.byref(_cfg(**bad)), C.byref(need)) == -1, bad
        assert L.fkv_cache_last_error(None)
    assert L.fkv_cache_arena_bytes(None, C.byref(need)) == -1


def test_as_many_open_pages_as_a_copy_has_blocks_for():
    L = fkv.lib()
    need = C.c_size_t()
    assert L.fkv_cache_arena_bytes(C.byref(_cfg(n_layers=256, max_seqs=4096, n_kv_heads=8)), C.byref(need)) == 0 and need.value > 2 ** 37
    assert (256 * 4096 * 8 + 2 ** 20) * 256 < 2 ** 32
    for more in (dict(n_layers=257, max_seqs=4096), dict(n_layers=512, max_seqs=4096), dict(n_layers=4096, max_seqs=4096, n_kv_heads=1, n_q_heads=1)):
        assert L.fkv_cache_arena_bytes(C.byref(_cfg(**more)), C.byref(need)) == -1, more
        assert b"open pages" in L.fkv_cache_last_error(None)


def test_create_refuses_bad_arenas_without_touching_the_gpu():
    L = fkv.lib()
    h = C.c_void_p()
    assert L.fkv_cache_create(C.byref(_cfg()), None, 1 << 40, C.byref(h)) == -1
    assert L.fkv_cache_create(C.byref(_cfg()), C.c_void_p(0x1000101), 1 << 40, C.byref(h)) == -1
    assert L.fkv_cache_create(C.byref(_cfg()), C.c_void_p(0x1000100), 16, C.byref(h)) == -4
    assert L.fkv_cache_create(C.byref(_cfg()), C.c_void_p(0x1000100), 1 << 40, None) == -1
    assert not h.value
    assert L.fkv_cache_destroy(None) == -1 and L.fkv_cache_health(None) == -1 and L.fkv_cache_used_pages(None) == -1
    assert L.fkv_cache_extend(None, None, 0, None, None) == -1 and L.fkv_cache_copy(None, None, None, None, 0, None) == -1


def test_binding_without_gpu_fails_loudly():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(fkv.FreeKVError, match="no GPU"):
        fkv.PagedCache(n_layers=1, n_q_heads=4, n_kv_heads=1, max_seqs=1, max_ctx=64, n_pages=4)
    with pytest.raises(fkv.FreeKVError, match="head_dim"):
        fkv.PagedCache(n_layers=1, n_q_heads=4, n_kv_heads=1, max_seqs=1, max_ctx=64, n_pages=4, head_dim=64)


def test_the_models_values_are_within_half_a_step():
    x = torch.randn((32, 2, 128), generator=torch.Generator().manual_seed(1)).bfloat16()
    value, lo, step = kept(x)
    # half a step, and what 15 roundings of the step to fp16 leave at the top of the range
    assert ((value - x.double()).abs() <= step * (0.5 + 15 * 2.0 ** -11)).all()
    assert torch.equal(lo, x.double().min(0).values) and (step > 0).all()
    same = kept(torch.ones((32, 1, 128)).bfloat16() * 3)
    assert (same[0] == 3).all() and not same[2].any()


def test_the_models_pages():
    m = Model(n_layers=1, n_kv=1, max_seqs=4, max_ctx=256, n_pages=6, dtype=torch.bfloat16)
    assert m.extend([0, 1], [64, 40]) and m.pages == [[0, 1], [2], [], []] and m.used() == 3
    m.fork([0], [2])
    m.free([0])
    assert m.used() == 3 and m.extend([3], [33]) and m.pages[3] == [3]
    m.free([2])
    m.compact()
    assert m.pages == [[], [0], [], [1]] or m.pages == [[], [1], [], [0]]
    assert not m.extend([0], [200])
