"""No-GPU check of where a paged cache may be."""
import pytest

import paper_2505_13109_amd as fkv


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_a_cache_is_not_put_on_a_gpu_where_another_device_is_named(device):
    with pytest.raises(fkv.FreeKVError, match="device"):
        fkv.PagedCache(n_layers=1, n_q_heads=4, n_kv_heads=1, max_seqs=1, max_ctx=64, n_pages=4, device=device)
