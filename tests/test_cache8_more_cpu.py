"""The paged 8-bit cache without a GPU: clusters of the eviction, limits of how an attention is split."""
import ctypes as C

import pytest

from test_cache8_cpu import ONE, cache


# device: what one holds is asked once, so that each case takes another
@pytest.mark.parametrize("device,units,resident,size", [
    (23, 18, {8: 15, 4: 33, 2: 74}, 4), (24, 15, {8: 15, 4: 33, 2: 74}, 8), (25, 34, {8: 15, 4: 33, 2: 74}, 2), (26, 4, {8: 0, 4: 30, 2: 74}, 4),
    (27, 4, {8: 0, 4: 0, 2: 0}, 1)])
def test_clusters_of_an_eviction_are_resident_at_once(fake_cuda, device, units, resident, size):
    fake_cuda.reset(device=device, resident=resident)
    c, into = cache(batch=1, kv_heads=units, max_pages=1024), cache(batch=1, kv_heads=units, rows=ONE + 1024)
    assert fake_cuda.lib.mixkv_cache_evict(C.byref(c), C.byref(into), 4096, None, 1, 1, 65536, ONE, None, None) == 0
    pick = fake_cuda.launches()[0]
    assert pick.kernel == "k_cache8_pick" and pick.cluster == size and pick.grid == units * size
