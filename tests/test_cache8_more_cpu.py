"""The paged 8-bit cache without a GPU: clusters of the eviction, limits of how an attention is split."""
import ctypes as C

import pytest

from test_cache8_cpu import ONE, cache, lib  # noqa: F401


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


@pytest.mark.parametrize("units,tiles", [(1023, 2099202), (1024, 2097151), (1000, 2147483), (1, 1 << 26), (32, (1 << 26) - 1), (1009, 2128328)])
@pytest.mark.parametrize("eights,half", [(1, 0), (2, 0), (2, 1), (4, 1)])
def test_shares_are_counted_in_32_bits(lib, units, tiles, eights, half):
    # CTAs that share all tiles find their first and last ones with sums up to tiles + CTAs, and warps step past the end by four
    S, shared, resident = C.c_int32(), C.c_int32(), (C.c_int32 * 9)(*[148] * 9)
    lib.mixkv_internal_cache8_shape(C.c_int64(units), 1, C.c_int64(tiles), 0, eights, half, 148, resident, C.byref(S), C.byref(shared))
    if shared.value:
        share = -(-units * tiles // shared.value)
        assert max(units * tiles + shared.value - 1, (shared.value - 1) * share + share, units * tiles + 4) < 1 << 31
    else:      # a cluster for each
        assert units * tiles > (1 << 31) - 1000
