"""The paged 4-bit cache without a GPU: a limit of how an attention is split."""
import ctypes as C

import pytest

from paper_2510_20707_b200 import binding, build


@pytest.mark.parametrize("units,steps", [(1023, 2099202), (1024, 2097151), (1000, 2147483), (32, (1 << 26) - 1)])
@pytest.mark.parametrize("eights", [1, 2, 3, 4])
def test_shares_are_counted_in_32_bits(units, steps, eights):
    # CTAs that share all steps find their first and last ones with sums up to steps + CTAs, and warps go past the end by a CTA's number of them
    build.build()
    lib = binding.load_library()
    ctas, large, shared = (C.c_int32() for _ in range(3))
    resident = (C.c_int32 * 9)(*[148] * 9)
    lib.mixkv_internal_paged_shape(C.c_int64(units), 1, C.c_int64(steps), eights, 148, resident, resident, C.byref(ctas), C.byref(large),
                                   C.byref(shared))
    if shared.value:
        assert max(units * steps + shared.value - 1, shared.value * -(-units * steps // shared.value), units * steps + 16) < 1 << 31
    else:
        assert units * steps > (1 << 31) - 1000
