"""The paged 4-bit cache without a GPU: its plain definition, and what the entry points refuse before any CUDA call."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_plain as plain
from paper_2510_20707_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def test_e4m3_and_codes_against_torch():
    x = np.concatenate([np.linspace(0, 460, 4001), 2.0 ** np.linspace(-12, 9, 999), plain.E4M3[:0x7F],
                        (plain.E4M3[:0x7E] + plain.E4M3[1:0x7F]) / 2]).astype(np.float32)
    want = torch.from_numpy(np.minimum(x, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(plain.to_e4m3(x), want)
    # a block whose scale is 1: codes are the nearest grid values, ties to the even one
    row = np.zeros(128, np.float32)
    row[:16] = [6, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 4.99, -0.25, -0.75, -5, 5.01, 0.0, -0.0]
    codes, s = plain.quantise(row)
    assert plain.E4M3[s[0]] == 1.0
    assert plain.values(codes, s)[:16].tolist() == [6, 0, .5, 1, 1, 2, 2, 4, 4, 4, 0, -1, -4, 6, 0, 0]


def test_a_tile_holds_every_row_once():
    every = np.concatenate([plain.K_AT[:, ::2].ravel(), plain.V_AT[:, ::2].ravel(), plain.KS_AT.ravel(), plain.VS_AT.ravel()])
    assert np.array_equal(np.sort(every), np.arange(plain.TILE_BYTES))
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 37, 128)).astype(np.float32)
    (kc, ks), (vc, vs) = plain.quantise(x[0]), plain.quantise(x[1])
    pool = np.zeros((3, 2 * plain.TILE_BYTES), np.uint8)
    table = np.array([2, 0], np.int32)
    for r in range(37):
        plain.put_row(pool.reshape(-1, plain.TILE_BYTES)[table[r // 32] * 2 + r % 32 // 16], r % 16, kc[r], ks[r], vc[r], vs[r])
    k, v = plain.get_rows(pool, table, 32, 37)
    assert np.array_equal(k, plain.values(kc, ks)) and np.array_equal(v, plain.values(vc, vs))
    # a block's error is at most half of the grid's widest step (2, between 4 and 6) and what the scale's own rounding (2^-4)
    # leaves above 6
    s = plain.E4M3[ks].repeat(16, -1)
    assert (np.abs(k - x[0]) <= s * 1.0 + 1e-6).all()


def test_values_are_exact_in_sixteen_bits():
    c, s = np.meshgrid(np.arange(16, dtype=np.uint8), np.arange(0x7F, dtype=np.uint8))
    v = plain.CODE_VALUES[c] * plain.E4M3[s]
    assert np.array_equal(v.astype(np.float16).astype(np.float64), v)
    assert np.array_equal(torch.from_numpy(v).bfloat16().double().numpy(), v)


def test_attention_is_the_softmax_of_what_is_seen():
    rng = np.random.default_rng(1)
    q, K, V = rng.standard_normal((2, 3, 128)), rng.standard_normal((9, 128)), rng.standard_normal((9, 128))
    out, _, _ = plain.attention(q, K, V, 2, 0.1)
    for t in range(2):
        w = torch.softmax(torch.from_numpy(q[t] @ K[:8 + t].T * 0.1), 1).numpy()
        assert np.allclose(out[t], w @ V[:8 + t])
    assert (plain.attention(q, K[:1], V[:1], 2, 0.1)[0][0] == 0).all()


def test_scores_bound_the_products_and_order_pages():
    rng = np.random.default_rng(2)
    K = rng.standard_normal((6, 16, 128)).astype(np.float32)
    q = rng.standard_normal((5, 128)).astype(np.float32)
    s = plain.scores(q, K.min(1), K.max(1))
    assert (s + 1e-4 >= np.einsum("rd,pnd->rpn", q, K).max((0, 2))).all()
    assert plain.select(np.array([1.0, 5, 5, 0, 5]), 2, 0, 0) == [1, 2]
    assert plain.select(np.array([1.0, 5, 5, 0, 5]), 3, 1, 1) == [0, 1, 4]
    assert plain.select(np.array([1.0, 5, np.nan, 0, 5]), 2, 0, 0) == [1, 2]


def test_page_bytes(lib):
    assert binding.page_bytes(16) == 2304 and binding.page_bytes(256) == 16 * 2304
    for bad in (0, 8, 24, 272, -16):
        with pytest.raises(binding.MixKVError) as e:
            binding.page_bytes(bad)
        assert e.value.status == -1


ONE = C.c_void_p(256)


def pages(**kw):
    base = dict(pool=256, bounds_opt=256, table=256, rows=256, num_pages=100, max_pages=10, page_rows=64, batch=2, kv_heads=4,
                head_dim=128, k_scale=1.0, v_scale=1.0)
    base.update(kw)
    return C.byref(binding._CPages(**base))


def append(lib, c, **kw):
    a = dict(k=ONE, v=ONE, type=0, n=8, kr=512, kh=128, vr=512, vh=128, off=ONE, per=0, most=4, cos=None, sin=None, len=0, rot=0,
             inter=0, pos=None)
    a.update(kw)
    return lib.mixkv_paged_append(c, *a.values(), None, None)


def attend(lib, c, **kw):
    a = dict(q=ONE, type=0, qb=2048, qt=2048, T=1, G=4, scale=0.0, rows=600, list=None, counts=None, top=0, ws=ONE, bytes=1 << 40, out=ONE)
    a.update(kw)
    return lib.mixkv_paged_attention(c, *a.values(), None)


def select(lib, c, **kw):
    a = dict(q=ONE, type=0, qb=2048, qt=2048, T=1, G=4, rows=600, top=4, first=0, last=0, list=ONE, counts=ONE)
    a.update(kw)
    return lib.mixkv_paged_select(c, *a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(pool=None), -1), (dict(pool=264), -1), (dict(table=None), -1), (dict(rows=258), -1), (dict(num_pages=0), -1),
    (dict(page_rows=24), -1), (dict(page_rows=272), -1), (dict(head_dim=64), -2), (dict(k_scale=0.0), -1),
    (dict(v_scale=float("inf")), -1), (dict(v_scale=float("nan")), -1), (dict(batch=0), -1), (dict(max_pages=0), -1),
    (dict(batch=1 << 22, kv_heads=8), -2), (dict(max_pages=1 << 28), -2), (dict(num_pages=1 << 31), -2), (dict(bounds_opt=8), -1)])
def test_bad_caches_are_refused_by_every_entry(lib, kw, status):
    size = C.c_size_t()
    c = pages(**kw)
    assert append(lib, c) == status and attend(lib, c) == status and select(lib, c) == status
    assert lib.mixkv_paged_read(c, ONE, ONE, 0, 8, ONE, 0, 4, None) == status
    assert lib.mixkv_paged_workspace_size(c, 1, 4, C.byref(size)) == status
    assert lib.mixkv_paged_append(None, *[ONE] * 2, 0, *[0] * 5, None, 0, 1, None, None, 0, 0, 0, None, None, None) == -1


def test_bad_arguments_are_refused_before_any_cuda_call(lib):
    c = pages()
    for kw in (dict(k=None), dict(v=C.c_void_p(264)), dict(type=2), dict(n=-1), dict(kr=4), dict(vh=-8), dict(most=0),
               dict(off=None, per=1), dict(cos=ONE), dict(cos=ONE, sin=ONE, len=4, rot=64), dict(cos=ONE, sin=ONE, len=0, rot=64, pos=ONE),
               dict(cos=ONE, sin=ONE, len=4, rot=130, pos=ONE), dict(cos=ONE, sin=ONE, len=4, rot=0, pos=ONE)):
        assert append(lib, c, **kw) == -1, kw
    assert append(lib, c, cos=ONE, sin=ONE, len=4, rot=24, pos=ONE) == -2
    for kw in (dict(q=None), dict(q=C.c_void_p(264)), dict(type=-1), dict(qb=4), dict(qt=-8), dict(T=0), dict(G=0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(rows=0), dict(list=ONE), dict(counts=ONE), dict(list=ONE, counts=ONE), dict(ws=None),
               dict(out=None), dict(out=C.c_void_p(8))):
        assert attend(lib, c, **kw) == -1, kw
    assert attend(lib, c, T=33) == -2 and attend(lib, c, bytes=64) == -3
    for kw in (dict(q=None), dict(type=7), dict(T=0), dict(G=-1), dict(rows=0), dict(top=0), dict(first=-1), dict(last=-1), dict(list=None),
               dict(counts=None), dict(qt=12)):
        assert select(lib, c, **kw) == -1, kw
    assert select(lib, pages(bounds_opt=None)) == -1
    assert select(lib, c, T=33) == -2
    wide = pages(max_pages=40000, page_rows=16)
    assert select(lib, wide, rows=16 * 32769) == -2
    assert lib.mixkv_paged_read(c, None, ONE, 0, 8, ONE, 0, 4, None) == -1
    assert lib.mixkv_paged_read(c, ONE, ONE, 3, 8, ONE, 0, 4, None) == -1
    if not torch.cuda.is_available():     # good arguments get as far as the device
        assert append(lib, c) == -4 and attend(lib, c) == -4 and select(lib, c) == -4


def test_workspace_does_not_depend_on_rows_and_grows_with_queries(lib):
    def size(T, G, **kw):
        s = C.c_size_t()
        assert lib.mixkv_paged_workspace_size(pages(**kw), T, G, C.byref(s)) == 0
        return s.value
    assert 0 < size(1, 4) < size(1, 8) and size(1, 4) == size(1, 4, max_pages=1000)


NARROW = {1: 592, 2: 296, 3: 180, 4: 148, 5: 110, 6: 95, 7: 80, 8: 68}
WIDE = {1: 148, 2: 74, 3: 45, 4: 33, 5: 26, 6: 22, 7: 15, 8: 15}


@pytest.mark.parametrize("units,groups,steps,eights,shape", [
    (4, 1, 16, 1, (4, 0, 0)),            # a short cache: a step for every warp of four small CTAs
    (8, 1, 64, 1, (8, 0, 0)), (8, 1, 65, 1, (4, 1, 0)),       # two steps a warp, and one more: large CTAs
    (32, 1, 512, 1, (4, 1, 0)), (32, 1, 513, 1, (1, 0, 592)),    # eight steps a warp of a large CTA, and one more: shares
    (16, 1, 300, 1, (6, 1, 0)),          # of clusters of seven and eight large CTAs fifteen are held at once
    (896, 1, 80, 1, (1, 0, 0)), (896, 1, 81, 1, (1, 0, 592)),    # more heads than SMs: twenty steps a warp
    (1025, 1, 4096, 1, (1, 0, 0)),       # more heads than the shares' table holds
    (8, 1, 4096, 1, (1, 0, 592)), (1, 1, 1025, 1, (1, 0, 129)),    # few long heads; no more shares than steps are worth
    (32, 2, 230, 3, (1, 0, 148)), (32, 2, 128, 3, (4, 0, 0)), (1, 4, 1, 4, (1, 0, 0))])
def test_how_an_attention_is_split(lib, units, groups, steps, eights, shape):
    table = lambda t: (C.c_int32 * 9)(0, *[t[n] for n in range(1, 9)])
    ctas, large, shared = (C.c_int32() for _ in range(3))
    lib.mixkv_internal_paged_shape(C.c_int64(units), groups, C.c_int64(steps), eights, 148, table(NARROW), table(WIDE),
                                   C.byref(ctas), C.byref(large), C.byref(shared))
    assert (ctas.value, large.value, shared.value) == shape


def test_what_the_paged_calls_enqueue(fake_cuda):
    fake_cuda.reset(device=9, resident={n: 148 // n for n in range(1, 9)})
    lib, names = fake_cuda.lib, lambda: [(x.kernel, x.grid, x.threads, x.cluster) for x in fake_cuda.launches()]
    assert append(lib, pages(), off=None, most=1, n=2) == 0 and append(lib, pages(), n=5000, most=4000) == 0
    assert names() == [("k_paged_append", 8, 64, 1), ("k_paged_append", 8 * 11, 128, 1)]
    fake_cuda.reset(device=9, resident={n: 148 // n for n in range(1, 9)})
    assert attend(lib, pages(), rows=512) == 0 and attend(lib, pages(max_pages=4096), rows=1 << 18) == 0
    assert attend(lib, pages(max_pages=4096), rows=1 << 18, list=ONE, counts=ONE, top=8) == 0
    assert names() == [("k_paged_attention", 32, 128, 4), ("k_paged_attention", 592, 128, 1),
                       ("k_paged_join", 32, 512, 1), ("k_paged_attention", 32, 128, 4)]
    fake_cuda.reset(device=9, resident={n: 148 // n for n in range(1, 9)})
    assert select(lib, pages(), rows=640) == 0 and select(lib, pages(max_pages=4096), rows=1 << 18) == 0
    assert names() == [("k_paged_select", 8, 512, 1), ("k_paged_select", 64, 512, 8)]


def test_a_device_without_clusters_gets_none_for_the_attention(fake_cuda):
    fake_cuda.reset(device=10, resident={n: 0 for n in range(2, 9)})
    for rows in (100, 512, 4000):
        assert attend(fake_cuda.lib, pages(max_pages=100), rows=rows) == 0
    assert all(x.cluster == 1 for x in fake_cuda.launches())


def test_division_by_multiplication():
    # the reciprocal that the kernels index with, at the ends of every divisor's range
    for d in [1, 2, 3, 5, 6, 7, 9, 15, 16, 17, 100, 127, 128, 129, 592, 1000, 65535, 65536, 65537, (1 << 24) - 1, 1 << 24,
              (1 << 30) + 1, (1 << 31) - 1]:
        l = (d - 1).bit_length()
        m = (1 << (31 + l)) // d + 1
        assert l == 0 or m < 1 << 32
        for q in {0, 1, 2, (2 ** 31 - 1) // d, (2 ** 31 - 1) // d // 2}:
            for n in (q * d - 1, q * d, q * d + d - 1):
                if 0 <= n < 1 << 31:
                    assert (n if l == 0 else (n * m >> 32) >> (l - 1)) == n // d, (n, d)


@pytest.mark.parametrize("units,size", [(1, 8), (14, 8), (15, 6), (16, 6), (21, 6), (22, 6), (23, 5), (26, 5), (27, 4), (34, 4), (37, 3),
                                        (44, 3), (45, 2), (48, 2), (74, 2), (75, 1), (148, 1), (600, 1)])
def test_clusters_of_the_selection_are_resident_at_once(fake_cuda, units, size):
    # of clusters of seven and eight fourteen are held at once, as the SM groups of a chip leave it (the runtime without a device
    # answers with twice what it is given for small CTAs)
    fits = {1: 148, 2: 74, 3: 44, 4: 34, 5: 26, 6: 22, 7: 14, 8: 14}
    fake_cuda.reset(device=11, resident={n: m // 2 for n, m in fits.items()})
    assert select(fake_cuda.lib, pages(batch=units, kv_heads=1, max_pages=4096), rows=1 << 18) == 0
    launch, = fake_cuda.launches()
    assert (launch.kernel, launch.grid, launch.cluster) == ("k_paged_select", units * size, size)


def test_a_device_without_clusters_gets_none_for_the_selection(fake_cuda):
    fake_cuda.reset(device=12, resident={n: 0 for n in range(2, 9)})
    assert select(fake_cuda.lib, pages(max_pages=4096), rows=1 << 18) == 0
    launch, = fake_cuda.launches()
    assert (launch.grid, launch.cluster) == (8, 1)


def test_lists_longer_than_the_heads_do_not_run_over_the_shares_sum(fake_cuda):
    # what `counts` says is taken for the number of entries: 1024 heads x 2^20 entries x 8 steps are 2^33, which no prefix of 31 bits
    # holds, so a cluster has a head each; lists of 2^17 entries (2^30 steps) are shared out
    fake_cuda.reset(device=13, resident={n: 148 // n for n in range(1, 9)})
    c = pages(batch=128, kv_heads=8, max_pages=1024, page_rows=256)
    for top in (1 << 20, (1 << 18) + 1, 1 << 17):
        assert attend(fake_cuda.lib, c, rows=1 << 18, list=ONE, counts=ONE, top=top) == 0
    assert [(x.kernel, x.grid) for x in fake_cuda.launches()] == [
        ("k_paged_attention", 1024), ("k_paged_attention", 1024), ("k_paged_attention", 592), ("k_paged_join", 1024)]


@pytest.mark.parametrize("name", ["k_scale", "v_scale"])
def test_scales_without_a_reciprocal_are_refused(lib, name):
    # 1 / (6 x) of a subnormal number can be beyond fp32: a block of zeros would become one of NaN
    least = float(np.finfo(np.float32).tiny)
    most = float(np.finfo(np.float32).max)
    assert 1 / (6 * least) < most < 1 / (6 * 1e-40)
    for bad in (1e-40, float(np.nextafter(np.float32(least), np.float32(0))), 3.1e38, -1.0):
        c = pages(**{name: bad})
        assert append(lib, c) == attend(lib, c) == select(lib, c) == -1, bad
    if not torch.cuda.is_available():
        assert append(lib, pages(**{name: least})) == -4 and append(lib, pages(**{name: 3e38})) == -4


def test_words_between_words_are_refused(lib):
    # (the kernels would fault on them)
    c, odd = pages(), C.c_void_p(258)
    assert select(lib, c, list=odd) == select(lib, c, counts=odd) == -1
    assert attend(lib, c, list=odd, counts=ONE, top=4) == attend(lib, c, list=ONE, counts=odd, top=4) == -1
    assert append(lib, c, off=odd) == append(lib, c, cos=ONE, sin=ONE, len=4, rot=64, pos=odd) == -1
    assert lib.mixkv_paged_append(c, ONE, ONE, 0, 8, 512, 128, 512, 128, ONE, 0, 4, None, None, 0, 0, 0, None, odd, None) == -1
    assert lib.mixkv_paged_read(c, ONE, ONE, 0, 8, odd, 0, 4, None) == -1
