"""The paged 8-bit cache without a GPU: its plain definition, what the entry points refuse before any CUDA call, how a call is split."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache8_plain as plain
from paper_2510_20707_b200 import binding, build

ONE = 4096      # an aligned address that is not null; nothing looks behind it


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_codes_against_torch(code):
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal((40, 128)) * 10.0 ** rng.integers(-4, 5, (40, 1)), np.zeros((1, 128))]).astype(np.float32)
    for row in x:
        s = plain.scale_of(row[None], code)
        got = plain.encode(row, s, code)
        t = torch.from_numpy(row)
        if s == 0:
            assert (got == 0).all()
            continue
        y = t * (1.0 / torch.tensor(s))
        want = (y.round().clamp(-127, 127).to(torch.int8) if code == "int8" else y.clamp(-448, 448).to(torch.float8_e4m3fn))
        assert np.array_equal(got, want.view(torch.uint8).numpy())
        # the largest value has the largest code, and an error is at most half a step: of the scale, or 2^-4 of the value
        back = plain.values(got, s, code)
        assert np.abs(plain.NUMBERS[code][got]).max() == plain.CODES[code]
        step = np.maximum(np.abs(row) * 2.0 ** -4, s * 2.0 ** -10) if code == "e4m3" else s / 2
        assert (np.abs(back - row) <= step * 1.0001).all()


def test_a_tile_holds_every_row_once():
    assert np.array_equal(np.sort(plain.AT.ravel()), np.arange(2048))
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 37, 128)).astype(np.float32)
    pool, table = np.full((3, 2 * plain.TILE_BYTES), 0xFF, np.uint8), np.array([2, 0], np.int32)
    plain.append(pool, table, 32, 0, x[0][:20], x[1][:20], "int8")
    plain.append(pool, table, 32, 20, x[0][20:], x[1][20:], "int8")
    for got, want in zip(plain.rows_of(pool, table, 32, 37, "int8"), x):
        for t in range(0, 37, 16):     # (the second block's old rows were rounded twice at most)
            assert np.abs(got[t:t + 16] - want[t:t + 16]).max() <= 1.0001 * np.abs(want[t:t + 16]).max() / 127


def test_a_block_grows_and_its_old_rows_are_rounded_again():
    a, b = np.full((1, 128), 1.0, np.float32), np.full((1, 128), 10.0, np.float32)
    tile = np.full(plain.TILE_BYTES, 0xFF, np.uint8)
    plain.put(tile, 0, 0, a, "int8", False)
    assert plain.scales_at(tile)[0] == np.float32(1) * plain.BY["int8"] and (tile[plain.AT[0]] == 127).all()
    plain.put(tile, 0, 1, b, "int8", True)
    assert plain.scales_at(tile)[0] == np.float32(10) * plain.BY["int8"]
    assert (tile[plain.AT[0]] == 13).all() and (tile[plain.AT[1]] == 127).all() and (tile[plain.AT[2:]] == 0).all()
    plain.put(tile, 0, 1, a, "int8", True)      # the scale stays when the row is written anew
    assert plain.scales_at(tile)[0] == np.float32(10) * plain.BY["int8"] and (tile[plain.AT[1]] == 13).all()
    plain.put(tile, 0, 2, np.full((1, 128), np.inf, np.float32), "int8", True)
    assert np.isnan(plain.scales_at(tile)[0])


def test_what_a_window_sees():
    assert plain.seen(6, 2, 2, 1).astype(int).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert plain.seen(3, 4, 0, 0).astype(int).tolist() == [[0, 0, 0], [1, 0, 0], [1, 1, 0], [1, 1, 1]]
    rng = np.random.default_rng(2)
    q, K, V = rng.standard_normal((2, 3, 128)), rng.standard_normal((9, 128)), rng.standard_normal((9, 128))
    out, w, _ = plain.attention(q, K, V, 0.1, 3, 2)
    for t, rows in enumerate(([0, 1, 5, 6, 7], [0, 1, 6, 7, 8])):
        p = torch.softmax(torch.from_numpy(q[t] @ K[rows].T * 0.1), 1).numpy()
        assert np.allclose(out[t], p @ V[rows]) and np.allclose(w[t][:, rows], p) and np.allclose(w[t].sum(-1), 1)
    assert (plain.attention(q, K[:1], V[:1], 0.1)[0][0] == 0).all()


def test_what_an_eviction_keeps():
    m = np.array([0, 3, 1, 3, np.nan, 0, 2, 9], np.float32)
    assert plain.kept_rows(m, 8, 1, 1).tolist() == list(range(8))
    assert plain.kept_rows(m, 4, 0, 0).tolist() == [1, 3, 4, 7]
    assert plain.kept_rows(m, 4, 1, 1).tolist() == [0, 1, 4, 7]
    assert plain.kept_rows(m, 2, 1, 1).tolist() == [0, 7]
    assert plain.kept_rows(np.zeros(5, np.float32), 3, 0, 1).tolist() == [0, 1, 4]


def test_page_bytes(lib):
    assert binding.cache8_page_bytes(16) == 4112 and binding.cache8_page_bytes(256) == 16 * 4112
    for bad in (0, 8, 24, 272, -16):
        with pytest.raises(binding.MixKVError) as e:
            binding.cache8_page_bytes(bad)
        assert e.value.status == -1


def fake_attention(fake, batch, heads, rows, T=1, G=4, accumulate=0, window=0, sinks=0, device=20):
    fake.reset(device=device)
    c = cache(batch=batch, kv_heads=heads, max_pages=-(-rows // 64), num_pages=1 << 20)
    rc = fake.lib.mixkv_cache_attention(C.byref(c), ONE, 0, 128 * T * heads * G, 128 * heads * G, T, G, 0.0, rows, window, sinks, accumulate,
                                        ONE, 1 << 40, ONE, None)
    assert rc == 0
    return fake.launches()


def cache(**kw):
    d = dict(pool=ONE, mass_opt=ONE, table=ONE, rows=ONE, num_pages=10, max_pages=4, page_rows=64, batch=2, kv_heads=3, head_dim=128, code=0)
    d.update(kw)
    return binding._CCache8(**d)


BAD_CACHES = [(dict(pool=0), -1), (dict(pool=ONE + 8), -1), (dict(table=0), -1), (dict(rows=0), -1), (dict(table=ONE + 2), -1),
              (dict(rows=ONE + 1), -1), (dict(mass_opt=ONE + 2), -1), (dict(num_pages=0), -1), (dict(max_pages=0), -1), (dict(batch=0), -1),
              (dict(kv_heads=0), -1), (dict(page_rows=24), -1), (dict(page_rows=0), -1), (dict(page_rows=272), -1), (dict(code=2), -1),
              (dict(head_dim=64), -2), (dict(batch=1 << 24, kv_heads=2), -2), (dict(max_pages=1 << 30), -2), (dict(num_pages=1 << 31), -2)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_every_entry_refuses_a_cache_that_is_none(lib, change, status):
    c, good = cache(**change), cache(rows=ONE + 64)
    size = C.c_size_t()
    assert lib.mixkv_cache_append(C.byref(c), ONE, ONE, 0, 2, 384, 128, 384, 128, None, 0, 1, None, None) == status
    assert lib.mixkv_cache_read(C.byref(c), ONE, ONE, 0, 2, None, 0, 1, None) == status
    assert lib.mixkv_cache_workspace_size(C.byref(c), 1, 4, 100, 0, 0, 0, C.byref(size)) == status
    assert lib.mixkv_cache_attention(C.byref(c), ONE, 0, 1536, 1536, 1, 4, 0.0, 100, 0, 0, 0, ONE, 1 << 40, ONE, None) == status
    assert lib.mixkv_cache_evict(C.byref(c), C.byref(good), 64, None, 1, 1, 100, ONE, None, None) == status
    assert lib.mixkv_cache_evict(C.byref(good), C.byref(c), 64, None, 1, 1, 100, ONE, None, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(k=0), -1), (dict(v=0), -1), (dict(k=ONE + 16), -1), (dict(type=2), -1), (dict(tokens=-1), -1), (dict(ks=8), -1), (dict(vh=-16), -1),
    (dict(max_new=0), -1), (dict(per_head=1), -1), (dict(offsets=ONE + 2), -1), (dict(status=ONE + 2), -1), (dict(max_new=(1 << 30) + 1), -2)])
def test_append_and_read_refuse(lib, change, status):
    a = dict(k=ONE, v=ONE, type=0, tokens=2, ks=384, kh=128, vs=384, vh=128, offsets=None, per_head=0, max_new=1, status=None)
    a.update(change)
    c = cache()
    got = lib.mixkv_cache_append(C.byref(c), a["k"], a["v"], a["type"], a["tokens"], a["ks"], a["kh"], a["vs"], a["vh"], a["offsets"],
                                  a["per_head"], a["max_new"], a["status"], None)
    assert got == status
    if not {"ks", "vh", "status"} & set(change):
        assert lib.mixkv_cache_read(C.byref(c), a["k"], a["v"], a["type"], a["tokens"], a["offsets"], a["per_head"], a["max_new"],
                                     None) == status
    big = cache(batch=1 << 12, kv_heads=1 << 10, max_pages=1 << 12)
    assert lib.mixkv_cache_read(C.byref(big), ONE, ONE, 0, 2, ONE, 0, 1 << 20, None) == -2


@pytest.mark.parametrize("change,status", [
    (dict(q=0), -1), (dict(q=ONE + 8), -1), (dict(type=3), -1), (dict(qb=4), -1), (dict(qt=-8), -1), (dict(T=0), -1), (dict(G=0), -1),
    (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(max_rows=0), -1), (dict(window=-1), -1),
    (dict(sinks=-1), -1), (dict(ws=0), -1), (dict(ws=ONE + 8), -1), (dict(out=0), -1), (dict(out=ONE + 4), -1), (dict(T=43, G=3), -2),
    (dict(nbytes=1000), -3), (dict(accumulate=1, mass=0), -1)])
def test_attention_refuses(lib, change, status):
    a = dict(q=ONE, type=0, qb=1536, qt=1536, T=1, G=4, scale=0.0, max_rows=100, window=0, sinks=0, accumulate=0, ws=ONE, nbytes=1 << 40,
             out=ONE, mass=ONE, pages=4, page_rows=64)
    a.update(change)
    c = cache(mass_opt=a["mass"], max_pages=a["pages"], page_rows=a["page_rows"])
    assert lib.mixkv_cache_attention(C.byref(c), a["q"], a["type"], a["qb"], a["qt"], a["T"], a["G"], a["scale"], a["max_rows"],
                                      a["window"], a["sinks"], a["accumulate"], a["ws"], a["nbytes"], a["out"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(idx=0), -1), (dict(idx=ONE + 2), -1), (dict(budget=0), -1), (dict(first=-1), -1), (dict(last=-1), -1), (dict(first=40, last=30), -1),
    (dict(max_rows=0), -1), (dict(budgets=ONE + 2), -1), (dict(status=ONE + 1), -1), (dict(mass=0), -1), (dict(batch=3), -1), (dict(heads=1), -1),
    (dict(code=1), -1), (dict(rows=ONE), -1), (dict(budget=1 << 30, first=1 << 30, last=1 << 30), -1), (dict(budget=(1 << 30) + 1), -2)])
def test_evict_refuses(lib, change, status):
    a = dict(budget=64, budgets=None, first=1, last=1, max_rows=100, idx=ONE, status=None, mass=ONE, batch=2, heads=3, code=0, rows=ONE + 64)
    a.update(change)
    c, into = cache(mass_opt=a["mass"]), cache(batch=a["batch"], kv_heads=a["heads"], code=a["code"], rows=a["rows"], mass_opt=0)
    assert lib.mixkv_cache_evict(C.byref(c), C.byref(into), a["budget"], a["budgets"], a["first"], a["last"], a["max_rows"], a["idx"],
                                  a["status"], None) == status


def test_a_workspace_for_more_rows_serves_fewer(lib):
    def need(max_rows, window=0, sinks=0, acc=1, T=2, G=3):
        size = C.c_size_t()
        c = cache(max_pages=1000)
        assert lib.mixkv_cache_workspace_size(C.byref(c), T, G, max_rows, window, sinks, acc, C.byref(size)) == 0
        return size.value
    sizes = [need(n) for n in (1, 16, 17, 1000, 64000, 1 << 29)]
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2]
    assert need(64000, acc=0) == need(1, acc=0) < need(1)
    # a window's logits: at most what the sinks, the window and the draft can touch
    tiles = lambda w, s, T: -(-s // 16) + (w + T - 1 + 14) // 16 + 1
    assert need(64000, 100, 5) - need(1) == (tiles(100, 5, 2) - 1) * 16 * 6 * 4 * 6
    assert need(64000, 1 << 30, 1 << 30) == need(64000)


def tiles_of(n, T, window, sinks):
    """What the kernel makes of a unit (cache8_attention.cu, unit_tiles): its tiles in order."""
    tiles, sink, gap = (n + 15) >> 4, (n + 15) >> 4, 0
    if window > 0:
        low, s = max(0, n - T + 1 - window) >> 4, (min(sinks, n) + 15) >> 4
        if low > s:
            sink, gap = s, low - s
            tiles -= gap
    return [i if i < sink else i + gap for i in range(tiles)]


def test_the_tiles_of_a_window_hold_all_that_is_seen():
    rng = np.random.default_rng(3)
    for _ in range(3000):
        n, T = int(rng.integers(0, 300)), int(rng.integers(1, 9))
        window, sinks = int(rng.integers(0, 90)), int(rng.integers(0, 50))
        got = tiles_of(n, T, window, sinks)
        want = set((np.flatnonzero(plain.seen(n, T, window, sinks).any(0)) // 16).tolist()) if n else set()
        assert want <= set(got) and len(set(got)) == len(got) and all(0 <= t < (n + 15) // 16 for t in got)
        if window:      # room for their logits, and few that nobody needs
            assert len(got) <= -(-sinks // 16) + (window + T - 1 + 14) // 16 + 1
            assert len(got) <= len(want) + 1 + (T > n)


@pytest.mark.parametrize("units,groups,tiles,eights", [(1, 1, 1, 1), (4, 1, 32, 1), (8, 1, 8192, 1), (256, 1, 1024, 1), (2000, 1, 900, 1),
                                                       (32, 2, 459, 3), (3, 4, 10, 4)])
def test_how_a_call_is_split(lib, units, groups, tiles, eights):
    S, shared = C.c_int32(), C.c_int32()
    slots = (4 if eights == 1 else 3 if eights == 2 else 2) * 148
    resident = (C.c_int32 * 9)(0, *[slots // n - (n > 2) for n in range(1, 9)])
    lib.mixkv_internal_cache8_shape(C.c_int64(units), groups, C.c_int64(tiles), tiles % 2, eights, 0, 148, resident, C.byref(S), C.byref(shared))
    assert 1 <= S.value <= 8 and 0 <= shared.value <= slots
    if shared.value:
        assert S.value == 1 and shared.value * groups <= slots and units <= 1024
    elif S.value > 1:
        assert units * groups <= resident[S.value] and S.value * 4 <= tiles


def test_what_an_attention_enqueues(fake_cuda):
    names = lambda calls: [x.kernel for x in calls]
    # a short call is one kernel in clusters, which add up the weights themselves
    for acc in (0, 1):
        calls = fake_attention(fake_cuda, 1, 4, 512, accumulate=acc)
        assert names(calls) == ["k_cache8_attention"] and calls[0].cluster == 8 and calls[0].grid == 32
    # a long one is dealt out evenly and joined; its weights are added up by the kernel that joins
    join = fake_attention(fake_cuda, 1, 8, 131072)
    both = fake_attention(fake_cuda, 1, 8, 131072, accumulate=1)
    for calls in (join, both):
        assert names(calls) == ["k_cache8_attention", "k_cache8_finish"]
        assert all(x.cluster == 1 for x in calls) and calls[0].grid == 4 * 148
    assert both[1].grid > join[1].grid
    # query rows of several groups: no cluster has all of them
    calls = fake_attention(fake_cuda, 1, 2, 200, T=16, G=8, accumulate=1)
    assert names(calls) == ["k_cache8_attention", "k_cache8_finish"] and calls[0].cluster > 1
    # more heads than are dealt out; a window that makes long heads short ones
    assert names(fake_attention(fake_cuda, 64, 32, 4000)) == ["k_cache8_attention"]
    assert names(fake_attention(fake_cuda, 1, 8, 131072, window=500, sinks=4)) == ["k_cache8_attention"]


def test_a_device_that_holds_no_cluster_gets_none(fake_cuda):
    fake_cuda.reset(device=21, resident={n: 0 for n in range(2, 9)})
    c = cache(batch=1, kv_heads=4, max_pages=8, num_pages=64)
    assert fake_cuda.lib.mixkv_cache_attention(C.byref(c), ONE, 0, 512, 512, 1, 1, 0.0, 512, 0, 0, 0, ONE, 1 << 40, ONE, None) == 0
    assert all(x.cluster == 1 for x in fake_cuda.launches())


def test_what_rows_and_evictions_enqueue(fake_cuda):
    fake_cuda.reset(device=22)
    c, into = cache(batch=2, kv_heads=3, max_pages=100), cache(batch=2, kv_heads=3, rows=ONE + 64)
    lib = fake_cuda.lib
    # K and V of every tile that new rows can touch: two warps a tile, four to a CTA
    assert lib.mixkv_cache_append(C.byref(c), ONE, ONE, 0, 40, 384, 128, 384, 128, ONE, 0, 18, None, None) == 0
    assert lib.mixkv_cache_read(C.byref(c), ONE, ONE, 1, 40, ONE, 0, 1, None) == 0
    assert [(x.kernel, x.grid) for x in fake_cuda.launches()] == [("k_cache8_append", 2 * 3 * 3 * 2 // 4), ("k_cache8_read", 2 * 3 * 2 // 4)]
    for rows, budget, cluster in ((2048, 64, 1), (2049, 64, 2), (6400, 1000, 4)):
        fake_cuda.reset(device=22)
        assert lib.mixkv_cache_evict(C.byref(c), C.byref(into), budget, None, 1, 1, rows, ONE, None, None) == 0
        calls = fake_cuda.launches()
        assert [x.kernel for x in calls] == ["k_cache8_pick", "k_cache8_move"] and calls[0].cluster == cluster
        assert calls[1].grid == -(-6 * -(-budget // 16) // 4)
