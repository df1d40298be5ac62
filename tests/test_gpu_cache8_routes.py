"""How the 8-bit attention's work can be split, with every form of call on each way: outputs and the mass of every row against 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache8_plain as plain
from paper_2510_20707_b200 import binding
from test_gpu_cache8 import Cache, check_attention, query

pytestmark = pytest.mark.gpu


def is_dealt_out(units, R, rows, T, window, sinks, dtype, sms=148):
    """Whether the CTAs share all tiles of such a call; the same for a device that holds as many clusters as CTAs, and for one that holds three
    quarters of them."""
    eights = -(-R // 8)
    groups = -(-eights // 4)
    NT = -(-eights // groups)
    slots = (2 if NT > 1 else 3 if dtype == "fp16" else 4) * sms
    tiles = -(-rows // 16)
    some = -(-sinks // 16) + (window + T - 1 + 14) // 16 + 1
    even = window > 0 and some < tiles
    got = set()
    for part in (1.0, 0.75):
        S, shared, resident = C.c_int32(), C.c_int32(), (C.c_int32 * 9)(0, *[int(slots // n * part) for n in range(1, 9)])
        binding.load_library().mixkv_internal_cache8_shape(C.c_int64(units), groups, C.c_int64(some if even else tiles), int(even), NT,
                                                           int(dtype == "fp16"), sms, resident, C.byref(S), C.byref(shared))
        got.add(shared.value > 0)
    assert len(got) == 1
    return got.pop()


def spread(B, H, lo, hi, seed=0):
    lens = np.random.default_rng(seed).integers(lo, hi + 1, (B, H))
    lens[0, 0] = hi
    return lens


def attend_and_check(lens, page, code, dtype, T, G, window=0, sinks=0, dealt=True, strided=False):
    lens = np.asarray(lens)
    B, H = lens.shape
    c = Cache(lens, page, code, seed=T + G, spare=1)
    c.fill(seed=G, dtype=torch.bfloat16)
    start = torch.rand(c.cache.mass.shape, device="cuda")
    c.cache.mass.copy_(start)
    rows = int(lens.max())
    assert is_dealt_out(B * H, T * G, rows, T, window, sinks, dtype) == dealt
    q = query(B, T, H * G, dtype, seed=page)
    if strided:
        wide = torch.zeros((B, T + 2, 3 * H * G, 128), dtype=q.dtype, device="cuda")
        wide[:, 1:-1, H * G:2 * H * G] = q
        q = wide[:, 1:-1, H * G:2 * H * G]
    out = binding.cache8_attention(c.cache, q, rows, window=window, sinks=sinks, accumulate=True)
    # (masses begin at zero for the comparison: of sums, fp32 keeps less)
    kept = c.cache.mass.clone()
    c.cache.mass.zero_()
    again = binding.cache8_attention(c.cache, q, rows, window=window, sinks=sinks, accumulate=True)
    assert torch.equal(out, again) and torch.equal(kept, start + c.cache.mass)
    assert torch.equal(out, binding.cache8_attention(c.cache, q, rows, window=window, sinks=sinks))
    check_attention(c, q, dtype, 128 ** -0.5, window, sinks, out, c.cache.mass)


# one, two, three and four groups of eight query rows in a CTA; two to four CTAs for a head's query rows
@pytest.mark.parametrize("dtype,code,T,G,page,B,H,lo,hi", [
    ("fp16", "int8", 2, 7, 16, 64, 4, 70, 1639), ("bf16", "e4m3", 2, 7, 32, 60, 4, 0, 2500), ("fp16", "e4m3", 5, 7, 64, 8, 4, 2051, 7334),
    ("bf16", "int8", 5, 7, 64, 8, 4, 1, 7334), ("bf16", "int8", 4, 8, 128, 1, 8, 4000, 8192), ("fp16", "int8", 3, 7, 48, 20, 3, 100, 6000),
    ("bf16", "e4m3", 16, 8, 64, 4, 4, 900, 6000), ("fp16", "int8", 8, 11, 32, 6, 4, 1, 4100), ("fp16", "e4m3", 1, 1, 16, 5, 8, 1, 9000),
    ("bf16", "int8", 1, 5, 256, 2, 2, 30000, 60000)])
def test_all_tiles_dealt_out(dtype, code, T, G, page, B, H, lo, hi):
    attend_and_check(spread(B, H, lo, hi, hi), page, code, dtype, T, G)


# a gap inside units: rows of the window and the sinks numbered one after the other over CTAs' borders
@pytest.mark.parametrize("dtype,code,T,G,page,lens,window,sinks", [
    ("bf16", "int8", 1, 4, 64, [[20000, 20000, 20000]], 16000, 100), ("fp16", "e4m3", 3, 4, 32, [[30000, 25000, 17000, 40]], 20000, 33),
    ("bf16", "e4m3", 2, 7, 16, spread(6, 5, 0, 20000, 1), 14000, 4), ("fp16", "int8", 5, 7, 64, spread(8, 4, 1, 9000, 2), 7000, 64),
    ("bf16", "int8", 1, 1, 48, [[50000, 3], [0, 49999]], 30000, 0), ("bf16", "e4m3", 16, 8, 128, spread(3, 3, 10, 20000, 3), 15000, 17)])
def test_all_tiles_of_windows_dealt_out(dtype, code, T, G, page, lens, window, sinks):
    attend_and_check(lens, page, code, dtype, T, G, window, sinks)


@pytest.mark.parametrize("dtype,code,T,G,page,lens,window,sinks", [
    ("fp16", "e4m3", 2, 7, 16, spread(8, 4, 1, 500, 1), 0, 0), ("bf16", "int8", 4, 6, 64, spread(4, 4, 1, 700, 2), 0, 0),
    ("fp16", "int8", 4, 8, 32, spread(3, 3, 0, 400, 3), 100, 20), ("bf16", "e4m3", 16, 8, 32, spread(3, 3, 1, 300, 4), 0, 0),
    ("bf16", "int8", 1, 4, 64, spread(20, 4, 1, 20000, 5), 2048, 4), ("fp16", "int8", 1, 7, 64, [[512] * 4], 0, 0)])
def test_a_cluster_for_every_head(dtype, code, T, G, page, lens, window, sinks):
    attend_and_check(lens, page, code, dtype, T, G, window, sinks, dealt=False, strided=True)


def test_more_heads_than_are_dealt_out():
    attend_and_check(spread(260, 4, 1, 400, 6), 16, "e4m3", "fp16", 3, 3, 0, 0, dealt=False)


# ---- fp16 outputs: a weight is two numbers of fp16
def outputs_of(q, K, V, first, parts):
    """Outputs in 64 bits with weights as so many numbers of fp16, 2^6 times as large as the heaviest of the rows `first`."""
    _, w, _ = plain.attention(q, K, V, 1.0)
    w = w / w[..., first].max(-1, keepdims=True) * 2.0 ** 6
    p = w.astype(np.float16).astype(np.float64)
    if parts > 1:
        p = p + (w - p).astype(np.float16).astype(np.float64)
    return (p @ np.asarray(V, np.float64) / w.sum(-1, keepdims=True)).astype(np.float16).astype(np.float64)


def off(got, q, K, V):
    """How far fp16 outputs are, in units of what they may be: their rounding (2^-11, and 2^-25), two roundings of a weight and 2^-15 for the
    sums of values, 2^-18 of the products' magnitudes for the logits (as where blocks are of unlike size)."""
    ref, _, aw = plain.attention(q, K, V, 1.0)
    size = (np.abs(q) @ np.abs(np.asarray(K, np.float64)).T).max(-1, keepdims=True)
    return (np.abs(got - ref) / (2.0 ** -11 * np.abs(ref) + (2.0 ** -22 + 2.0 ** -15 + 2.0 ** -18 * size) * aw * (1 + 2.0 ** -11) + 2.0 ** -25)).max()


def one_heavy_row(code, rows=100, heads=1100, G=4):
    """Keys and values [rows, 128] and queries [heads * G, 128]: the last row has a third to two thirds of the weight, 2^6 to 2^8 times that of
    the others."""
    rng = np.random.default_rng(7)
    k, v = (rng.standard_normal((rows, 128)).astype(np.float16) for _ in range(2))
    k[:, 0], k[-1], k[-1, 0] = 0, 0, 1
    q = rng.standard_normal((heads * G, 128)) * 0.02
    q[:, 0] = np.linspace(4.2, 5.2, heads * G)
    return k, v, q.astype(np.float16)


FIRST = np.arange(32, 48)      # of the warp that takes the last row's tile, the seventh: its first tile, which its weights are relative to


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_weights_of_fp16_outputs_have_more_bits_than_one_number(code):
    # heads that share their pages, so many that a head has one CTA and a warp every fourth tile
    k, v, q = one_heavy_row(code)
    n, heads = len(k), len(q) // 4
    c = Cache([[n]], 32, code)
    binding.cache8_append(c.cache, *(torch.from_numpy(x).cuda() for x in (k, v)), max_new=n,
                          offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    many = binding.Cache8(pool=c.cache.pool, table=c.cache.table.expand(1, heads, -1).contiguous(),
                          rows=c.cache.rows.expand(1, heads).contiguous(), page_rows=32, code=code)
    out = binding.cache8_attention(many, torch.from_numpy(q).cuda().view(1, 1, -1, 128), softmax_scale=1.0)
    K, V = c.rows_of(0, 0)
    q = q.astype(np.float64)[None]
    # (the bound tells one number from two)
    assert off(outputs_of(q, K, V, FIRST, 1), q, K, V) > 1.3 and off(outputs_of(q, K, V, FIRST, 2), q, K, V) <= 1
    assert off(out.double().cpu().numpy()[0], q, K, V) <= 1
