"""The 8-bit attention where blocks of values are of unlike size, and where a row's weight is far below another's."""
import numpy as np
import pytest
import torch

from oracle import cache8_plain as plain
from paper_2510_20707_b200 import binding
from test_gpu_cache8 import TYPES, Cache, dev, query

pytestmark = pytest.mark.gpu


def attended(q, K, V, scale, window=0, sinks=0):
    """Outputs in 64 bits, sums of weight times |value|, and what they may be off by
    - the fp32 logits: 128 products in eight sums, each off by 2^-23 of the products' magnitudes at most, and three products: less than 2^-19 of
      them, twice with the sum of weights;
    - few bits of fp16: weights are 2^6 times as large as the share of the heaviest at least, the smallest step is 2^-24: 2^-31 of the
      heaviest, and never more than the weight;
    - a block with values above 2^64, of which a row gets something (2^-25 at least, of weights that sum to 2^31 at most for 2^17 rows: 2^-56):
      the row's sums are kept times 2^-48, so another block's scale s, as 2^-48 s, is off by 2^-150, half of fp32's smallest step, its codes
      are 448 at most, and the average is off by 448 2^(48 - 150) < 2^-93 (the large block's own rounding: 2^56 and more)."""
    ref, w, aw = plain.attention(q, K, V, scale, window, sinks)
    V = np.abs(np.asarray(V, np.float64))
    size = (np.abs(q) @ np.abs(np.asarray(K, np.float64)).T * scale).max(-1, keepdims=True)
    blocks = np.arange(0, len(V), plain.ROWS)
    large = np.maximum.reduceat(V.max(-1), blocks) > 2.0 ** 64
    coarse = (large & (np.add.reduceat(w, blocks, -1) > 2.0 ** -56)).any(-1, keepdims=True)
    return ref, aw, 2.0 ** -18 * size * aw + np.minimum(w, 2.0 ** -31) @ V + coarse * 2.0 ** -93


def close(got, want, dtype):
    """An output's own rounding; one rounding of every weight to fp16 for bf16 outputs (2^-11 of it), two for fp16 (2^-22); 2^-14 for the fp32
    sums of weighted values; half a step of the smallest numbers."""
    ref, aw, more = want
    half, part, least = {"bf16": (2.0 ** -8, 2.0 ** -11, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -22, 2.0 ** -25)}[dtype]
    tol = half * np.abs(ref) + ((part + 2.0 ** -14) * aw + more) * (1 + half) + least
    off = np.abs(got.double().cpu().numpy() - ref)
    assert (off <= tol).all(), ((off / tol).max(), np.argwhere(~(off <= tol))[:4])


def put(c, k, v):
    """Rows k, v [n, 128] of one head, or of all heads one after the other."""
    ends = np.concatenate([[0], c.lens.reshape(-1).cumsum()]).astype(np.int32)
    binding.cache8_append(c.cache, k, v, offsets=dev(ends), max_new=max(1, int(c.lens.max())))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tail", [-14.0, -15.4, -17.4, -18.5, -20.0])
def test_a_long_tail_beside_a_block_of_large_values(dtype, tail):
    # One row with the largest logit, a block of values 3000 times the others' that gets nothing, and thousands of rows of 2^tail of the first
    # row's weight each, alike: what is lost of one is lost of all.  Heads share their pages, and are so many that a warp has every fourth tile.
    n, heads = 16384, 1100
    c = Cache([[n]], 64, "int8")
    gen = torch.Generator(device="cuda").manual_seed(0)
    k = torch.zeros((n, 128), device="cuda")
    k[0, 0], k[64:80, 0] = 1.0, -8.0
    v = torch.rand((n, 128), generator=gen, device="cuda") * 0.5 + 0.5
    v[64:80] *= 3000.0
    put(c, k.to(TYPES[dtype]), v.to(TYPES[dtype]))
    many = binding.Cache8(pool=c.cache.pool, table=c.cache.table.expand(1, heads, -1).contiguous(),
                          rows=c.cache.rows.expand(1, heads).contiguous(), page_rows=64)
    q = torch.zeros((1, 1, heads, 128), device="cuda")
    q[..., 0] = -tail * float(np.log(2.0))
    q = q.to(TYPES[dtype])
    out = binding.cache8_attention(many, q, softmax_scale=1.0)
    assert (out == out[:, :, :1]).all()
    want = attended(q.double().cpu().numpy()[0, :, :1], *c.rows_of(0, 0), 1.0)
    close(out[0, :, :1], want, dtype)


SIZES = [(1e-20, 1e30), (1e30, 1e-20), (1e-36, 1e37), (1e37, 1e-36), (1.0, 1e20), (1e-30, 1.0)]


@pytest.mark.parametrize("n,heads", [(17, 2), (65, 2), (513, 2), (30001, 8), (161, 1100)])
@pytest.mark.parametrize("here,there", SIZES)
def test_values_that_a_token_does_not_see_leave_its_outputs_alone(n, heads, here, there):
    # the newest row, alone in its block, has values of another size: the token before it does not see it
    c = Cache([[n] * heads], 32, "int8")
    gen = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn((n * heads, 128), generator=gen, device="cuda") for _ in range(2))
    v.view(heads, n, 128)[:, :-1] *= here
    v.view(heads, n, 128)[:, -1] *= there
    put(c, k.bfloat16(), v.bfloat16())
    q = query(1, 2, 3 * heads, "bf16", seed=n)
    out = binding.cache8_attention(c.cache, q)
    for h in range(0, heads, max(1, heads // 3)):
        close(out[0, :, 3 * h:3 * h + 3], attended(q.double().cpu().numpy()[0, :, 3 * h:3 * h + 3], *c.rows_of(0, h), 128 ** -0.5), "bf16")


@pytest.mark.parametrize("here,there", SIZES)
def test_values_that_have_left_the_window(here, there):
    # the second token does not see the first block any more, the sinks' block is of the other size again for one of the heads
    for sinks in (0, 3):
        c = Cache([[160, 400]], 16, "e4m3")
        gen = torch.Generator(device="cuda").manual_seed(1)
        k, v = (torch.randn((560, 128), generator=gen, device="cuda") for _ in range(2))
        size = torch.full((560, 1), here, device="cuda")
        size[:16], size[160:320] = there, there
        v *= size
        put(c, k.bfloat16(), v.bfloat16())
        q = query(1, 2, 4, "bf16")
        out = binding.cache8_attention(c.cache, q, window=240 if sinks else 144, sinks=sinks)
        for h in range(2):
            close(out[0, :, 2 * h:2 * h + 2], attended(q.double().cpu().numpy()[0, :, 2 * h:2 * h + 2], *c.rows_of(0, h), 128 ** -0.5,
                                                      240 if sinks else 144, sinks), "bf16")


@pytest.mark.parametrize("n", [64, 257, 5000])
@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("here,there", SIZES)
def test_values_without_weight_leave_the_outputs_alone(n, order, here, there):
    # rows that are seen and get e^-200 of the weight by one query row, all of it by the other
    c = Cache([[n]], 64, "int8")
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((n, 128), generator=gen, device="cuda") for _ in range(2))
    some = (torch.arange(n, device="cuda") // 16) % 2 == 0
    k[:, 0] = torch.where(some, 10.0, -10.0)
    v *= torch.where(some, here, there).unsqueeze(1)
    put(c, (k if order > 0 else k.flip(0)).bfloat16(), (v if order > 0 else v.flip(0)).bfloat16())
    q = query(1, 1, 2, "bf16", gain=0.1)
    q[0, 0, :, 0] = torch.tensor([10.0, -10.0])
    out = binding.cache8_attention(c.cache, q, softmax_scale=1.0)
    close(out[0], attended(q.double().cpu().numpy()[0], *c.rows_of(0, 0), 1.0), "bf16")


def test_blocks_of_every_size():
    # values from 1e-37 to 3e38, in no order, each seen by a query row that looks for it
    n = 16 * 76
    c = Cache([[n]], 64, "int8")
    gen = torch.Generator(device="cuda").manual_seed(3)
    size = torch.from_numpy(np.random.default_rng(0).permutation(76) - 37.0).cuda()
    v = (torch.rand((n, 128), generator=gen, device="cuda", dtype=torch.float64) + 1) * (10.0 ** size).repeat_interleave(16).unsqueeze(1)
    k = torch.zeros((n, 128), device="cuda")
    k[torch.arange(n), torch.arange(n) // 16] = 1.0
    put(c, k.bfloat16(), v.bfloat16())
    q = torch.zeros((1, 1, 76, 128), device="cuda")
    q[0, 0, torch.arange(76), torch.arange(76)] = 300.0
    q = q.bfloat16()
    out = binding.cache8_attention(c.cache, q, softmax_scale=1.0)
    close(out[0], attended(q.double().cpu().numpy()[0], *c.rows_of(0, 0), 1.0), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("heads,n,where", [(2, 129, 128), (8, 20001, 20000), (8, 20001, 9000)])
def test_a_block_of_nan_reaches_the_rows_that_see_it(dtype, code, heads, n, where):
    # among the newest rows, where the first token does not see it; or before the window of the second one, block's last row first
    c = Cache([[n] * heads], 64, code)
    gen = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn((n * heads, 128), generator=gen, device="cuda").to(TYPES[dtype]) for _ in range(2))
    v.view(heads, n, 128)[::2, where, 5] = float("nan")
    put(c, k, v)
    q = query(1, 2, 3 * heads, dtype)
    last = where | 15                                    # of the block
    window = 0 if where == n - 1 else n - 1 - last       # the first token sees rows from `last` on, the second from the next
    c.cache.mass.fill_(0.0)
    out = binding.cache8_attention(c.cache, q, window=window, accumulate=True).view(2, heads, 3, 128)
    sees = 1 if where == n - 1 else 0
    assert torch.isnan(out[sees, ::2]).all() and not torch.isnan(out[1 - sees]).any() and not torch.isnan(out[:, 1::2]).any()
    assert not torch.isnan(c.cache.mass).any()           # (a value of NaN is in no weight)
    for h in range(heads):
        K, V = c.rows_of(0, h)
        t = np.arange(2) if h % 2 else np.array([1 - sees])
        ref = attended(q.double().cpu().numpy()[0, :, 3 * h:3 * h + 3], K, np.nan_to_num(V), 128 ** -0.5, window)
        close(out.transpose(0, 1)[h][torch.from_numpy(t).cuda()], tuple(x[t] for x in ref), dtype)
