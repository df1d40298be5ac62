"""The 8-bit attention where a row's weight is far below another's."""
import numpy as np
import pytest
import torch

from oracle import cache8_plain as plain
from paper_2510_20707_b200 import binding
from test_gpu_cache8 import TYPES, Cache, dev

pytestmark = pytest.mark.gpu


def attended(q, K, V, scale, window=0, sinks=0):
    """Outputs in 64 bits, sums of weight times |value|, and what they may be off by
    - the fp32 logits: 128 products in eight sums, each off by 2^-23 of the products' magnitudes at most, and three products: less than 2^-19 of
      them, twice with the sum of weights;
    - few bits of fp16: weights are 2^6 times as large as the share of the heaviest at least, the smallest step is 2^-24: 2^-31 of the
      heaviest, and never more than the weight."""
    ref, w, aw = plain.attention(q, K, V, scale, window, sinks)
    V = np.abs(np.asarray(V, np.float64))
    size = (np.abs(q) @ np.abs(np.asarray(K, np.float64)).T * scale).max(-1, keepdims=True)
    return ref, aw, 2.0 ** -18 * size * aw + np.minimum(w, 2.0 ** -31) @ V


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
