"""Masses of the 8-bit cache: pages that several sequences share get what each of them gives; what a draft has given stays."""
import numpy as np
import pytest
import torch

from oracle import cache8_plain as plain
from paper_2510_20707_b200 import binding
from test_gpu_cache8 import Cache, dev, query

pytestmark = pytest.mark.gpu


# (clusters that add up the weights themselves; all tiles dealt out and joined; several groups of query rows)
@pytest.mark.parametrize("B,H,G,T,prefix,own", [(16, 2, 4, 1, 320, 40), (4, 8, 4, 1, 16000, 400), (8, 2, 8, 16, 960, 33), (32, 1, 3, 2, 64, 0)])
def test_masses_of_shared_pages(B, H, G, T, prefix, own):
    page, n = 32, prefix + own
    c = Cache(np.full((B, H), n), page, "int8", spare=0)
    table = c.table.copy()
    table[:, :, :prefix // page] = table[:1, :, :prefix // page]      # the first sequence's, for all
    c.fill()
    c.table = table
    c.cache.table.copy_(dev(table))
    q = query(B, T, H * G, "bf16")
    got, times = [], 5
    start = torch.rand(c.cache.mass.shape, device="cuda")
    for _ in range(times):
        c.cache.mass.copy_(start)
        binding.cache8_attention(c.cache, q, accumulate=True)
        got.append(c.cache.mass.double().cpu().numpy())
    want, tol = start.double().cpu().numpy().copy(), np.zeros(c.cache.mass.shape)
    r = np.arange(n)
    for b in range(B):
        for h in range(H):
            qq = q.double().cpu().numpy()[b, :, h * G:(h + 1) * G]
            K, V = c.rows_of(b, h)
            w = plain.attention(qq, K, V, 128 ** -0.5)[1]
            at = table[b, h, r // page], r % page
            want[at] += w.sum((0, 1))
            # as for pages of one owner: the fp32 logits, and 2^-19 for exponentials, products and sums
            size = np.abs(qq) @ np.abs(K).T * 128 ** -0.5
            tol[at] += (w * (2.0 ** -15 * size.max(-1, keepdims=True) + 2.0 ** -19)).sum((0, 1))
    tol += B * 2.0 ** -24 * want      # a rounding for each addition
    for m in got:
        assert (np.abs(m - want) <= tol).all(), np.nanmax(np.abs(m - want) / np.maximum(tol, 1e-30))
    # rows of one owner: the same bits every time
    mine = np.zeros(c.cache.mass.shape, int)
    for b in range(B):
        for h in range(H):
            np.add.at(mine, (table[b, h, r // page], r % page), 1)
    for m in got[1:]:
        assert np.array_equal(m[mine <= 1], got[0][mine <= 1])


def test_a_head_whose_pages_are_all_one():
    # the same page again and again: every row of it is as many rows of the sequence
    c = Cache([[64 * 40]], 64, "e4m3", spare=0)
    c.fill()
    c.table[:] = c.table[0, 0, 7]
    c.cache.table.copy_(dev(c.table))
    c.cache.mass.fill_(0.0)
    q = query(1, 1, 8, "fp16")
    binding.cache8_attention(c.cache, q, accumulate=True)
    m = c.cache.mass[c.table[0, 0, 0]].double().cpu().numpy()
    K, V = c.rows_of(0, 0)
    w = plain.attention(q.double().cpu().numpy()[0], K, V, 128 ** -0.5)[1].sum((0, 1)).reshape(40, 64).sum(0)
    assert np.allclose(m, w, rtol=1e-4) and abs(m.sum() - 8) < 1e-4


def test_weights_of_a_draft():
    # five tokens are checked, two of them stay
    c = Cache([[300, 77]], 32, "int8")
    c.fill()
    c.cache.mass.fill_(0.0)
    q = query(1, 5, 8, "bf16")
    weights = lambda T, n: [plain.attention(q.double().cpu().numpy()[0, :T, 4 * h:4 * h + 4], *(x[:n[h]] for x in c.rows_of(0, h)),
                                            128 ** -0.5)[1].sum((0, 1)) for h in range(2)]
    out = binding.cache8_attention(c.cache, q)
    assert (c.cache.mass == 0).all()
    c.cache.rows -= 3
    again = binding.cache8_attention(c.cache, q[:, :2], accumulate=True)
    # (the same rows for each token; how the work is split may differ, and with it an output's last bit)
    assert torch.allclose(out[:, :2].float(), again.float(), rtol=2.0 ** -7, atol=1e-5)
    for h, w in enumerate(weights(2, [297, 74])):
        m = c.mass_of(0, h)
        assert np.allclose(m[:len(w)], w, rtol=1e-4, atol=1e-7) and (m[len(w):] == 0).all()
    # with the weights at once, those of the rejected tokens stay on the rows that stay
    c.cache.mass.fill_(0.0)
    c.cache.rows += 3
    binding.cache8_attention(c.cache, q, accumulate=True)
    c.cache.rows -= 3
    for h, w in enumerate(weights(5, [300, 77])):
        assert np.allclose(c.mass_of(0, h), w, rtol=1e-4, atol=1e-7)
