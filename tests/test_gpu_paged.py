"""GPU parity of the paged 4-bit cache (append, read back, page selection, attention) against its plain definition."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_plain as plain
from paper_2510_20707_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def f32(t):
    return t.float().cpu().numpy()


class Cache:
    """A cache of `lens` [batch][heads] rows behind a shuffled page table; every byte starts as 0xff (scales of NaN)."""

    def __init__(self, lens, page=32, bounds=False, ks=1.0, vs=1.0, seed=0, spare=2, room=0):
        lens = np.asarray(lens)
        rng = np.random.default_rng(seed)
        count = -(-np.maximum(lens, room) // page)
        cols, total = max(1, int(count.max())), int(count.sum())
        table = np.full((*lens.shape, cols), -1, np.int32)
        table[np.arange(cols) < count[..., None]] = rng.permutation(total + spare)[:total]
        self.lens, self.table, self.page = lens, table, page
        n = total + spare
        self.pages = binding.Pages(
            pool=torch.full((n, binding.page_bytes(page)), 0xFF, dtype=torch.uint8, device="cuda"),
            table=torch.from_numpy(table).cuda(), rows=torch.from_numpy(lens.astype(np.int32)).cuda(), page_rows=page,
            bounds=torch.full((n, 2, 128), 7.0, dtype=torch.float16, device="cuda") if bounds else None,
            k_scale=ks, v_scale=vs)

    def pool(self):
        return self.pages.pool.cpu().numpy()

    def rows_of(self, b, h):
        k, v = plain.get_rows(self.pool(), self.table[b, h], self.page, int(self.lens[b, h]))
        return k * self.pages.k_scale, v * self.pages.v_scale

    def fill(self, seed=1, k_gain=1.0, dtype=torch.bfloat16, positions=None):
        """Random rows everywhere, one offset per (sequence, head)."""
        flat = self.lens.reshape(-1)
        off = torch.from_numpy(np.concatenate([[0], flat.cumsum()]).astype(np.int32)).cuda()
        gen = torch.Generator(device="cuda").manual_seed(seed)
        n = int(flat.sum())
        k, v = (torch.randn((max(n, 1), 128), generator=gen, device="cuda") for _ in range(2))
        k[:, 3::31] *= 3.0
        k, v = (k * k_gain).to(dtype)[:n], v.to(dtype)[:n]
        binding.paged_append(self.pages, k, v, offsets=off, max_new=max(1, int(flat.max())))
        return k, v, off


def expect_rows(cache, token_rows, kx, vx):
    """The bytes that fp32 rows kx, vx [n, 128] leave: token_rows [n] of (b, h, row)."""
    want = np.full(cache.pages.pool.shape, 0xFF, np.uint8)
    tiles = want.reshape(-1, plain.TILE_BYTES)
    kc, ks = plain.quantise(kx, cache.pages.k_scale)
    vc, vs = plain.quantise(vx, cache.pages.v_scale)
    per = cache.page // 16
    for i, (b, h, r) in enumerate(token_rows):
        t = int(cache.table[b, h, r // cache.page]) * per + r % cache.page // 16
        plain.put_row(tiles[t], r % 16, kc[i], ks[i], vc[i], vs[i])
    return want, plain.values(kc, ks), plain.values(vc, vs)


def expect_bounds(cache, token_rows, kv, start):
    """Bounds of pages, by fp64 minima and maxima of all rows a page has; kv[(b, h, r)] -> values."""
    want = np.full((cache.pages.pool.shape[0], 2, 128), 7.0)
    pages = {}
    for i, (b, h, r) in enumerate(token_rows):
        pages.setdefault((b, h, r // cache.page), []).append(kv[i])
    for (b, h, p), rows in pages.items():
        x = np.stack(rows)
        want[cache.table[b, h, p]] = x.min(0), x.max(0)
    return want


def rope_tables(n, rot, seed=0):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))[None]
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


@pytest.mark.parametrize("dtype,page,rot,inter,H", [
    ("bf16", 16, 128, False, 3), ("fp16", 32, 64, True, 1), ("bf16", 64, 32, False, 2), ("fp16", 128, 16, True, 4),
    ("bf16", 256, 0, False, 2), ("fp16", 48, 96, False, 5)])
def test_append_and_read_back(dtype, page, rot, inter, H):
    # new rows of several sequences (none, one, a page and more) behind rows that are there, K and V slices of one tensor
    new, old = np.array([0, 1, 17, 2 * page + 5, 15]), np.array([3, page - 1, 2, page // 2 + 1, 0])
    B, N = len(new), int(new.sum())
    c = Cache((old + new)[:, None].repeat(H, 1), page, ks=0.5, vs=2.0, bounds=True, seed=page)
    off = np.concatenate([[0], new.cumsum()]).astype(np.int32)
    gen = torch.Generator(device="cuda").manual_seed(page)
    qkv = torch.randn((N, 3 * H, 128), generator=gen, device="cuda").to(TYPES[dtype])
    k, v = qkv[:, H:2 * H], qkv[:, 2 * H:]
    pos = np.random.default_rng(1).integers(0, 5000, N).astype(np.int32)
    cos, sin = rope_tables(5000, rot) if rot else (None, None)
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(offsets=dev(off), max_new=int(new.max()))
    binding.paged_append(c.pages, k, v, cos=dev(cos), sin=dev(sin), positions=dev(pos) if rot else None,
                         interleaved=inter, status=status, **kw)
    assert status.item() == 0
    kx, vx = f32(k), f32(v)
    if rot:
        kx = np.stack([plain.rotate(kx[:, h], cos[pos], sin[pos], inter) for h in range(H)], 1)
    where = [(b, h, int(old[b]) + i) for b in range(B) for i in range(new[b]) for h in range(H)]
    want, kv, vv = expect_rows(c, where, kx.reshape(-1, 128), vx.reshape(-1, 128))
    assert np.array_equal(c.pool(), want)
    # pages that had rows keep what was in their bounds (7.0 here), those that begin with a new row are set
    got = c.pages.bounds.double().cpu().numpy()
    bounds = expect_bounds(c, where, kv, old)
    for b in range(B):
        if new[b] and old[b] % page:
            ids = c.table[b, :, old[b] // page]
            bounds[ids, 0], bounds[ids, 1] = np.minimum(bounds[ids, 0], 7.0), np.maximum(bounds[ids, 1], 7.0)
    assert np.array_equal(got, bounds)
    kr, vr = binding.paged_read(c.pages, N, TYPES[dtype], **kw)
    back = lambda x, s: torch.from_numpy((x * s).reshape(N, H, 128)).to(TYPES[dtype])
    assert torch.equal(kr.cpu(), back(kv, 0.5)) and torch.equal(vr.cpu(), back(vv, 2.0))


@pytest.mark.parametrize("dtype,inter", [("bf16", False), ("fp16", True), ("bf16", True)])
def test_products_of_the_rotation_are_rounded_before_their_sum(dtype, inter):
    # 100 cos - 100 sin is 8, a quarter of the block's scale and so a code of zero, if both products are rounded first; with one
    # of them unrounded it is more, and the code is the next.  One pair of eight sets the scale (192 / 6 = 32).
    rng = np.random.default_rng(0)
    n, pairs = 24, 64
    s = rng.uniform(0.5, 0.9, 400000).astype(np.float32)
    c = ((np.float32(100) * s).astype(np.float64) + 8.0) / 100.0
    c = c.astype(np.float32)
    cp, sp = np.float32(100) * c, np.float32(100) * s
    exact_c, exact_s = 100.0 * c.astype(np.float64), 100.0 * s.astype(np.float64)
    near = (cp - sp == 8) & ((exact_c - sp).astype(np.float32) > 8) & ((cp - exact_s).astype(np.float32) > 8)
    assert near.sum() > n * pairs
    cos, sin = (t[near][:n * pairs].reshape(n, pairs).copy() for t in (c, s))
    cos[:, ::8], sin[:, ::8] = 1.0, 0.0
    x = np.full((n, pairs), 100, np.float32)
    y = x.copy()
    x[:, ::8], y[:, ::8] = 192.0, 0.0
    rows = np.stack([x, y], -1).reshape(n, 128) if inter else np.concatenate([x, y], 1)
    cache = Cache([[n]], 32)
    k = torch.from_numpy(rows).to(TYPES[dtype]).cuda()
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    binding.paged_append(cache.pages, k, torch.zeros_like(k), offsets=off, max_new=n, cos=torch.from_numpy(cos).cuda(),
                         sin=torch.from_numpy(sin).cuda(), positions=torch.arange(n, dtype=torch.int32, device="cuda"),
                         interleaved=inter)
    kx = plain.rotate(rows, cos, sin, inter)
    want = plain.values(*plain.quantise(kx))
    firsts = want[:, ::2] if inter else want[:, :64]
    assert (firsts[:, np.arange(pairs) % 8 != 0] == 0).all()
    assert np.array_equal(cache.rows_of(0, 0)[0], want)


@pytest.mark.parametrize("dtype,page,rot,inter", [
    ("bf16", 16, 128, False), ("fp16", 16, 64, False), ("bf16", 16, 32, True), ("fp16", 32, 0, False), ("bf16", 32, 96, False)])
def test_many_pages_in_one_call_leave_what_few_at_a_time_leave(dtype, page, rot, inter):
    # more pages than a GPU has warps' groups for: a warp has a page alone; a piece of a hundred rows is shared by four
    B, H, n, piece = 3, 4, 2105 * page // 16, 100
    old = np.arange(B * H).reshape(B, H) * 7 % 40
    gen = torch.Generator(device="cuda").manual_seed(page + rot)
    k, v = (torch.randn((B, n, H, 128), generator=gen, device="cuda").to(TYPES[dtype]) for _ in range(2))
    k[1, 77], v[2, 5, 1, 16:32] = 0.0, 0.0          # blocks of zeros
    k[0, 1000, 2, 40], v[0, 13, 3, 3] = float("inf"), float("nan")
    pos = torch.randint(0, 3000, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    kw = {}
    if rot:
        pos[1, 1500] = 3000                          # outside the tables: not written, reported
        kw = dict(zip(("cos", "sin"), (torch.from_numpy(t).cuda() for t in rope_tables(3000, rot))), interleaved=inter)
    whole, parts = (Cache(old + n, page, ks=0.5, bounds=True, seed=7) for _ in range(2))
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    off = lambda m: torch.arange(0, B * m + 1, m, dtype=torch.int32, device="cuda")
    flat = lambda t: t.reshape(-1, *t.shape[2:]).contiguous()
    binding.paged_append(whole.pages, flat(k), flat(v), offsets=off(n), max_new=n, status=status[:1],
                         **(dict(kw, positions=flat(pos)) if rot else {}))
    parts.pages.rows.copy_(torch.from_numpy(old.astype(np.int32)))
    for i in range(0, n, piece):
        m = min(piece, n - i)
        parts.pages.rows += m
        binding.paged_append(parts.pages, flat(k[:, i:i + m]), flat(v[:, i:i + m]), offsets=off(m), max_new=m, status=status[1:],
                             **(dict(kw, positions=flat(pos[:, i:i + m])) if rot else {}))
    assert torch.equal(whole.pages.pool, parts.pages.pool)
    assert torch.equal(whole.pages.bounds.view(torch.int16), parts.pages.bounds.view(torch.int16))
    assert (status != 0).tolist() == [bool(rot)] * 2


def test_tokens_one_by_one_leave_what_one_call_leaves():
    B, H, page, n = 3, 2, 16, 37
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((B, n, H, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    whole, steps = (Cache(np.full((B, H), n), page, bounds=True, seed=5) for _ in range(2))
    off = torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda")
    binding.paged_append(whole.pages, k.reshape(-1, H, 128), v.reshape(-1, H, 128), offsets=off, max_new=n)
    steps.pages.rows.zero_()
    for i in range(n):
        steps.pages.rows += 1
        binding.paged_append(steps.pages, k[:, i], v[:, i])     # (strided: a token of every sequence)
    assert torch.equal(whole.pages.pool, steps.pages.pool)
    used = torch.from_numpy(np.unique(whole.table[whole.table >= 0])).cuda()
    assert torch.equal(whole.pages.bounds[used], steps.pages.bounds[used])


def test_compact_rows_of_a_compressed_layer():
    # what compress_layer leaves (heads of different lengths) goes into pages as it is
    lens = np.array([[40, 7, 0], [129, 64, 1]])
    c = Cache(lens, 64, bounds=True, seed=2)
    k, v, off = c.fill()
    where = [(b, h, r) for b in range(2) for h in range(3) for r in range(lens[b, h])]
    want, kv, vv = expect_rows(c, where, f32(k), f32(v))
    assert np.array_equal(c.pool(), want)
    kr, vr = binding.paged_read(c.pages, k.shape[0], offsets=off, max_new=129, compact=True)
    assert torch.equal(kr.cpu(), torch.from_numpy(kv).bfloat16()) and torch.equal(vr.cpu(), torch.from_numpy(vv).bfloat16())


def test_rounding_of_special_values():
    rows = np.zeros((12, 128), np.float32)
    rows[1] = np.linspace(-6, 6, 128)                      # ties among them
    rows[2] = np.repeat([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], 16) * np.tile([1, -1], 64)
    rows[2, 15::16] = 6.0                                  # scale 1: every tie goes to the even code
    rows[3] = 1e-4                                         # a scale below the smallest e4m3 number
    rows[4] = 0.004
    rows[5] = 30000.0                                      # beyond 6 * 448: saturates
    rows[6, 5], rows[7, 20], rows[8, 127] = np.inf, -np.inf, np.nan
    rows[6, :16] += 1.0
    rows[9] = -0.0
    rows[10] = np.random.default_rng(0).standard_normal(128)
    rows[11, ::16] = 448.0
    x = torch.from_numpy(rows).cuda().half()
    c = Cache([[12]], 16, bounds=True)
    off = torch.tensor([0, 12], dtype=torch.int32, device="cuda")
    binding.paged_append(c.pages, x, x, offsets=off, max_new=12)
    kc, ks = plain.quantise(f32(x))
    got, _ = plain.get_rows(c.pool(), c.table[0, 0], 16, 12)
    assert np.array_equal(got, plain.values(kc, ks), equal_nan=True)
    assert np.isnan(got[8, 112:]).all() and np.isfinite(np.delete(got, 8, 0)).all() and got[5, 0] == 2688.0
    lo, hi = c.pages.bounds[int(c.table[0, 0, 0])].double().cpu().numpy()
    assert np.array_equal(lo, got.min(0), equal_nan=True) and np.array_equal(hi, got.max(0), equal_nan=True)


def test_rows_without_a_place_are_reported_and_not_written():
    k = torch.ones((4, 1, 128), device="cuda").bfloat16()
    cos, sin = (torch.from_numpy(x).cuda() for x in rope_tables(8, 128))

    def run(change, tokens=4, **kw):
        c = Cache([[4], [5], [6], [7]], 16)
        change(c)
        before = c.pages.pool.clone()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        binding.paged_append(c.pages, k[:tokens], k[:tokens], status=status, **kw)
        ids = [int(x) for x in c.table[:, 0, 0]]
        return status.item(), [not torch.equal(c.pages.pool[i], before[i]) for i in ids]

    pos = lambda *p: dict(cos=cos, sin=sin, positions=torch.tensor(p, dtype=torch.int32, device="cuda"))
    assert run(lambda c: None, **pos(0, 7, 1, 2)) == (0, [True] * 4)
    assert run(lambda c: None, **pos(0, 8, -1, 2)) == (-1, [True, False, False, True])
    assert run(lambda c: c.pages.table[1].fill_(c.pages.pool.shape[0])) == (-1, [True, False, True, True])
    assert run(lambda c: c.pages.table[2].fill_(-5)) == (-1, [True, True, False, True])
    assert run(lambda c: c.pages.rows[0].fill_(17)) == (-1, [False, True, True, True])       # beyond the table
    assert run(lambda c: c.pages.rows[0].fill_(0)) == (-1, [False, True, True, True])        # a token more than rows
    off = dict(offsets=torch.tensor([0, 1, 2, 3, 5], dtype=torch.int32, device="cuda"), max_new=2)   # one past the input
    assert run(lambda c: None, **off) == (-1, [True] * 4)


def check_attention(c, q, out, T, G, ctx=""):
    """out against fp64.  A value may be off by the output's rounding, by the weights' (fp16, 2^-11 each, and 2^-25 of the
    smallest next to a largest of 2^6 at least), and by what the logits' fp32 sums (128 products, their terms 2^-23 of the
    largest partial sum each) do to the weights."""
    unit = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -11
    got, qf = out.double().cpu().numpy(), q.double().cpu().numpy()
    pool = c.pool()
    for b in range(c.lens.shape[0]):
        for h in range(c.lens.shape[1]):
            n = int(c.lens[b, h])
            K, V = plain.get_rows(pool, c.table[b, h], c.page, n)
            K, V = K * c.pages.k_scale, V * c.pages.v_scale
            want, mass, size = plain.attention(qf[b, :, h * G:(h + 1) * G], K, V, T, 1 / np.sqrt(128))
            most = np.abs(V).max() if n else 0.0
            off = 2.0 ** -23 * 128 * size[..., None] + 2.0 ** -20
            tol = unit * np.abs(want) + mass * (2.0 ** -11 + 2 * off) + n * 2.0 ** -31 * most + 2.0 ** -24 * (unit < 2.0 ** -10)
            bad = np.abs(got[b, :, h * G:(h + 1) * G] - want) > tol
            assert not bad.any(), (ctx, b, h, n, int(bad.sum()))


def queries(B, T, HG, dtype, seed=0, gain=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((B, T, HG, 128), generator=gen, device="cuda") * gain).to(TYPES[dtype])


@pytest.mark.parametrize("G,T,dtype,page", [
    (1, 1, "bf16", 16), (7, 1, "fp16", 32), (8, 1, "bf16", 64), (9, 1, "bf16", 128), (16, 1, "fp16", 48),
    (4, 2, "bf16", 16), (7, 5, "fp16", 64), (5, 3, "bf16", 256), (16, 8, "bf16", 32), (3, 11, "fp16", 16)])
def test_lengths_at_the_edges_of_tiles_and_pages(G, T, dtype, page):
    # no row, fewer than the tokens, one, a tile, a page, one more and one less; heads of their own lengths; what was
    # never written holds scales of NaN
    lens = np.array([[0, 1, 2], [15, 16, 17], [page - 1, page, page + 1], [2 * page + 3, 33, 5]])
    c = Cache(lens, page, ks=0.5, vs=0.25, seed=G)
    c.fill()
    q = queries(4, T, 3 * G, dtype, G)
    out = binding.paged_attention(c.pages, q)
    assert out.dtype == q.dtype
    check_attention(c, q, out, T, G)
    assert (out[0, :, :G] == 0).all()


@pytest.mark.parametrize("lens,G,T,page", [
    ([[20000, 513], [4097, 1]], 4, 1, 64), ([[9000] * 8], 7, 1, 32), ([[70000]], 8, 2, 64), ([[6000], [33], [0]], 16, 3, 16)])
def test_long_rows_split_over_many_ctas(lens, G, T, page):
    lens = np.array(lens)
    c = Cache(lens, page, seed=3)
    c.fill()
    q = queries(lens.shape[0], T, lens.shape[1] * G, "bf16", 1)
    ws = binding.paged_workspace(c.pages, q)
    ws.fill_(0xFF)       # nothing of it is read before it is written
    out = binding.paged_attention(c.pages, q, workspace=ws)
    check_attention(c, q, out, T, G)
    for _ in range(5):
        assert torch.equal(out, binding.paged_attention(c.pages, q, workspace=ws))


@pytest.mark.parametrize("B,H,G,lo,hi", [(75, 8, 7, 0, 40), (37, 4, 16, 1, 300), (149, 1, 4, 100, 140), (19, 3, 12, 1, 700),
                                         (300, 4, 4, 1, 90), (64, 8, 4, 10, 2000)])
def test_many_units(B, H, G, lo, hi):
    rng = np.random.default_rng(B)
    lens = rng.integers(lo, hi + 1, (B, H))
    lens[0, 0], lens[-1, -1] = lo, hi
    c = Cache(lens, 16, seed=B)
    c.fill()
    q = queries(B, 1, H * G, "bf16", B)
    out = binding.paged_attention(c.pages, q, max_rows=hi)
    check_attention(c, q, out, 1, G)
    assert torch.equal(out, binding.paged_attention(c.pages, q, max_rows=hi))


def test_sharp_and_flat_rows():
    # a row far above the rest late in a long head (the running reference moves), all rows alike (the weights of thousands),
    # logits that fall steadily and rise steadily
    n, G = 5000, 4
    c = Cache([[n, n, n, n]], 64)
    gen = torch.Generator(device="cuda").manual_seed(0)
    base = torch.randn(128, generator=gen, device="cuda")
    k = torch.randn((4, n, 128), generator=gen, device="cuda")
    k[0, n - 700] = 8 * base
    k[1] = base
    ramp = torch.linspace(-6, 6, n, device="cuda").unsqueeze(1)
    k[2], k[3] = ramp * base, -ramp * base
    v = torch.randn((4, n, 128), generator=gen, device="cuda")
    off = torch.arange(0, 4 * n + 1, n, dtype=torch.int32, device="cuda")
    binding.paged_append(c.pages, k.reshape(-1, 128).bfloat16(), v.reshape(-1, 128).bfloat16(), offsets=off, max_new=n)
    q = (base * torch.tensor([0.2, 1.0, 3.0, -1.0], device="cuda").repeat(4).unsqueeze(1)).view(1, 1, 16, 128).bfloat16()
    check_attention(c, q, binding.paged_attention(c.pages, q), 1, G)


@pytest.mark.parametrize("gain", [1e-30, 1e-6, 1e3, 1e20])
def test_queries_of_any_size(gain):
    c = Cache([[300]], 32)
    c.fill(k_gain=0.0 if gain > 1e10 else 1.0)     # (logits of 1e20 would leave one row: keys of zero keep it even)
    q = queries(1, 1, 3, "bf16", 0, gain)
    check_attention(c, q, binding.paged_attention(c.pages, q), 1, 3)


def test_not_a_number():
    n, G, T = 100, 2, 3
    c = Cache([[n, n, n]], 16)
    k, v, off = c.fill()
    k, v = k.view(3, n, 128), v.view(3, n, 128)
    v[0, n - 1, 40] = float("nan")     # the last token's value: its own output alone, in that block
    k[1, n - 2, 3] = float("nan")      # the last token but one's key: its own and the last one's
    binding.paged_append(c.pages, k.reshape(-1, 128), v.reshape(-1, 128), offsets=off, max_new=n)
    q = queries(1, T, 3 * G, "bf16")
    q[0, 1, 2 * G, 7] = float("inf")   # a query: its own row
    nan = torch.isnan(binding.paged_attention(c.pages, q)).cpu()
    want = torch.zeros_like(nan)
    want[0, 2, :G, 32:48] = True
    want[0, 1:, G:2 * G] = True
    want[0, 1, 2 * G] = True
    assert torch.equal(nan, want)


def test_a_page_outside_the_pool_counts_as_empty():
    n, page, G = 100, 16, 4
    for bad in (-1, 10 ** 6):
        c = Cache([[n]], page)
        c.fill()
        keep = np.r_[0:32, 48:n]
        K, V = c.rows_of(0, 0)
        c.pages.table[0, 0, 2] = bad
        q = queries(1, 1, G, "bf16")
        want, mass, _ = plain.attention(q[0].double().cpu().numpy(), K[keep], V[keep], 1, 1 / np.sqrt(128))
        got = binding.paged_attention(c.pages, q)[0].double().cpu().numpy()
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + mass * 2.0 ** -10).all()


def test_strided_queries_streams_and_capture():
    c = Cache([[3000, 20], [700, 701]], 32, bounds=True)
    c.fill()
    big = queries(2, 4, 10, "bf16")
    q = big[:, 1:3, 2:8]            # two of four tokens, six of ten heads
    want = binding.paged_attention(c.pages, q.contiguous())
    assert torch.equal(binding.paged_attention(c.pages, q), want)
    swant = binding.paged_sparse_attention(c.pages, q.contiguous(), 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = binding.paged_attention(c.pages, q, stream=side)
    sout = binding.paged_sparse_attention(c.pages, q, 5, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(sout, swant))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = binding.paged_attention(c.pages, q)
        sout = binding.paged_sparse_attention(c.pages, q, 5)
    out.zero_(), sout[0].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(sout, swant))


def test_a_pool_beyond_four_gigabytes():
    page, total = 64, 500_000         # 4.6 GB; the pages in use are the last ones
    pool = torch.empty((total, binding.page_bytes(page)), dtype=torch.uint8, device="cuda")
    c = Cache([[200, 130]], page, bounds=True)
    pool[-16:] = 0xFF
    c.table = np.where(c.table >= 0, total - 1 - c.table, -1).astype(np.int32)
    c.pages.pool, c.pages.table = pool, torch.from_numpy(c.table).cuda()
    c.pages.bounds = torch.zeros((total, 2, 128), dtype=torch.float16, device="cuda")
    c.pool = lambda: torch.cat([torch.zeros((1, pool.shape[1]), dtype=torch.uint8), pool[-16:].cpu()]).numpy()
    k, v, off = c.fill()
    kr, vr = binding.paged_read(c.pages, 330, offsets=off, max_new=200, compact=True)
    kc, ks = plain.quantise(f32(k))
    assert torch.equal(kr.cpu(), torch.from_numpy(plain.values(kc, ks)).bfloat16())
    real = c.table
    c.table = np.where(real >= 0, real - (total - 17), -1)
    q = queries(1, 1, 8, "bf16")
    check_attention(c, q, binding.paged_attention(c.pages, q), 1, 4)
    lists, counts = binding.paged_select(c.pages, q, 2)
    out = binding.paged_attention(c.pages, q, page_list=lists, counts=counts)
    assert torch.isfinite(out).all() and counts.tolist() == [[2, 2]]


def oracle_select(c, q, T, G, top, first, last):
    lists = np.full((*c.lens.shape, top), -1, np.int32)
    bounds = f32(c.pages.bounds)
    for b in range(c.lens.shape[0]):
        for h in range(c.lens.shape[1]):
            n = -(-int(c.lens[b, h]) // c.page)
            ids = c.table[b, h, :n]
            s = plain.scores(f32(q[b, :, h * G:(h + 1) * G]).reshape(-1, 128), bounds[ids, 0], bounds[ids, 1])
            picked = plain.select(s, top, first, last)
            lists[b, h, :len(picked)] = picked
    return lists


@pytest.mark.parametrize("B,H,G,T,page,top,first,last,hi,dtype", [
    (2, 2, 7, 1, 16, 5, 1, 1, 700, "bf16"), (3, 1, 1, 1, 32, 1, 0, 0, 900, "fp16"), (1, 4, 4, 2, 16, 64, 0, 2, 20000, "bf16"),
    (2, 3, 16, 1, 64, 7, 2, 3, 5000, "fp16"), (1, 1, 9, 4, 16, 3, 5, 5, 1000, "bf16"), (40, 8, 4, 1, 16, 9, 1, 1, 400, "bf16"),
    (1, 2, 16, 8, 128, 200, 1, 1, 9000, "bf16")])
def test_selected_pages(B, H, G, T, page, top, first, last, hi, dtype):
    rng = np.random.default_rng(top)
    lens = rng.integers(0, hi + 1, (B, H))
    lens[0, 0], lens[-1, -1] = hi, rng.integers(0, page)
    c = Cache(lens, page, bounds=True, seed=top)
    c.fill()
    q = queries(B, T, H * G, dtype, top)
    lists, counts = binding.paged_select(c.pages, q, top, keep_first=first, keep_last=last)
    want = oracle_select(c, q, T, G, top, first, last)
    assert np.array_equal(lists.cpu().numpy(), want)
    assert np.array_equal(counts.cpu().numpy(), (want >= 0).sum(-1))
    out, lists2, counts2 = binding.paged_sparse_attention(c.pages, q, top, keep_first=first, keep_last=last)
    assert torch.equal(lists, lists2) and torch.equal(counts, counts2)
    assert torch.equal(out, binding.paged_attention(c.pages, q, page_list=lists, counts=counts))
    # what is attended to: the rows of the listed pages
    for b, h in [(0, 0), (B - 1, H - 1), (B // 2, H // 2)]:
        K, V = c.rows_of(b, h)
        rows = [r for p in want[b, h] if p >= 0 for r in range(p * page, min((p + 1) * page, lens[b, h]))]
        qf = q[b, :, h * G:(h + 1) * G].double().cpu().numpy()
        for t in range(T):
            seen = [r for r in rows if r <= lens[b, h] - T + t]
            ref, mass, size = plain.attention(qf[t:t + 1], K[seen], V[seen], 1, 1 / np.sqrt(128))
            got = out[b, t, h * G:(h + 1) * G].double().cpu().numpy()
            unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
            tol = unit * np.abs(ref[0]) + mass[0] * (2.0 ** -11 + 2.0 ** -15 * size[0][:, None] + 2.0 ** -19) + 2.0 ** -24
            assert (np.abs(got - ref[0]) <= tol).all(), (b, h, t)


def test_equal_scores_go_to_the_lower_page_and_nan_goes_first():
    c = Cache([[16 * 40]], 16, bounds=True)
    c.fill()
    ids = c.table[0, 0]
    q = queries(1, 1, 2, "bf16")
    c.pages.bounds.fill_(1.0)           # one score for all
    assert binding.paged_select(c.pages, q, 6, keep_first=0, keep_last=0)[0].tolist() == [[[0, 1, 2, 3, 4, 5]]]
    assert binding.paged_select(c.pages, q, 6, keep_first=1, keep_last=2)[0].tolist() == [[[0, 1, 2, 3, 38, 39]]]
    c.pages.bounds[int(ids[17])] = float("nan")
    assert binding.paged_select(c.pages, q, 3, keep_first=0, keep_last=0)[0].tolist() == [[[0, 1, 17]]]
    assert binding.paged_select(c.pages, q, 1, keep_first=0, keep_last=1)[0].tolist() == [[[39]]]
    c.pages.bounds.zero_()              # scores of 0 and -0 are equal
    q[0, 0, :, ::2] *= -1
    assert binding.paged_select(c.pages, q, 4, keep_first=0, keep_last=0)[0].tolist() == [[[0, 1, 2, 3]]]
    assert binding.paged_select(c.pages, q, 50, keep_first=0, keep_last=0)[0][0, 0].tolist() == list(range(40)) + [-1] * 10


def test_refusals():
    c = Cache([[40, 40]], 16, bounds=True)
    c.fill()
    q = queries(1, 1, 4, "bf16")
    k = torch.zeros((1, 2, 128), dtype=torch.bfloat16, device="cuda")
    P = binding.Pages
    change = lambda **kw: P(**{**c.pages.__dict__, **kw})

    def _status(f):
        with pytest.raises(binding.MixKVError) as e:
            f()
        return e.value.status

    assert _status(lambda: binding.paged_attention(change(k_scale=0.0), q)) == -1
    assert _status(lambda: binding.paged_attention(change(v_scale=float("nan")), q)) == -1
    assert _status(lambda: binding.paged_attention(c.pages, q, max_rows=0)) == -1
    assert _status(lambda: binding.paged_attention(c.pages, q, softmax_scale=-1.0)) == -1
    assert _status(lambda: binding.paged_attention(c.pages, q, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))) == -3
    assert _status(lambda: binding.paged_attention(c.pages, queries(1, 33, 8, "bf16"))) == -2        # 132 query rows
    assert _status(lambda: binding.paged_select(change(bounds=None), q, 3)) == -1
    assert _status(lambda: binding.paged_select(c.pages, q, 0)) == -1
    assert _status(lambda: binding.paged_select(c.pages, q, 3, keep_first=-1)) == -1
    assert _status(lambda: binding.paged_append(c.pages, k, k, max_new=0)) == -1
    table = lambda n: torch.zeros((4, n), device="cuda")
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert _status(lambda: binding.paged_append(c.pages, k, k, cos=table(4), sin=table(4), positions=pos)) == -2   # 8 dimensions
    assert _status(lambda: binding.paged_append(c.pages, k, k, cos=table(72), sin=table(72), positions=pos)) == -1
    for bad in (dict(table=c.pages.table.long()), dict(rows=c.pages.rows[:, :1]), dict(page_rows=32),
                dict(bounds=c.pages.bounds.float()), dict(pool=c.pages.pool.cpu())):
        with pytest.raises(AssertionError):
            binding.paged_attention(change(**bad), q)
    for bad in (q[..., :64], q[:, :, :3], q.float(), q.cpu(), q[0], queries(1, 1, 8, "bf16")[:, :, ::2]):
        with pytest.raises(AssertionError):
            binding.paged_attention(c.pages, bad)
    with pytest.raises(AssertionError):
        binding.paged_append(c.pages, k.view(2, 128), k.view(2, 128))       # compact rows without offsets
    with pytest.raises(AssertionError):
        binding.paged_append(c.pages, k, k.half())
    with pytest.raises(AssertionError):
        binding.paged_append(c.pages, torch.cat([k, k]), torch.cat([k, k]))     # two tokens, one sequence, no offsets
    with pytest.raises(TypeError):
        binding.paged_read(c.pages, 1, torch.float32)


def test_the_example_runs():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    errors, outs = example.main(3)
    # two 4-bit codes to a byte, blocks of 16: the rounding of normal values is about a tenth of them
    assert len(errors) == 2 and max(errors) < 0.3
    assert len(outs) == 4 and all(o.shape == (1, 1, 28, 128) and torch.isfinite(o.float()).all() for o in outs)


def test_what_changes_from_step_to_step_is_read_anew():
    # rows, table, lists and rows of the pool are written by one kernel and read by the next, which is resident by then: in one
    # loop without a pause, with outputs in the memory of earlier ones, every step gives what it gives when nothing overlaps
    B, H, G, page, n = 3, 2, 4, 16, 60
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((n, B, H, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((n, B, 1, H * G, 128), generator=gen, device="cuda").bfloat16()
    caches = [Cache(np.zeros((B, H), int), page, bounds=True, seed=i, room=n) for i in range(2)]

    def steps(c, wait):
        outs = []
        for i in range(n):
            c.pages.rows += 1
            binding.paged_append(c.pages, k[i], v[i])
            out, lists, counts = binding.paged_sparse_attention(c.pages, q[i], 2)
            full = binding.paged_attention(c.pages, q[i])
            if wait:
                torch.cuda.synchronize()
            outs.append((out, full))
            del lists, counts
        torch.cuda.synchronize()
        return outs

    for (a, b), (x, y) in zip(steps(caches[0], True), steps(caches[1], False)):
        assert torch.equal(a, x) and torch.equal(b, y)


@pytest.mark.parametrize("pages,top,G", [(40, 6, 2), (700, 3, 7), (1999, 500, 4)])
def test_pages_of_one_score_in_every_head(pages, top, G):
    # the search for the threshold has nothing to take apart: equal scores, a query of NaN, or every page kept
    B, H, page = 4, 8, 16
    c = Cache(np.full((B, H), pages * page), page, bounds=True)
    c.pages.bounds.fill_(1.0)
    q = queries(B, 1, H * G, "bf16")
    odd = q.clone()
    odd[..., 5] = float("nan")
    want = torch.arange(top, dtype=torch.int32, device="cuda").expand(B, H, top)
    for query, first, last in ((q, 0, 0), (odd, 0, 0), (q, pages // 2, pages), (q, pages, 0)):
        got = [binding.paged_select(c.pages, query, top, keep_first=first, keep_last=last) for _ in range(100)]
        assert all(torch.equal(lists, want) and bool((counts == top).all()) for lists, counts in got)


def test_a_wait_that_runs_out_does_so_for_the_whole_warp():
    # (a wait inside the attention; here one that is over for half of a warp's lanes, after the time is up)
    answers = torch.full((64,), 7, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert binding.load_library().mixkv_internal_warp_waits(C.c_void_p(answers.data_ptr()), C.c_void_p(stream)) == 0
    assert answers.tolist() == [0] * 32 + [1] * 32


@pytest.mark.parametrize("compact", [False, True])
def test_more_new_rows_than_a_call_allows_are_reported(compact):
    # 5, 1 and 40 new rows of two heads; without a bound, or with the longest, all of them are written; with a smaller one a head's
    # last rows are, and the status says that it was too small
    new, H, page = np.array([5, 1, 40]), 2, 16
    per = np.repeat(new, H) if compact else new
    N = int(per.sum())
    off = torch.from_numpy(np.concatenate([[0], per.cumsum()]).astype(np.int32)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((N, 128) if compact else (N, H, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    pools = {}
    for most in (None, 40, 39, 8, 1):
        c = Cache(new[:, None].repeat(H, 1), page, bounds=True, seed=4)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        binding.paged_append(c.pages, k, v, offsets=off, status=status, **({} if most is None else dict(max_new=most)))
        assert status.item() == (0 if most in (None, 40) else -1), most
        pools[most] = c.pages.pool
    assert torch.equal(pools[None], pools[40])
    rows, _ = plain.get_rows(pools[40].cpu().numpy(), c.table[2, 1], page, 40)
    last, _ = plain.get_rows(pools[8].cpu().numpy(), c.table[2, 1], page, 40)
    assert np.isfinite(rows).all() and np.isnan(last[:32]).all() and np.array_equal(last[32:], rows[32:])
    c.pages.pool = pools[40]
    kr, vr = binding.paged_read(c.pages, N, offsets=off, compact=compact)
    kq, vq = (plain.values(*plain.quantise(f32(x))) for x in (k, v))
    assert torch.equal(kr.cpu(), torch.from_numpy(kq).bfloat16()) and torch.equal(vr.cpu(), torch.from_numpy(vq).bfloat16())


@pytest.mark.parametrize("ks,vs,top", [(1e-13, 1.0, 9e29), (1.0, 3e-16, 1e25), (1e-20, 1e-25, 1.0), (1e-30, 1e-36, 60000.0),
                                       (1e17, 1e25, 3e18), (1e30, 1e30, 2e38), (0.7, 1.3, 50.0), (3e-5, 700.0, 1e3)])
def test_values_far_from_their_scale(ks, vs, top):
    # quotients from far below a code to far beyond the largest, where a quotient may leave the range of fp32: each keeps its sign.  Scales of
    # every kind of significand
    rng = np.random.default_rng(3)
    n = 64
    x = rng.standard_normal((n, 128)) * top * 10.0 ** rng.uniform(-9, 0, (n, 8)).repeat(16, 1)
    x[0], x[1, :64], x[1, 64:] = -top, top, -top
    x = torch.from_numpy(x).bfloat16().cuda()
    c = Cache([[n]], 16, ks=ks, vs=vs)
    binding.paged_append(c.pages, x, x, offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"), max_new=n)
    k, v = plain.get_rows(c.pool(), c.table[0, 0], 16, n)
    for got, scale in ((k, ks), (v, vs)):
        want = plain.values(*plain.quantise(f32(x), scale))
        assert np.array_equal(got, want)
        assert (want[0] <= 0).all() and (want[1, :64] >= 0).all()


def test_blocks_of_zeros_at_the_least_scale():
    c = Cache([[16]], 16, ks=float(np.finfo(np.float32).tiny), vs=float(np.finfo(np.float32).tiny))
    x = torch.zeros((16, 128), device="cuda").bfloat16()
    x[3], x[5, :16] = 1e-38, 2e-36
    binding.paged_append(c.pages, x, x, offsets=torch.tensor([0, 16], dtype=torch.int32, device="cuda"))
    want = plain.values(*plain.quantise(f32(x), c.pages.k_scale))
    assert all(np.array_equal(got, want) for got in plain.get_rows(c.pool(), c.table[0, 0], 16, 16))
    assert (want[[0, 1, 2, 4]] == 0).all() and (want[3] > 0).all() and (want[5, :16] > 0).all()


@pytest.mark.parametrize("scale", [1.25, 0.7, 1.3])
def test_the_scale_is_a_product_with_the_reciprocal(scale):
    # every fp16 magnitude as a block's largest: the stored byte is that of the product with the rounded reciprocal, worked out here in
    # 64 bits; the quotient max |x| / (6 scale) can have another (46 of them at 1.25, none at 0.7)
    every = np.arange(1, 0x7C00, dtype=np.uint16).view(np.float16).astype(np.float64)
    c = np.float64(np.float32(1.0 / (6.0 * np.float64(np.float32(scale)))))
    byte = lambda y: torch.from_numpy(np.minimum(y, 448.0).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    product = byte(np.float32(every * c).astype(np.float64))
    quotient = byte(every / (6.0 * np.float64(np.float32(scale))))
    assert (product != quotient).sum() == {1.25: 46, 0.7: 0, 1.3: 16}[scale]
    at = np.arange(every.size)
    n = -(-every.size // 8)
    rows = np.zeros((n, 128))
    rows.reshape(-1)[at * 16 + at % 16] = every * np.where(at % 3, 1, -1)
    x = torch.from_numpy(rows).half().cuda()
    cache = Cache([[n]], 16, ks=scale, vs=scale)
    binding.paged_append(cache.pages, x, x, offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"), max_new=n)
    tiles, r = cache.pool().reshape(-1, plain.TILE_BYTES), np.arange(n)
    mine = tiles[cache.table[0, 0, r // 16]]
    for place in (plain.KS_AT, plain.VS_AT):
        assert np.array_equal(mine[r[:, None], place[r % 16]].reshape(-1)[:every.size], product)


def test_a_table_without_heads_is_refused():
    # (the binding divided q's heads by the table's)
    pages = binding.Pages(pool=torch.zeros((1, binding.page_bytes(16)), dtype=torch.uint8, device="cuda"),
                          table=torch.zeros((1, 0, 1), dtype=torch.int32, device="cuda"),
                          rows=torch.zeros((1, 0), dtype=torch.int32, device="cuda"), page_rows=16,
                          bounds=torch.zeros((1, 2, 128), dtype=torch.float16, device="cuda"))
    q = queries(1, 1, 4, "bf16")
    for call in (lambda: binding.paged_attention(pages, q, 16), lambda: binding.paged_select(pages, q, 1, 16),
                 lambda: binding.paged_sparse_attention(pages, q, 1, 16), lambda: binding.paged_workspace(pages, q),
                 lambda: binding.paged_append(pages, torch.zeros((1, 0, 128), device="cuda").half(),
                                              torch.zeros((1, 0, 128), device="cuda").half()),
                 lambda: binding.paged_read(pages, 1)):
        with pytest.raises((AssertionError, binding.MixKVError)):
            call()


def test_the_stride_of_a_dimension_of_one_does_not_matter():
    # one token of one sequence in the output of a projection whose width is no multiple of 16, one KV head
    G, wide = 4, 6 * 128 + 3
    proj = torch.randn((2, wide), generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").bfloat16()
    q = proj[:1].as_strided((1, 1, G, 128), (wide, 7, 128, 1))
    k, v = (proj[:1].as_strided((1, 1, 128), (wide, 5, 1), 128 * i) for i in (4, 5))
    packed = lambda t: torch.empty(t.shape, dtype=t.dtype, device="cuda").copy_(t)
    caches = [Cache([[40]], 16, bounds=True, seed=1) for _ in range(2)]
    outs = []
    for c, (x, y, z) in zip(caches, ((q, k, v), tuple(map(packed, (q, k, v))))):
        c.fill()
        binding.paged_append(c.pages, y, z)
        outs.append((c.pages.pool, binding.paged_attention(c.pages, x), *binding.paged_select(c.pages, x, 2),
                     *binding.paged_sparse_attention(c.pages, x, 2)))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def on_device(t, index):
    """t as a tensor that says it is on CUDA device `index` (there may be no such device: nothing of it may be touched)."""
    class Managed(C.Structure):
        _fields_ = [("data", C.c_void_p), ("device_type", C.c_int32), ("device", C.c_int32), ("ndim", C.c_int32),
                    ("code", C.c_uint8), ("bits", C.c_uint8), ("lanes", C.c_uint16), ("shape", C.POINTER(C.c_int64)),
                    ("strides", C.c_void_p), ("offset", C.c_uint64), ("context", C.c_void_p), ("deleter", C.c_void_p)]
    assert t.dim() == 1 and t.dtype == torch.int32
    size = (C.c_int64 * 1)(t.numel())
    m = Managed(data=t.data_ptr(), device_type=2, device=index, ndim=1, code=0, bits=32, lanes=1, shape=size)
    new = C.pythonapi.PyCapsule_New
    new.restype, new.argtypes = C.py_object, [C.c_void_p, C.c_char_p, C.c_void_p]
    out = torch.utils.dlpack.from_dlpack(new(C.addressof(m), b"dltensor", None))
    out.held = m, size, t
    return out


def test_a_status_word_of_another_device_is_refused():
    c = Cache([[3, 3]], 16)
    k = torch.zeros((1, 2, 128), dtype=torch.bfloat16, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.paged_append(c.pages, k, k, status=on_device(word, 0))
    for bad in (on_device(word, 1), word.cpu(), word[:0], word.float()):
        with pytest.raises(AssertionError):
            binding.paged_append(c.pages, k, k, status=bad)


@pytest.mark.parametrize("gain", [-1e35, -1e32, -1e29, 1e29, 1e35])
@pytest.mark.parametrize("n,T", [(100, 1), (100, 3), (9000, 1)])
def test_logits_of_any_size(gain, n, T):
    # keys of one value, and one of half of it in the second head: with logits this far from zero the first head's output is the mean
    # of its values, the second's the value of the odd key alone, or the mean of the others
    c, odd = Cache([[n, n]], 32), n // 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = torch.ones((2, n, 128), device="cuda"), torch.randn((2, n, 128), generator=gen, device="cuda")
    k[1, odd] = 0.5
    off = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    binding.paged_append(c.pages, k.view(-1, 128).bfloat16(), v.view(-1, 128).bfloat16(), offsets=off, max_new=n)
    q = torch.full((1, T, 4, 128), gain, device="cuda").bfloat16()
    out = binding.paged_attention(c.pages, q)[0].double().cpu().numpy()
    for h in range(2):
        _, V = c.rows_of(0, h)
        for t in range(T):
            seen = np.arange(n - T + 1 + t)
            if h:
                seen = np.array([odd]) if gain < 0 else seen[seen != odd]
            want, mass = V[seen].mean(0), np.abs(V[seen]).mean(0)
            # the output's rounding; sums of n equal weights in fp32
            assert (np.abs(out[t, 2 * h:2 * h + 2] - want) <= 2.0 ** -8 * np.abs(want) + n * 2.0 ** -23 * mass).all(), (h, t)


@pytest.mark.parametrize("G", [2, 7])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_a_query_that_is_no_number_selects_like_nan(bad, G):
    # keys of one sign and keys of zero: bounds that are zero on one side or on both
    c = Cache([[16 * 50] * 4], 16, bounds=True)
    k, v, off = c.fill()
    k = k.view(4, -1, 128).clone()
    k[0], k[1], k[2, ::3] = k[0].abs(), -k[1].abs(), 0.0
    k[:2, 100:300, ::2] = 0.0
    binding.paged_append(c.pages, k.view(-1, 128), v, offsets=off, max_new=800)
    q = queries(1, 1, 4 * G, "bf16", 3)
    q[0, 0, G - 1::G, 20] = bad
    for first, last in ((0, 0), (1, 2)):
        lists, _ = binding.paged_select(c.pages, q, 7, keep_first=first, keep_last=last)
        assert np.array_equal(lists.cpu().numpy(), oracle_select(c, q, 1, G, 7, first, last))
        assert lists[0, 0].tolist() == ([0, 1, 2, 3, 4, 5, 6] if not last else [0, 1, 2, 3, 4, 48, 49])


def test_rows_that_are_taken_back():
    # a draft of six tokens behind 29 rows (pages of 16), of which two are kept; then four others.  Rows and attention are those of a
    # cache that never saw the rejected ones; bounds of the page that kept rows cover them as well, those of the page that begins anew do not
    H, G, page = 2, 4, 16
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((39, H, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    kept = list(range(31)) + list(range(35, 39))
    for nan in (False, True):
        if nan:
            k[31, 1, 9] = float("nan")        # the first rejected token, row 31 of the second page
        c, clean = (Cache([[35, 35]], page, bounds=True, seed=1) for _ in range(2))

        def put(cache, rows, tokens):
            cache.pages.rows.fill_(rows)
            off = torch.tensor([0, len(tokens)], dtype=torch.int32, device="cuda")
            binding.paged_append(cache.pages, k[tokens], v[tokens], offsets=off)

        put(c, 29, list(range(29)))
        put(c, 35, list(range(29, 35)))
        put(c, 35, kept[31:])
        put(clean, 35, kept)
        q = queries(1, 4, H * G, "bf16")
        assert torch.equal(binding.paged_attention(c.pages, q), binding.paged_attention(clean.pages, q))
        values = plain.values(*plain.quantise(f32(k)))
        for h in range(H):
            ids = c.table[0, h]
            got = c.pages.bounds.double().cpu().numpy()[ids]
            had = [kept[:16], kept[16:31] + [31, 35], kept[32:]]     # (row 31: the rejected token, then the one that took its place)
            for p, rows in enumerate(had):
                assert np.array_equal(got[p], [values[rows, h].min(0), values[rows, h].max(0)], equal_nan=True)
            lists, _ = binding.paged_select(c.pages, q[:, :1], 1, keep_first=0, keep_last=0)
            assert not (nan and h) or lists[0, 1].tolist() == [1]


@pytest.mark.parametrize("ks,vs", [(1.0, 1e-37), (1e-37, 1e30), (1.3, 0.7), (1e3, 1e-30)])
@pytest.mark.parametrize("lens", [[[700, 33]], [[9000, 5000]], [[300] * 4] * 40])
def test_caches_of_any_scale(lens, ks, vs):
    # rows whose K is of the size of k_scale, V of that of v_scale, attended to by queries that make logits of ordinary size, over
    # clusters, shares and single CTAs: outputs of the size of v_scale, with the error of ordinary ones
    lens = np.array(lens)
    c = Cache(lens, 32, ks=ks, vs=vs, seed=2)
    n, off = int(lens.sum()), torch.from_numpy(np.concatenate([[0], lens.reshape(-1).cumsum()]).astype(np.int32)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((n, 128), generator=gen, device="cuda") for _ in range(2))
    binding.paged_append(c.pages, (k * ks).bfloat16(), (v * vs).bfloat16(), offsets=off, max_new=int(lens.max()))
    B, H = lens.shape
    q = (torch.randn((B, 1, 3 * H, 128), generator=gen, device="cuda") / ks).bfloat16()
    out = binding.paged_attention(c.pages, q).double().cpu().numpy() / vs
    qf = q.double().cpu().numpy() * ks
    for b, h in {(0, 0), (B - 1, H - 1)}:
        K, V = plain.get_rows(c.pool(), c.table[b, h], 32, int(lens[b, h]))
        want, mass, size = plain.attention(qf[b, :, 3 * h:3 * h + 3], K, V, 1, 1 / np.sqrt(128))
        off_by = 2.0 ** -23 * 128 * size[..., None] + 2.0 ** -20
        tol = 2.0 ** -8 * np.abs(want) + mass * (2.0 ** -11 + 2 * off_by) + lens[b, h] * 2.0 ** -31 * np.abs(V).max()
        assert (np.abs(out[b, :, 3 * h:3 * h + 3] - want) <= tol).all(), (b, h)


@pytest.mark.parametrize("lens", [[[70000]], [[900, 7]], [[4000, 4000]]])
def test_many_equal_weights_at_the_least_scale(lens):
    # (the quotient of the least scale and a sum of weights is subnormal; the output is not)
    lens, vs = np.array(lens), float(np.finfo(np.float32).tiny)
    c = Cache(lens, 64, vs=vs, seed=2)
    n, off = int(lens.sum()), torch.from_numpy(np.concatenate([[0], lens.reshape(-1).cumsum()]).astype(np.int32)).cuda()
    k, v = torch.ones((n, 128), device="cuda").bfloat16(), torch.full((n, 128), 3 * vs, device="cuda").bfloat16()
    binding.paged_append(c.pages, k, v, offsets=off, max_new=int(lens.max()))
    out = binding.paged_attention(c.pages, torch.zeros((1, 1, 2 * lens.shape[1], 128), dtype=torch.bfloat16, device="cuda"))
    V = c.rows_of(0, 0)[1]
    assert (np.abs(out.double().cpu().numpy() - V[0, 0]) <= 2.0 ** -8 * V[0, 0]).all() and (V == V[0, 0]).all()
