"""GPU parity of the paged 8-bit cache (append, read back, attention with window, sinks and weights, eviction) against its plain
definition."""
import numpy as np
import pytest
import torch

from oracle import cache8_plain as plain
from paper_2510_20707_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def f32(t):
    return t.float().cpu().numpy()


class Cache:
    """A cache of `lens` [batch][heads] rows behind a shuffled page table; every byte starts as 0xff (scales and codes of NaN), every mass
    as -5."""

    def __init__(self, lens, page=32, code="int8", seed=0, spare=2, room=0, mass=True):
        lens = np.asarray(lens)
        rng = np.random.default_rng(seed)
        count = -(-np.maximum(lens, room) // page)
        cols, total = max(1, int(count.max())), int(count.sum())
        table = np.full((*lens.shape, cols), -1, np.int32)
        table[np.arange(cols) < count[..., None]] = rng.permutation(total + spare)[:total]
        self.lens, self.table, self.page, self.code = lens.copy(), table, page, code
        n = total + spare
        self.cache = binding.Cache8(
            pool=torch.full((n, binding.cache8_page_bytes(page)), 0xFF, dtype=torch.uint8, device="cuda"), table=dev(table),
            rows=dev(lens.astype(np.int32)), page_rows=page, code=code, mass=torch.full((n, page), -5.0, device="cuda") if mass else None)
        self.want = np.full((n, binding.cache8_page_bytes(page)), 0xFF, np.uint8)

    def count(self, lens):
        self.lens = np.asarray(lens).copy()
        self.cache.rows.copy_(dev(self.lens.astype(np.int32)))

    def pool(self):
        return self.cache.pool.cpu().numpy()

    def same_pool(self):
        """Whether the bytes that have a meaning are those of `want`."""
        got, want = (x.reshape(-1, plain.TILE_BYTES)[:, :4104] for x in (self.pool(), self.want))
        nan = lambda x: np.isnan(x[:, 4096:].copy().view(np.float32))
        assert np.array_equal(nan(got), nan(want))
        ok = np.concatenate([np.ones((len(got), 4096), bool), ~nan(got).repeat(4, 1)], 1)
        bad = np.flatnonzero((got != want)[:, :][ok].ravel())
        assert not len(bad), (len(bad), np.argwhere((got != want) & ok)[:5])

    def expect(self, b, h, held, k, v):
        plain.append(self.want, self.table[b, h], self.page, held, k, v, self.code)

    def rows_of(self, b, h):
        return plain.rows_of(self.pool(), self.table[b, h], self.page, int(self.lens[b, h]), self.code)

    def mass_of(self, b, h, n=None):
        r = np.arange(int(self.lens[b, h]) if n is None else n)
        return self.cache.mass.cpu().numpy()[self.table[b, h, r // self.page], r % self.page]

    def fill(self, seed=1, k_gain=1.0, dtype=torch.bfloat16):
        """Random rows everywhere."""
        flat = self.lens.reshape(-1)
        off = dev(np.concatenate([[0], flat.cumsum()]).astype(np.int32))
        gen = torch.Generator(device="cuda").manual_seed(seed)
        n = int(flat.sum())
        k, v = (torch.randn((max(n, 1), 128), generator=gen, device="cuda") for _ in range(2))
        k[:, 3::31] *= 3.0
        k, v = (k * k_gain).to(dtype)[:n], v.to(dtype)[:n]
        binding.cache8_append(self.cache, k, v, offsets=off, max_new=max(1, int(flat.max())))
        return k, v, off


# ------------------------------------------------------------------------------------------------ rows
@pytest.mark.parametrize("dtype,code,page,H", [("bf16", "int8", 16, 3), ("fp16", "e4m3", 32, 1), ("bf16", "e4m3", 64, 2), ("fp16", "int8", 48, 5),
                                               ("bf16", "int8", 256, 2)])
def test_append_and_read_back(dtype, code, page, H):
    # new rows of several sequences (none, one, a page and more) behind rows that are there, K and V slices of one tensor
    new, old = np.array([0, 1, 17, 2 * page + 5, 15, 16]), np.array([3, page - 1, 2, page // 2 + 1, 0, 16])
    B, N = len(new), int(new.sum())
    c = Cache(old[:, None].repeat(H, 1), page, code, seed=page, room=int((old + new).max()))
    k0, v0, off0 = c.fill(seed=2, dtype=TYPES[dtype])
    i = 0
    for b in range(B):
        for h in range(H):
            c.expect(b, h, 0, f32(k0)[i:i + old[b]], f32(v0)[i:i + old[b]])
            i += old[b]
    c.same_pool()
    gen = torch.Generator(device="cuda").manual_seed(page)
    qkv = torch.randn((N, 3 * H, 128), generator=gen, device="cuda")
    qkv[::2] *= 2.0       # (some blocks grow, some do not)
    qkv = qkv.to(TYPES[dtype])
    k, v = qkv[:, H:2 * H], qkv[:, 2 * H:]
    off = np.concatenate([[0], new.cumsum()]).astype(np.int32)
    c.count((old + new)[:, None].repeat(H, 1))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = c.cache.mass.clone()
    binding.cache8_append(c.cache, k, v, offsets=dev(off), max_new=int(new.max()), status=status)
    assert status.item() == 0
    mass = before.cpu().numpy()
    for b in range(B):
        for h in range(H):
            c.expect(b, h, int(old[b]), f32(k)[off[b]:off[b + 1], h], f32(v)[off[b]:off[b + 1], h])
            r = np.arange(old[b], old[b] + new[b])
            mass[c.table[b, h, r // page], r % page] = 0
    c.same_pool()
    assert np.array_equal(c.cache.mass.cpu().numpy(), mass)
    kr, vr = binding.cache8_read(c.cache, N, TYPES[dtype], offsets=dev(off), max_new=int(new.max()))
    for b in range(B):
        for h in range(H):
            for got, want in zip((kr, vr), c.rows_of(b, h)):
                assert torch.equal(got[off[b]:off[b + 1], h].cpu(), torch.from_numpy(want[old[b]:]).to(TYPES[dtype]))


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_tokens_one_by_one(code):
    # forty tokens of three sequences, one a call, of magnitudes that rise and fall; then five are taken back and written anew
    B, H, page = 3, 2, 32
    c = Cache(np.zeros((B, H), int), page, code, room=64)
    rng = np.random.default_rng(3)
    gain = rng.choice([0.1, 1.0, 3.0, 10.0], 45)
    for i in range(45):
        n = i if i < 40 else i - 5
        k, v = (dev((rng.standard_normal((B, H, 128)) * g).astype(np.float32)).bfloat16() for g in (gain[i], 1 + i / 7))
        c.count(np.full((B, H), n + 1))
        binding.cache8_append(c.cache, k, v)
        for b in range(B):
            for h in range(H):
                c.expect(b, h, n, f32(k)[b, h][None], f32(v)[b, h][None])
    c.same_pool()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_values_of_every_kind(code):
    # blocks of zeros, of subnormal numbers, of extreme ones, of codes that lie at ties, with a NaN, with an infinity
    rng = np.random.default_rng(4)
    x = np.zeros((8, 16, 128), np.float32)
    x[1] = rng.standard_normal((16, 128)) * 1e-39
    x[2] = rng.standard_normal((16, 128)) * 1e-36
    x[3] = rng.standard_normal((16, 128)) * 1e37
    x[4] = (rng.integers(-253, 254, (16, 128)) / 2).astype(np.float32)
    x[4, 0, 0] = 127
    x[5] = -0.0
    x[6] = rng.standard_normal((16, 128))
    x[6, 3, 5] = np.nan
    x[7] = rng.standard_normal((16, 128))
    x[7, 15, 127] = -np.inf
    rows = dev(x.reshape(-1, 128)).bfloat16()
    c = Cache(np.full((1, 1), 128), 64, code)
    off = dev(np.array([0, 128], np.int32))
    binding.cache8_append(c.cache, rows, rows.flip(0), offsets=off)
    c.expect(0, 0, 0, f32(rows), f32(rows.flip(0)))
    c.same_pool()
    back = binding.cache8_read(c.cache, 128, torch.bfloat16, offsets=off, compact=True)[0]
    assert torch.isnan(back[96:]).all() and not torch.isnan(back[:96]).any()


def test_rows_without_a_place_are_reported_and_the_others_written():
    page, H = 16, 2
    lens = np.array([[20, 20], [40, 40], [5, 5], [18, 18]])
    c = Cache(lens, page, spare=3)
    c.table[0, 1, 1] = c.want.shape[0]      # a page past the pool
    c.table[1, 0, 0] = -7
    c.cache.table.copy_(dev(c.table))
    off = np.array([0, 20, 70, 75, 91], np.int32)      # the second sequence has ten more tokens than rows, the fourth five less
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((89, H, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))      # two tokens are missing
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.cache8_append(c.cache, k, v, offsets=dev(off), max_new=50, status=status)
    assert status.item() == -1
    kx, vx = f32(k), f32(v)
    tiles = c.want.reshape(-1, plain.TILE_BYTES)
    for b, h, rows, token in [(0, 0, range(20), 0), (0, 1, range(16), 0), (1, 0, range(16, 40), 30), (1, 1, range(40), 30), (2, 0, range(5), 70),
                              (2, 1, range(5), 70)]:
        for t in sorted({r // 16 for r in rows}):
            r = [x for x in rows if x // 16 == t]
            at = [token + x for x in r]
            for i, x in enumerate((kx, vx)):
                plain.put(tiles[c.table[b, h, t]], i, r[0] % 16, x[at, h], "int8", False)
    for h in range(H):      # rows 2 .. 17 are new, tokens 75 .. 90, of which 89 and 90 do not exist; rows 0 and 1 are from before: 0xff
        for i, x in enumerate((kx, vx)):
            tile = tiles[c.table[3, h, 0]]
            plain.scales_at(tile)[i] = np.nan
            tile[2048 * i + plain.AT] = 0
            tile = tiles[c.table[3, h, 1]]
            plain.scales_at(tile)[i] = 0
            tile[2048 * i + plain.AT] = 0
    c.same_pool()


@pytest.mark.parametrize("max_new", [1, 7, 16, 40])
def test_of_more_rows_than_max_new_the_last_are_written(max_new):
    c = Cache(np.array([[37], [50]]), 32)
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((87, 128), generator=gen, device="cuda").half() for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.cache8_append(c.cache, k, v, offsets=dev(np.array([0, 37, 87], np.int32)), max_new=max_new, status=status)
    assert status.item() == -1
    per = 2
    for b, first, n in ((0, 0, 37), (1, 37, 50)):
        lo = max(0, n - max_new)
        for t in range(lo // 16, (n - 1) // 16 + 1):      # (every block begins in this call: rows before lo count as new)
            r = np.arange(max(lo, 16 * t), min(n, 16 * t + 16))
            for i, x in enumerate((k, v)):
                plain.put(c.want.reshape(-1, plain.TILE_BYTES)[c.table[b, 0, t // per] * per + t % per], i, r[0] % 16, f32(x)[first + r], "int8",
                          False)
    c.same_pool()
    # and the last rows are read
    kr, _ = binding.cache8_read(c.cache, 87, torch.float16, offsets=dev(np.array([0, 37, 87], np.int32)), max_new=max_new, compact=True)
    want = c.rows_of(1, 0)[0][-max_new:]
    assert np.array_equal(f32(kr[-len(want):]), want.astype(np.float16).astype(np.float32))


# ------------------------------------------------------------------------------------------- attention
def close(got, ref, aw, dtype, n, vmax):
    """Outputs differ by their own rounding, by one rounding of every weight to fp16 (2^-11 of it; weights below 2^-14 of fp16's range, of which
    the sum is 2^6 at least, by 2^-25 / 2^6 each), and by fp32 sums, which n products of either sign change by n 2^-24 at most, far less as
    a rule (allowed: 2^-14)."""
    half = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype]
    tol = half * np.abs(ref) + (2.0 ** -11 + 2.0 ** -14) * aw * (1 + half) + n * 2.0 ** -31 * vmax + 2.0 ** -24
    bad = np.abs(got - ref) > tol
    assert not bad.any(), (np.abs(got - ref)[bad].max(), np.argwhere(bad)[:4], (np.abs(got - ref) / tol).max())


def check_attention(c, q, dtype, scale, window=0, sinks=0, out=None, added=None, skip=()):
    """Outputs, and what was added to the masses (fp32 [pages, page]), against 64 bits."""
    B, T, HG, _ = q.shape
    H = c.lens.shape[1]
    G, got, qx = HG // H, out.double().cpu().numpy(), q.double().cpu().numpy()
    want = np.zeros(added.shape) if added is not None else None
    tol = np.zeros(added.shape) if added is not None else None
    for b in range(B):
        for h in range(H):
            if (b, h) in skip:
                continue
            K, V = c.rows_of(b, h)
            qq = qx[b, :, h * G:(h + 1) * G]
            ref, w, aw = plain.attention(qq, K, V, scale, window, sinks)
            close(got[b, :, h * G:(h + 1) * G], ref, aw, dtype, len(K), np.abs(V).max(initial=0))
            if added is not None and len(K):
                r = np.arange(len(K))
                at = c.table[b, h, r // c.page], r % c.page
                want[at] = w.sum((0, 1))
                # a logit's 128 products are summed in fp32, each sum rounded or cut: 2^-23 of the sum of magnitudes at most, for each
                # of 128 (a weight changes by as much of itself, twice with its row's sum); exponentials, products and sums: 2^-19
                size = np.abs(qq) @ np.abs(K).T * scale
                tol[at] = (w * (2.0 ** -15 * size.max(-1, keepdims=True) + 2.0 ** -19)).sum((0, 1))
    if added is not None:
        a = added.double().cpu().numpy()
        assert (np.abs(a - want) <= tol + 1e-30).all(), np.nanmax(np.abs(a - want) - tol)


def query(B, T, HG, dtype, seed=0, gain=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((B, T, HG, 128), generator=gen, device="cuda") * gain).to(TYPES[dtype])


@pytest.mark.parametrize("dtype,code,T,G,page,lens,window,sinks", [
    ("bf16", "int8", 1, 7, 64, [[512] * 4], 0, 0),
    ("bf16", "e4m3", 1, 1, 16, [[1, 15], [16, 17], [0, 33]], 0, 0),
    ("fp16", "int8", 3, 4, 32, [[2, 3], [16, 100], [0, 1]], 0, 0),
    ("fp16", "e4m3", 5, 7, 64, [[2051, 777]], 0, 0),
    ("bf16", "int8", 8, 16, 128, [[300], [9]], 0, 0),
    ("bf16", "e4m3", 2, 12, 48, [[1000, 640, 65]], 0, 0),
    ("fp16", "int8", 1, 8, 256, [[5000, 300], [4097, 1]], 0, 0),
    ("bf16", "int8", 1, 4, 64, [[20001] * 2, [131] * 2], 0, 0),
    ("bf16", "int8", 1, 4, 64, [[3000, 20], [100, 1]], 64, 4),
    ("fp16", "e4m3", 4, 7, 16, [[500, 37], [36, 3]], 33, 0),
    ("bf16", "e4m3", 3, 5, 32, [[700, 90], [20, 2]], 1, 17),
    ("fp16", "int8", 1, 2, 64, [[9000, 4000, 15]], 2500, 64),
    ("bf16", "int8", 2, 3, 32, [[300, 40]], 1000, 4),
    ("bf16", "int8", 32, 4, 32, [[100, 31], [40, 32]], 20, 3),
    ("fp16", "e4m3", 1, 128, 64, [[200, 100]], 0, 0)])
def test_attention(dtype, code, T, G, page, lens, window, sinks):
    c = Cache(lens, page, code, seed=T)
    c.fill(dtype=TYPES[dtype])
    c.cache.mass.fill_(0.0)
    B, H = c.lens.shape
    q = query(B, T, H * G, dtype)
    out = binding.cache8_attention(c.cache, q, window=window, sinks=sinks, accumulate=True)
    check_attention(c, q, dtype, 128 ** -0.5, window, sinks, out, c.cache.mass)
    # without the weights the same outputs, bit for bit; a second call adds to the masses
    again = binding.cache8_attention(c.cache, q, window=window, sinks=sinks)
    assert torch.equal(out, again)
    once = c.cache.mass.clone()
    binding.cache8_attention(c.cache, q, window=window, sinks=sinks, accumulate=True)
    assert torch.equal(c.cache.mass, once + once)


@pytest.mark.parametrize("B,H,G,T,rows", [(1, 8, 4, 1, 40000), (70, 8, 7, 1, 600), (1100, 1, 2, 1, 60), (16, 4, 5, 4, 3000), (40, 8, 1, 1, 3001)])
@pytest.mark.parametrize("own", [False, True])
def test_attention_however_it_is_split(B, H, G, T, rows, own):
    # one cluster a head, all tiles dealt out, more heads than are dealt out; lengths alike and from one row up
    rng = np.random.default_rng(rows)
    lens = rng.integers(1, rows + 1, (B, H)) if own else np.full((B, H), rows)
    c = Cache(lens, 64, "int8")
    c.fill()
    c.cache.mass.fill_(0.0)
    q = query(B, T, H * G, "bf16")
    out = binding.cache8_attention(c.cache, q, max_rows=rows, accumulate=True)
    some = {(b, h) for b in rng.permutation(B)[:4] for h in rng.permutation(H)[:2]}
    check_attention(c, q, "bf16", 128 ** -0.5, 0, 0, out, None, {(b, h) for b in range(B) for h in range(H)} - some)
    for b in range(0, B, 7):     # a head's weights sum to the number of its query rows
        for h in range(H):
            seen = sum(1 for t in range(T) if c.lens[b, h] - T + t >= 0) * G
            assert abs(c.mass_of(b, h).astype(np.float64).sum() - seen) < 1e-4 * max(1, seen)


def test_queries_and_scales_far_from_one():
    # large and tiny queries and keys, another softmax scale, values of 1e30 beside values of 1e-30
    for q_gain, k_gain, scale in ((3e4, 1e-5, 0.0), (1e-30, 1e30, 0.05), (2e30, 3e-32, 0.2), (40.0, 3.0, 0.0)):
        c = Cache([[200, 77]], 32, "int8")
        c.fill(k_gain=k_gain)
        q = query(1, 2, 6, "bf16", gain=q_gain)
        out = binding.cache8_attention(c.cache, q, softmax_scale=scale)
        check_attention(c, q, "bf16", float(np.float32(scale or 128 ** -0.5)), 0, 0, out)
    c = Cache([[64]], 32, "e4m3")
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((64, 128), generator=gen, device="cuda") for _ in range(2))
    v[:16] *= 1e30
    v[16:32] *= 1e-30
    v[48:] = 0
    binding.cache8_append(c.cache, k.bfloat16(), v.bfloat16(), offsets=dev(np.array([0, 64], np.int32)))
    q = query(1, 1, 4, "bf16")
    check_attention(c, q, "bf16", 128 ** -0.5, 0, 0, binding.cache8_attention(c.cache, q))


def test_nan_and_infinite_rows_reach_those_that_see_them_alone():
    # a query of NaN, one of infinities; a block of NaN that the first of two tokens does not see yet, one that the second sees no more
    c = Cache([[33, 65]], 16, "int8")
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((98, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    k[32, 3], v[32, 4] = float("nan"), float("inf")      # row 32 of the first head, alone in its block
    v[33 + 15, 0] = float("nan")                         # row 15 of the second
    off = dev(np.array([0, 33, 98], np.int32))
    binding.cache8_append(c.cache, k, v, offsets=off)
    q = query(1, 2, 4, "bf16")
    out = binding.cache8_attention(c.cache, q)
    assert not torch.isnan(out[0, 0, :2]).any() and torch.isnan(out[0, 1, :2]).all() and torch.isnan(out[0, :, 2:]).all()
    # rows 15 .. 63 and 16 .. 64
    out = binding.cache8_attention(c.cache, q, window=49, sinks=0)
    assert torch.isnan(out[0, 0, 2:]).all() and not torch.isnan(out[0, 1, 2:]).any()
    ref = plain.attention(q.double().cpu().numpy()[0, 1:, 2:], *(x[16:] for x in c.rows_of(0, 1)), 128 ** -0.5)
    close(out[0, 1:, 2:].double().cpu().numpy(), ref[0], ref[2], "bf16", 65, 5.0)
    c.cache.mass.fill_(0.0)
    q[0, 0, 0, 5], q[0, 1, 1, 7] = float("nan"), float("-inf")
    out = binding.cache8_attention(c.cache, q, window=17, accumulate=True)      # (second head: rows 47 .. 63 and 48 .. 64)
    assert torch.isnan(out[0, 0, 0]).all() and not torch.isnan(out[0, 0, 1]).any() and torch.isnan(out[0, 1, :2]).all()
    assert not torch.isnan(out[0, :, 2:]).any()
    # the mass of rows that a row of NaN sees is NaN, that of others is not
    m = c.mass_of(0, 0)
    assert np.isnan(m[15:33]).all() and (m[:15] == 0).all() and not np.isnan(c.mass_of(0, 1)).any()


def test_pages_outside_the_pool_have_no_rows():
    c = Cache([[100, 70]], 16, "int8")
    c.fill()
    rows = c.rows_of(0, 0)
    c.table[0, 0, 2], c.table[0, 0, 6] = -1, 1 << 30
    c.cache.table.copy_(dev(c.table))
    c.cache.mass.fill_(0.0)
    q = query(1, 1, 6, "fp16")
    out = binding.cache8_attention(c.cache, q, accumulate=True)
    left = np.r_[0:32, 48:96]
    ref, w, aw = plain.attention(q.double().cpu().numpy()[0, :, :3], *(x[left] for x in rows), 128 ** -0.5)
    close(out[0, :, :3].double().cpu().numpy(), ref, aw, "fp16", 80, 5.0)
    got = c.cache.mass.cpu().numpy()[c.table[0, 0][left // 16], left % 16]
    assert np.allclose(got, w.sum((0, 1)), rtol=1e-4)
    check_attention(c, q, "fp16", 128 ** -0.5, 0, 0, out, None, {(0, 0)})


def test_rows_beyond_max_rows_do_not_exist():
    c = Cache([[100, 40]], 16, "e4m3")
    c.fill()
    c.cache.mass.fill_(0.0)
    q = query(1, 2, 6, "bf16")
    out = binding.cache8_attention(c.cache, q, max_rows=50, accumulate=True)
    m = c.mass_of(0, 0)
    c.lens[0, 0] = 50
    check_attention(c, q, "bf16", 128 ** -0.5, 0, 0, out)
    assert (m[50:] == 0).all() and abs(m.sum() - 6) < 1e-3


def test_strided_queries_and_a_stream_of_its_own():
    c = Cache([[300, 40], [77, 2]], 32, "int8")
    c.fill()
    c.cache.mass.fill_(0.0)
    wide = query(2, 5, 18, "bf16")
    q = wide[:, 1:4, 6:12]       # tokens and sequences strided
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = binding.cache8_attention(c.cache, q, accumulate=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check_attention(c, q, "bf16", 128 ** -0.5, 0, 0, out, c.cache.mass)


# -------------------------------------------------------------------------------------------- eviction
def evict_and_check(c, budget, budgets=None, first=0, last=0, page=None, max_rows=None, room=None):
    lens = c.lens if max_rows is None else np.minimum(c.lens, max_rows)
    each = np.full(lens.shape, budget) if budgets is None else np.clip(budgets, first + last, budget)
    kept = np.minimum(lens, each)
    into = Cache(np.zeros_like(lens), page or c.page, c.code, seed=7, room=int(kept.max()) if room is None else room)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = c.cache.pool.clone(), c.cache.mass.clone()
    idx = binding.cache8_evict(c.cache, into.cache, budget, budgets=None if budgets is None else dev(budgets.astype(np.int32)),
                               keep_first=first, keep_last=last, max_rows=max_rows, status=status)
    assert status.item() == 0 and idx.shape == (*lens.shape, budget)
    assert torch.equal(before[0], c.cache.pool) and torch.equal(before[1].view(torch.int32), c.cache.mass.view(torch.int32))
    assert np.array_equal(into.cache.rows.cpu().numpy(), kept)
    idx, pool, mass = idx.cpu().numpy(), c.pool(), into.cache.mass.cpu().numpy()
    for b in range(lens.shape[0]):
        for h in range(lens.shape[1]):
            m = c.mass_of(b, h, lens[b, h])
            want = plain.kept_rows(m, int(each[b, h]), first, last)
            assert np.array_equal(idx[b, h, :len(want)], want) and (idx[b, h, len(want):] == -1).all(), (b, h)
            k, v = plain.rows_of(pool, c.table[b, h], c.page, int(lens[b, h]), c.code)
            into.expect(b, h, 0, k[want], v[want])
            r = np.arange(len(want))
            assert np.array_equal(mass[into.table[b, h, r // into.page], r % into.page].view(np.int32), m[want].view(np.int32))
    into.same_pool()
    into.lens = kept
    return into


def masses(shape, seed=0, ties=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    m = torch.exp(2 * torch.randn(shape, generator=gen, device="cuda"))
    return (m * 2).round() / 2 if ties else m


@pytest.mark.parametrize("code,page,lens,budget,first,last,ties", [
    ("int8", 32, [[100, 64], [65, 3]], 64, 0, 0, False), ("e4m3", 16, [[100, 40], [300, 20]], 33, 4, 16, True),
    ("int8", 64, [[5000, 1]], 700, 1, 0, True), ("e4m3", 128, [[2049], [2048]], 2000, 4, 32, False), ("int8", 48, [[700, 500]], 1, 0, 0, False),
    ("int8", 16, [[90, 0]], 20, 10, 10, False), ("int8", 32, [[90, 50]], 1, 0, 1, True)])
def test_eviction(code, page, lens, budget, first, last, ties):
    c = Cache(lens, page, code, seed=budget)
    c.fill()
    c.cache.mass.copy_(masses(c.cache.mass.shape, 1, ties))
    evict_and_check(c, budget, None, first, last)
    evict_and_check(c, budget, None, first, last, page=16 if page != 16 else 64)


def test_eviction_of_many_heads_with_budgets_of_their_own():
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 400, (60, 4))
    c = Cache(lens, 16, "int8")
    c.fill()
    c.cache.mass.copy_(masses(c.cache.mass.shape, 2, True))
    evict_and_check(c, 128, rng.integers(-5, 200, (60, 4)), 3, 8)
    evict_and_check(c, 128, rng.integers(0, 200, (60, 4)), 0, 0, max_rows=150)


def test_eviction_of_one_long_head():
    # (keys that do not fit the shared memory of eight CTAs are read again for every digit)
    n = 8 * 40960 + 4321
    c = Cache([[n]], 256, "int8")
    c.cache.pool.zero_()
    m = masses(c.cache.mass.shape, 3)
    c.cache.mass.copy_(m)
    idx = binding.cache8_evict(c.cache, binding.new_cache8(1, 1, 5000, 64), 5000, keep_first=4, keep_last=64)
    got, mine = idx.cpu().numpy()[0, 0], c.mass_of(0, 0)
    best = np.sort(np.argsort(-mine[4:n - 64], kind="stable")[:5000 - 68] + 4)
    assert np.array_equal(got, np.r_[0:4, best, n - 64:n])


def test_masses_of_every_kind():
    # NaN, infinities, zeros of both signs, negative numbers, all alike
    c = Cache([[64, 64, 64]], 16, "int8")
    c.fill()
    rng = np.random.default_rng(1)
    m = c.cache.mass.cpu().numpy()
    r = np.arange(64)
    at = lambda h: (c.table[0, h, r // 16], r % 16)
    kinds = np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1.0, 3.0, 1e38, -np.nan], np.float32)
    m[at(0)] = kinds[rng.integers(0, len(kinds), 64)]
    m[at(1)] = 2.5
    m[at(2)] = np.where(rng.random(64) < 0.5, 0.0, -0.0)
    c.cache.mass.copy_(dev(m))
    for budget in (3, 20, 40, 63):
        evict_and_check(c, budget, None, 1, 2)


def test_an_eviction_into_the_pool_it_comes_from_and_without_masses_of_its_own():
    c = Cache([[100, 80]], 16, "int8", spare=20)
    c.fill()
    c.cache.mass.copy_(masses(c.cache.mass.shape, 4))
    free = np.setdiff1d(np.arange(c.want.shape[0]), c.table[c.table >= 0])
    table = np.full((1, 2, 3), -1, np.int32)
    table[0, 0], table[0, 1] = free[:3], free[3:6]
    into = binding.Cache8(pool=c.cache.pool, table=dev(table), rows=torch.zeros((1, 2), dtype=torch.int32, device="cuda"), page_rows=16)
    before, old = c.pool(), [c.rows_of(0, h) for h in range(2)]
    idx = binding.cache8_evict(c.cache, into, 48, keep_last=5).cpu().numpy()
    want = before.copy()
    for h in range(2):
        rows = plain.kept_rows(c.mass_of(0, h), 48, 0, 5)
        assert np.array_equal(idx[0, h], rows)
        plain.append(want, table[0, h], 16, 0, *(x[rows] for x in old[h]), "int8")
    got = c.pool()
    for x in (got, want):      # (the spare bytes)
        x.reshape(-1, plain.TILE_BYTES)[:, 4104:] = 0
    assert np.array_equal(got, want)
    # a table that is too short, and a page that is none: reported, the others written
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    into.table = dev(np.array([[[free[0], free[1]], [free[3], -1]]], np.int32))
    binding.cache8_evict(c.cache, into, 48, keep_last=5, status=status)
    assert status.item() == -1 and into.rows.tolist() == [[48, 48]]


def test_rows_on_pages_outside_the_pool_go_first_and_are_zeros():
    c = Cache([[64]], 16, "int8")
    c.fill()
    c.cache.mass.fill_(-1e30)
    c.table[0, 0, 1] = 1 << 30
    c.cache.table.copy_(dev(c.table))
    into = binding.new_cache8(1, 1, 64, 16, mass=True)
    idx = binding.cache8_evict(c.cache, into, 48).cpu().numpy()[0, 0]
    assert np.array_equal(idx, np.r_[0:16, 32:64])
    idx = binding.cache8_evict(c.cache, into, 50, keep_first=18).cpu().numpy()[0, 0]
    assert np.array_equal(idx, np.r_[0:18, 32:64])
    k = binding.cache8_read(into, 50, torch.float16, offsets=dev(np.array([0, 50], np.int32)), compact=True)[0]
    assert (k[16:18] == 0).all() and (k[:16] != 0).any() and (into.mass.view(-1)[16:18] == 0).all()


# ------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_an_answer_with_eviction_step_by_step(code):
    # Append, attend with the weights counted, evict when a head is over its budget: two caches in turn, against 64 bits all along
    B, H, G, page, budget, spare = 2, 2, 3, 16, 40, 8
    here, there = (Cache(np.zeros((B, H), int), page, code, seed=s, room=budget + spare) for s in (1, 2))
    rng = np.random.default_rng(0)
    mass = [[np.zeros(0) for _ in range(H)] for _ in range(B)]
    n = 0
    for step in range(60):
        T = 1 if step % 3 else 2
        k, v = (dev(rng.standard_normal((B * T, H, 128)).astype(np.float32)).bfloat16() for _ in range(2))
        n += T
        here.count(np.full((B, H), n))
        binding.cache8_append(here.cache, k, v, offsets=dev(np.arange(0, B * T + 1, T, dtype=np.int32)), max_new=T)
        q = query(B, T, H * G, "bf16", seed=step)
        window, sinks = ((0, 0), (24, 2))[step % 2]
        out = binding.cache8_attention(here.cache, q, max_rows=budget + spare, window=window, sinks=sinks, accumulate=True)
        check_attention(here, q, "bf16", 128 ** -0.5, window, sinks, out)
        for b in range(B):
            for h in range(H):
                w = plain.attention(q.double().cpu().numpy()[b, :, h * G:(h + 1) * G], *here.rows_of(b, h), 128 ** -0.5, window, sinks)[1]
                mass[b][h] = np.concatenate([mass[b][h], np.zeros(T)]) + w.sum((0, 1))
                assert np.allclose(here.mass_of(b, h), mass[b][h], rtol=1e-4, atol=1e-6)
        if n > budget:
            idx = binding.cache8_evict(here.cache, there.cache, budget - spare, keep_first=2, keep_last=4, max_rows=n).cpu().numpy()
            for b in range(B):
                for h in range(H):
                    m = here.mass_of(b, h)
                    assert np.array_equal(idx[b, h], plain.kept_rows(m, budget - spare, 2, 4))
                    mass[b][h] = mass[b][h][idx[b, h]]
            n = budget - spare
            here, there = there, here
            here.lens[:] = n
            assert (here.cache.rows == n).all()


def test_calls_in_a_graph():
    # one step captured and replayed with new inputs: append, attend with weights, evict
    c = Cache(np.full((2, 2), 200), 32, "int8", room=224)
    c.fill()
    c.cache.mass.copy_(masses(c.cache.mass.shape, 5))
    into = binding.new_cache8(2, 2, 96, 32, mass=True)
    k, v, q = query(2, 2, 1, "bf16", 1)[:, :, 0], query(2, 2, 1, "bf16", 2)[:, :, 0], query(2, 1, 8, "bf16", 3)
    ws = binding.cache8_workspace(c.cache, q, 224, accumulate=True)

    def step():
        binding.cache8_append(c.cache, k, v)
        out = binding.cache8_attention(c.cache, q, 224, accumulate=True, workspace=ws)
        return out, binding.cache8_evict(c.cache, into, 96, keep_first=4, keep_last=8, max_rows=224)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, idx = step()
    for i in range(3):
        for t, s in ((k, 10), (v, 20), (q, 30)):
            t.copy_(query(*(t.shape if t.dim() == 4 else (2, 2, 1, 128))[:3], "bf16", s + i).view_as(t))
        c.cache.rows.add_(1)
        c.lens += 1
        held = c.cache.pool.clone(), c.cache.mass.clone()
        graph.replay()
        got = out.clone(), idx.clone(), into.pool.clone(), c.cache.mass.clone()
        c.cache.pool.copy_(held[0]), c.cache.mass.copy_(held[1])
        want = step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[3], c.cache.mass)
        assert torch.equal(got[2].view(-1, plain.TILE_BYTES)[:, :4104], into.pool.view(-1, plain.TILE_BYTES)[:, :4104])
        check_attention(c, q, "bf16", 128 ** -0.5, 0, 0, got[0])


def test_what_the_binding_refuses():
    c = Cache([[40, 40]], 16)
    q = query(1, 1, 4, "bf16")
    x = torch.zeros((1, 2, 128), dtype=torch.bfloat16, device="cuda")
    cc = c.cache
    bad = lambda **kw: binding.Cache8(**{**cc.__dict__, **kw})
    for call in (
            lambda: binding.cache8_attention(bad(code="int4"), q), lambda: binding.cache8_attention(bad(page_rows=32), q),
            lambda: binding.cache8_attention(bad(mass=cc.mass[:-1]), q), lambda: binding.cache8_attention(bad(rows=cc.rows.long()), q),
            lambda: binding.cache8_attention(bad(table=cc.table[:, :1]), q), lambda: binding.cache8_attention(cc, q.float()),
            lambda: binding.cache8_attention(cc, q[..., :64]), lambda: binding.cache8_attention(cc, q[:, :, :3]),
            lambda: binding.cache8_attention(cc, q.cpu()), lambda: binding.cache8_append(cc, x, x.half()),
            lambda: binding.cache8_append(cc, x[:, :1], x[:, :1]), lambda: binding.cache8_append(cc, x[0], x[0]),
            lambda: binding.cache8_append(cc, x.repeat(2, 1, 1), x.repeat(2, 1, 1)), lambda: binding.cache8_read(cc, 1, compact=True),
            lambda: binding.cache8_evict(cc, cc, 16, budgets=cc.rows.float()), lambda: binding.cache8_append(cc, x, x, status=cc.mass)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: binding.cache8_attention(bad(mass=None), q, accumulate=True), lambda: binding.cache8_evict(cc, cc, 16),
                 lambda: binding.cache8_evict(bad(mass=None), bad(rows=cc.rows.clone()), 16), lambda: binding.cache8_attention(cc, q, window=-1),
                 lambda: binding.cache8_evict(cc, bad(rows=cc.rows.clone(), code="e4m3"), 16),
                 lambda: binding.cache8_evict(cc, bad(rows=cc.rows.clone()), 0),
                 lambda: binding.cache8_attention(cc, q, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(binding.MixKVError):
            call()
    with pytest.raises(TypeError):
        binding.cache8_read(cc, 1, torch.float32)


def test_what_changes_from_step_to_step_is_read_anew():
    # rows, tables, masses and rows of the pool are written by one kernel and read by the next, which is resident by then: in one loop
    # without a pause, with outputs in the memory of earlier ones, every step gives what it gives when nothing overlaps
    B, H, G, page, n = 3, 2, 4, 16, 60
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((n, B, H, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((n, B, 1, H * G, 128), generator=gen, device="cuda").bfloat16()

    def steps(wait):
        here, there = (binding.new_cache8(B, H, 64, page, mass=True) for _ in range(2))
        outs, rows = [], 0
        for i in range(n):
            rows += 1
            here.rows += 1
            binding.cache8_append(here, k[i], v[i])
            out = binding.cache8_attention(here, q[i], accumulate=True)
            kept = None
            if rows == 40:
                kept = binding.cache8_evict(here, there, 24, keep_first=1, keep_last=6)
                here, there, rows = there, here, 24
            if wait:
                torch.cuda.synchronize()
            outs.append((out, kept, here.mass.clone()))
            del out, kept
        torch.cuda.synchronize()
        return outs, here.rows.tolist()

    (slow, a), (fast, b) = steps(True), steps(False)
    assert a == b
    for (o, kept, m), (p, also, w) in zip(slow, fast):
        assert torch.equal(o, p) and torch.equal(m, w) and (kept is None) == (also is None) and (kept is None or torch.equal(kept, also))


@pytest.mark.parametrize("ties", [False, True])
def test_an_eviction_gives_the_same_every_time(ties):
    # clusters of eight, keys counted in any order
    c = Cache(np.full((1, 2), 40000), 64, "int8")
    c.fill()
    c.cache.mass.copy_(masses(c.cache.mass.shape, 9, ties))
    into = [binding.new_cache8(1, 2, 3000, 64, mass=True) for _ in range(2)]
    for x in into:
        x.pool.zero_()
    first = binding.cache8_evict(c.cache, into[0], 3000, keep_last=8)
    for _ in range(20):
        assert torch.equal(binding.cache8_evict(c.cache, into[1], 3000, keep_last=8), first)
    assert torch.equal(into[0].pool, into[1].pool) and torch.equal(into[0].mass, into[1].mass)


def test_the_example_runs():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "evicting_decode.py")
    spec = importlib.util.spec_from_file_location("evicting_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    error, outs, held, evictions = example.main(40)
    # eight bits with one scale for sixteen rows: rounding is a percent of a value's typical size
    assert error < 0.05 and evictions >= 2 and max(held) <= example.BUDGET + example.SLACK
    assert all(o.shape == (1, 1, 28, 128) and torch.isfinite(o.float()).all() for o in outs)
