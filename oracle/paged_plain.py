"""Plain definition of the paged 4-bit KV cache: its format, what appending rounds to, which pages a query selects, and
attention over it.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  numpy, without the library's code.  Rounding to codes is done in
fp32, operation by operation, as the format defines it; attention in fp64.
"""
from __future__ import annotations

import numpy as np

D, TILE, TILE_BYTES = 128, 16, 2304
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
CODE_VALUES = np.concatenate([GRID, -GRID])


def _e4m3_values():
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = np.nan if (b & 0x7F) == 0x7F else (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[b] = -x if b & 0x80 else x
    return v


E4M3 = _e4m3_values()
_POSITIVE = E4M3[:0x7F]      # 0 .. 448, ascending with the byte


def to_e4m3(x):
    """Bytes of non-negative fp32 numbers: nearest, ties to even, at most 448; NaN gives 0x7f."""
    x = np.asarray(x, np.float64)
    y = np.where(np.isnan(x), 0.0, np.minimum(x, 448.0))
    hi = np.clip(np.searchsorted(_POSITIVE, y), 1, 0x7E)
    lo = hi - 1
    dl, dh = y - _POSITIVE[lo], _POSITIVE[hi] - y
    b = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(x), 0x7F, b).astype(np.uint8)


def quantise(x, scale=1.0):
    """fp32 rows [..., 128] -> (codes [..., 128], scale bytes [..., 8])."""
    x = np.asarray(x, np.float32)
    b = x.reshape(*x.shape[:-1], 8, 16)
    with np.errstate(invalid="ignore", over="ignore"):
        s = to_e4m3(np.max(np.abs(b), -1) * np.float32(1.0 / (6.0 * float(np.float32(scale)))))
        d = (E4M3[s].astype(np.float32) * np.float32(scale))[..., None]
        y = np.where(d == 0, np.float32(0), b / np.where(d == 0, np.float32(1), d))
        a = np.where(np.isnan(y), 0, np.minimum(np.abs(y), np.float32(6))).astype(np.float64)
    hi = np.clip(np.searchsorted(GRID, a), 1, 7)
    lo = hi - 1
    dl, dh = a - GRID[lo], GRID[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = code + 8 * np.signbit(y)
    return code.reshape(x.shape).astype(np.uint8), s


def values(codes, scales):
    """fp64 values without the call's scale."""
    v = CODE_VALUES[codes].reshape(*codes.shape[:-1], 8, 16)
    return (v * E4M3[scales][..., None]).reshape(codes.shape)


def _places():
    """Byte and shift of every (row, dimension) of K and V codes in a tile, bytes of the scales."""
    r, d = np.arange(TILE)[:, None], np.arange(D)[None, :]
    a, j, b = r // 4, r // 2 % 2, r % 2
    g = np.arange(8)[None, :]
    return (512 * j + 64 * (2 * a + b) + d // 2, 1024 + 512 * j + 64 * (d // 16) + 16 * a + 8 * b + d % 16 // 2,
            2048 + 16 * (2 * a + b) + 4 * (g // 2) + 2 * j + g % 2, 2176 + 16 * g + r)


K_AT, V_AT, KS_AT, VS_AT = _places()


def row_mask(rows):
    """Bytes of a tile that its first / the given rows own (bool [2304])."""
    m = np.zeros(TILE_BYTES, bool)
    for at in (K_AT, V_AT, KS_AT, VS_AT):
        m[at[rows].reshape(-1)] = True
    return m


def put_row(tile, r, kc, ks, vc, vs):
    tile[K_AT[r, ::2]] = kc[0::2] | (kc[1::2] << 4)
    tile[V_AT[r, ::2]] = vc[0::2] | (vc[1::2] << 4)
    tile[KS_AT[r]], tile[VS_AT[r]] = ks, vs


def get_rows(pool, table_row, page_rows, n):
    """K and V values [n, 128] of the first n rows of a head, without the calls' scales."""
    r = np.arange(n)
    tiles = pool.reshape(-1, TILE_BYTES)
    t = table_row[r // page_rows].astype(np.int64) * (page_rows // TILE) + r % page_rows // TILE
    w, odd = r % TILE, (np.arange(D) % 2) * 4
    code = lambda at: (tiles[t[:, None], at[w]] >> odd) & 15
    return values(code(K_AT), tiles[t[:, None], KS_AT[w]]), values(code(V_AT), tiles[t[:, None], VS_AT[w]])


def rotate(x, cos, sin, interleaved):
    """fp32 rows [n, 128] by tables' rows cos, sin [n, rot / 2], every operation rounded by itself."""
    x = np.array(x, np.float32)
    m = cos.shape[1]
    i, j = (slice(0, 2 * m, 2), slice(1, 2 * m, 2)) if interleaved else (slice(0, m), slice(m, 2 * m))
    a, b = x[:, i].copy(), x[:, j].copy()
    x[:, i], x[:, j] = a * cos - b * sin, b * cos + a * sin
    return x


def attention(q, K, V, T, scale):
    """q [T, G, 128], K, V [n, 128] fp64 (the last T rows are the tokens') -> (out, sum of w |v|, largest sum |q k| scale)."""
    n = K.shape[0]
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    size = np.zeros(q.shape[:2])
    for t in range(T):
        m = max(0, n - T + 1 + t)
        if m == 0:
            continue
        s = q[t] @ K[:m].T * scale
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        out[t], mass[t] = w @ V[:m], w @ np.abs(V[:m])
        size[t] = (np.abs(q[t]) @ np.abs(K[:m]).T).max(1) * scale
    return out, mass, size


def scores(q, lo, hi):
    """q [rows, 128], lo, hi [pages, 128], all fp32 -> scores [pages], summed as the format defines it."""
    q, lo, hi = (np.asarray(x, np.float32) for x in (q, lo, hi))
    q = np.where(np.isinf(q), np.float32(np.nan), q)
    with np.errstate(invalid="ignore"):
        x = np.maximum(q[:, None] * lo[None], q[:, None] * hi[None])
        for _ in range(7):
            x = x[..., 0::2] + x[..., 1::2]
    return x[..., 0].max(0)


def select(score, top, first, last):
    """Columns of the pages that are listed, ascending."""
    n = len(score)
    forced = (np.arange(n) < first) | (np.arange(n) >= n - last)
    order = sorted(range(n), key=lambda p: (not forced[p], 0 if forced[p] else 0 if np.isnan(score[p]) else 1,
                                            0 if forced[p] or np.isnan(score[p]) else -float(score[p]), p))
    return sorted(order[:top])
