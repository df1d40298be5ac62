"""The paged 8-bit cache by its definition, in numpy (test infrastructure only): blocks of sixteen rows with one scale for K and one for
V, attention in 64 bits with a window and sinks, the rows that an eviction keeps."""
import numpy as np

from .paged_plain import E4M3, to_e4m3

ROWS, DIM, TILE_BYTES = 16, 128, 4112
CODES = {"int8": np.float32(127), "e4m3": np.float32(448)}
BY = {"int8": np.float32(1.0 / 127.0), "e4m3": np.float32(1.0 / 448.0)}
_r, _d = np.arange(ROWS)[:, None], np.arange(DIM)[None]
AT = 128 * _r + 16 * ((_d >> 4) ^ (_r & 7)) + (_d & 15)      # byte of (row, dimension) of K
NUMBERS = {"int8": np.arange(256).astype(np.uint8).view(np.int8).astype(np.float32),
           "e4m3": E4M3.astype(np.float32)}


def scale_of(x, code):
    """Scale of a block whose new rows are x (fp32)."""
    if not np.isfinite(x).all():
        return np.float32(np.nan)
    s = np.float32(np.abs(x).max(initial=0)) * BY[code]
    return np.float32(0) if s < np.float32(2.0 ** -126) else np.float32(s)


def encode(x, scale, code):
    """Bytes of fp32 values under a block's scale."""
    x = np.asarray(x, np.float32)
    if not scale > 0:
        return np.zeros(x.shape, np.uint8)
    y = x * (np.float32(1) / np.float32(scale))
    if code == "int8":
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    return to_e4m3(np.minimum(np.abs(y), np.float32(448))) | (np.signbit(y).astype(np.uint8) << 7)


def values(codes, scale, code):
    return NUMBERS[code][codes] * np.float32(scale)


def scales_at(tile):
    """The two scales of a tile, as a view that can be written."""
    return tile[4096:4104].view(np.float32)


def put(tile, i, lo, x, code, begun):
    """New rows lo .. of K (i = 0) or V (1) into a tile; begun: it has rows from before."""
    new = np.zeros((ROWS, DIM), np.float32)
    new[lo:lo + len(x)] = x
    old = tile[2048 * i + AT]
    was = scales_at(tile)[i] if begun else np.float32(0)
    scale = scale_of(new, code)
    scale = np.float32(np.nan) if np.isnan(was) or np.isnan(scale) else max(was, scale)
    codes = encode(new, scale, code)
    if begun:
        kept = old if scale == was else encode(values(old, was, code), scale, code)
        fresh = (np.arange(ROWS) >= lo) & (np.arange(ROWS) < lo + len(x))
        codes = np.where(fresh[:, None], codes, kept)
    tile[2048 * i + AT] = codes
    scales_at(tile)[i] = scale


def append(pool, table, page, held, k, v, code):
    """Rows k, v [n, 128] fp32 behind the `held` rows of one head; pool [pages, bytes] is written."""
    tiles, per = pool.reshape(-1, TILE_BYTES), page // ROWS
    at, n = held, held + len(k)
    while at < n:
        t, end = at // ROWS, min(n, (at // ROWS + 1) * ROWS)
        for i, x in enumerate((k, v)):
            put(tiles[int(table[t // per]) * per + t % per], i, at - t * ROWS, x[at - held:end - held], code, at > t * ROWS)
        at = end


def rows_of(pool, table, page, n, code):
    """Rows 0 .. n - 1 of a head: K, V [n, 128] fp32."""
    t = np.arange(-(-n // ROWS))
    tiles = pool.reshape(-1, TILE_BYTES)[table[t * ROWS // page].astype(np.int64) * (page // ROWS) + t % (page // ROWS)]
    out = []
    for i in range(2):
        s = tiles[:, 4096 + 4 * i:4100 + 4 * i].copy().view(np.float32)
        out.append((NUMBERS[code][tiles[:, 2048 * i + AT]] * s[:, :, None]).reshape(-1, DIM)[:n])
    return out


def seen(n, T, window=0, sinks=0):
    """[T, n]: rows that the tokens see."""
    row, p = np.arange(n)[None], (n - T + np.arange(T))[:, None]
    ok = row <= p
    return ok & ((row < sinks) | (row > p - window)) if window else ok


def attention(q, K, V, scale, window=0, sinks=0):
    """q [T, G, 128], K, V [n, 128] -> out [T, G, 128], weights [T, G, n], sums of weight times |value| [T, G, 128]; fp64."""
    q, K, V = (np.asarray(x, np.float64) for x in (q, K, V))
    ok = seen(len(K), len(q), window, sinks)[:, None]
    if not len(K):
        z = np.zeros(q.shape)
        return z, np.zeros((*q.shape[:2], 0)), z
    s = np.where(ok, q @ K.T * scale, -np.inf)
    m = s.max(-1, keepdims=True)
    w = np.where(ok, np.exp(s - np.where(np.isfinite(m), m, 0)), 0.0)
    z = w.sum(-1, keepdims=True)
    w = w / np.where(z > 0, z, 1)
    return w @ V, w, w @ np.abs(V)


def kept_rows(mass, budget, first, last):
    """Rows that an eviction keeps of a head with these masses: the first and the last, of the others the heaviest (NaN above all,
    ties to the lower row)."""
    n = len(mass)
    if n <= budget:
        return np.arange(n)
    key = np.where(np.isnan(mass), np.inf, np.asarray(mass, np.float64))
    rank = np.where(np.isnan(mass), 1, 0)
    middle = np.arange(first, n - last)
    order = sorted(middle, key=lambda i: (-rank[i], -key[i], i))[:budget - first - last]
    return np.concatenate([np.arange(first), np.sort(np.asarray(order, np.int64)), np.arange(n - last, n)]).astype(np.int64)
