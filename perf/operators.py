"""The paged 4-bit KV cache and what decoding does with it: the cases it is measured on, its plain form, and its
definition in 64 bits.

Kinds of case (``"op"``):
  append  new rows of K and V are rotated, rounded to 4 bits and written to their pages, then read back as
          a model's dense attention over the chunk reads them
  attend  attention of one token, or of the few tokens of a draft, over all rows of its sequence's pages
  sparse  the same over the pages that a bound on their scores selects

The cache.  A page holds ``page_rows`` rows of one KV head, in tiles of 16 rows (2304 bytes): the K codes, the V codes,
the K scales, the V scales.  A row's 128 values are eight blocks of 16, a value is code (4 bits: a sign and one of
0 .5 1 1.5 2 3 4 6) times its block's scale (8 bits, e4m3) times the call's ``k_scale`` or ``v_scale``.  Inside a tile the
bytes lie as a warp's matrix fragments take them (``_tiles``).  ``table`` [batch, heads, pages] says which page of the pool
holds a head's rows p * page_rows and on, ``rows`` [batch, heads] how many rows there are, the call's own included.
``bounds`` [pages, 2, 128] holds a page's elementwise minimum and maximum of the K values, without ``k_scale``.
"""
import math
import random

import torch

own = False

D = 128
TILE = 16
TILE_BYTES = 2304
K_SCALE, V_SCALE = 0.5, 0.25
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------------------------------------- cases
def listed():
    one = dict(op="attend", dtype="bf16", batch=1, H=4, G=7, T=1, page=64, lo=0, hi=0, heads="even")
    add = dict(op="append", dtype="bf16", batch=1, H=4, page=64, new_lo=1, new_hi=1, rope="halves", rot=128)
    top = dict(op="sparse", dtype="bf16", batch=1, H=8, G=4, T=1, page=64, heads="even", first=1, last=1)
    return [
        # the step of one answer that has just begun: what a launch and the host cost
        dict(add, name="append_step", lo=520, hi=520),
        # the step of a served batch, every sequence at another length
        dict(add, name="append_batch", batch=64, H=8, lo=300, hi=8000),
        # a long video's prompt, as the benchmark's default workload has it
        dict(add, name="append_prompt", lo=32768, hi=32768, new_lo=32768, new_hi=32768),
        # chunks of odd lengths behind odd numbers of rows, half of the dimensions rotated by neighbours
        dict(add, name="append_chunks", dtype="f16", batch=8, H=8, page=32, lo=2051, hi=7334, new_lo=517,
             new_hi=2049, rope="pairs", rot=64),
        # one sequence's step over a cache of the size the paper's budgets leave
        dict(one, name="attend_step", lo=512, hi=512),
        # one sequence of a text model with a long context, nothing thrown away
        dict(one, name="attend_long", H=8, G=4, lo=131072, hi=131072),
        # the step of a served batch, lengths spread widely: the largest call
        dict(one, name="attend_batch", batch=32, H=8, G=4, lo=1021, hi=16384),
        # compressed caches with head-adaptive budgets, 28 layers of a batch of eight in one call
        dict(one, name="attend_compact", batch=224, lo=70, hi=1639, heads="own", page=16),
        # a draft of five tokens checked at once
        dict(one, name="attend_draft", dtype="f16", batch=8, T=5, lo=2051, hi=7334),
        # a prompt of a few thousand tokens, an eighth of its pages read
        dict(top, name="sparse_short", H=4, G=7, lo=4096, hi=4096, top=8),
        # the long context, a sixteenth of its pages read
        dict(top, name="sparse_long", lo=131072, hi=131072, top=128),
        # a batch of long contexts of several lengths
        dict(top, name="sparse_batch", dtype="f16", batch=8, G=7, H=4, lo=16001, hi=65536, top=96, page=32),
    ]


MOST_ROWS = 32 * 8 * 8704   # rows of all heads of the largest listed call


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(("append", "attend", "attend", "sparse"))
    H = rng.choice((1, 2, 3, 4, 8))
    page = rng.choice((16, 32, 64, 64, 128))
    case = dict(op=op, dtype=rng.choice(("bf16", "bf16", "f16")), H=H, page=page)
    if op == "append":
        batch = _log(rng, 1, 64)
        most = max(1, min(32768, 32768 * 4 // (batch * H)))
        hi = 1 if rng.random() < 0.4 else _log(rng, 1, most)
        lo = rng.randint(1, hi)
        old = _log(rng, 1, 8000)
        rope = rng.choice(("halves", "halves", "pairs", "none"))
        return dict(case, batch=batch, lo=hi + old // 3, hi=hi + old, new_lo=lo, new_hi=hi, rope=rope,
                    rot=0 if rope == "none" else rng.choice((128, 128, 64, 32)))
    G = rng.choice((1, 2, 4, 4, 5, 7, 7, 8, 12, 16))
    T = rng.choice((1, 1, 1, 1, 2, 3, 4, 5, 8))
    batch = _log(rng, 1, 64)
    if op == "attend":
        hi = _log(rng, 64, min(131072, MOST_ROWS // (batch * H * T)))
        return dict(case, batch=batch, G=G, T=T, lo=rng.randint(max(T, hi // 8), hi), hi=hi,
                    heads=rng.choice(("even", "even", "own")))
    batch = min(batch, 16)
    hi = _log(rng, 1024, min(131072, MOST_ROWS // (batch * H * T)))
    pages = -(-hi // page)
    return dict(case, batch=batch, G=G, T=T, lo=rng.randint(max(T, hi // 8), hi), hi=hi, heads="even",
                top=max(2, min(512, int(pages * rng.uniform(0.03, 0.4)))), first=rng.choice((0, 1)), last=rng.choice((1, 2)))


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, in no order, hi among them."""
    return [lo + int(round((hi - lo) * (1 - (0.6180339887498949 * i) % 1))) for i in range(n)]


def _rows(case):
    """Rows of every (sequence, head), the call's own included."""
    B, H = case["batch"], case["H"]
    if case.get("heads") == "own":
        flat = _spread(B * H, case["lo"], case["hi"])
        return [flat[b * H:(b + 1) * H] for b in range(B)]
    return [[n] * H for n in _spread(B, case["lo"], case["hi"])]


def _new(case):
    return _spread(case["batch"], case["new_lo"], case["new_hi"])


# ------------------------------------------------------------------------------- the cache's plain form
def _magnitude(a):
    """Index of the nearest of 0 .5 1 1.5 2 3 4 6, ties to the even index."""
    return ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))


def _quantise(x, scale):
    """x [..., 128] fp32 -> codes [..., 128] and the scales' bytes [..., 8]."""
    b = x.unflatten(-1, (8, 16))
    s = (b.abs().amax(-1) * (1.0 / (6.0 * scale))).clamp(max=448.0).to(torch.float8_e4m3fn)
    d = s.float() * scale
    y = torch.where((d == 0).unsqueeze(-1), torch.zeros_like(b), b / d.unsqueeze(-1))
    codes = _magnitude(y.abs()) + torch.signbit(y).to(torch.uint8) * 8
    return codes.flatten(-2), s.view(torch.uint8)


def _values(codes, scales):
    """Values without the call's scale, fp32: codes [..., 128], bytes of the scales [..., 8]."""
    m = codes & 7
    v = torch.where(m < 2, m.float() * 0.5, torch.exp2((m >> 1).float() - 1.0) * (1.0 + (m & 1).float() * 0.5))
    v = torch.where(codes > 7, -v, v)
    return (v.unflatten(-1, (8, 16)) * scales.view(torch.float8_e4m3fn).float().unsqueeze(-1)).flatten(-2)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _tiles(kc, ks, vc, vs):
    """Tiles [n, 2304] of codes [n, 16, 128] and scale bytes [n, 16, 8].  Row 4a + 2j + b of a tile has its K codes at
    512 j + 64 (2a + b), those of dimensions 32t and on at 16 t from there, and its K scales 2t, 2t + 1 at
    2048 + 16 (2a + b) + 4 t + 2 j.  Row 4t + 2i + e has the V codes of block g at 1024 + 512 i + 64 g + 16 t + 8 e and that
    block's scale at 2176 + 16 g + 4 t + 2 i + e."""
    n = kc.shape[0]
    k = _pack(kc).view(n, 4, 2, 2, 64).transpose(1, 2)               # j, a, b
    v = _pack(vc).view(n, 4, 2, 2, 8, 8).permute(0, 2, 4, 1, 3, 5)       # i, g, t, e
    s = ks.view(n, 4, 2, 2, 4, 2).permute(0, 1, 3, 4, 2, 5)       # a, b, t, j
    return torch.cat([k.reshape(n, -1), v.reshape(n, -1), s.reshape(n, -1), vs.transpose(1, 2).reshape(n, -1)], 1)


def _untile(t):
    """The reverse of _tiles: codes and scale bytes of K, then of V."""
    n = t.shape[0]
    k = t[:, :1024].view(n, 2, 4, 2, 64).permute(0, 2, 1, 3, 4).reshape(n, 16, 64)
    v = t[:, 1024:2048].view(n, 2, 8, 4, 2, 8).permute(0, 3, 1, 4, 2, 5).reshape(n, 16, 64)
    s = t[:, 2048:2176].view(n, 4, 2, 4, 2, 2).permute(0, 1, 4, 2, 3, 5).reshape(n, 16, 8)
    return _unpack(k), s, _unpack(v), t[:, 2176:].view(n, 8, 16).transpose(1, 2).contiguous()


def _pages(pool, ids, page):
    """K and V values (without the calls' scales) of pages ids [...]: two fp32 [..., page, 128]."""
    t = pool[ids.reshape(-1).long()].view(-1, TILE_BYTES)
    kc, ks, vc, vs = _untile(t)
    shape = (*ids.shape, page, D)
    return _values(kc, ks).view(shape), _values(vc, vs).view(shape)


def _rotate(x, cos, sin, rope, rot):
    """x [tokens, heads, 128] fp32; cos, sin [tokens, 1, rot / 2]."""
    if rope == "none":
        return x
    if rope == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)


# ---------------------------------------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _filled(gen, tiles, offset, page):
    """`tiles` tiles of random rows; K has its head's offset [tiles, 128] and a few dimensions of large values."""
    got, loud = [], torch.ones(D, device="cuda")
    loud[5::29] = 4.0
    for at in range(0, tiles, 8192):
        n = min(8192, tiles - at)
        k = (_randn(gen, n, TILE, D) + offset[at:at + n].unsqueeze(1)) * loud
        got.append(_tiles(*_quantise(k, K_SCALE), *_quantise(_randn(gen, n, TILE, D), V_SCALE)))
    return torch.cat(got).view(tiles * TILE // page, page // TILE * TILE_BYTES)


def _state(case, gen, seed):
    """The pool, its table and the rows of a case, pages in no order."""
    B, H, page = case["batch"], case["H"], case["page"]
    rows = torch.tensor(_rows(case))
    count = (rows + page - 1) // page
    most, total = int(count.max()), int(count.sum())
    here = torch.arange(most).view(1, 1, most) < count.unsqueeze(-1)
    order = torch.randperm(total + 3, generator=torch.Generator().manual_seed(seed))
    table = torch.full((B, H, most), -1, dtype=torch.int32)
    table[here] = order[:total].int()
    head = torch.zeros(total + 3, dtype=torch.int64)
    head[order[:total]] = (torch.arange(B * H).view(B, H, 1).expand(B, H, most)[here])
    offset = _randn(gen, B * H, D) * 0.7
    tiles = head.cuda().repeat_interleave(page // TILE)
    pool = _filled(gen, (total + 3) * page // TILE, offset[tiles], page)
    table, rows = table.cuda(), rows.int().cuda()
    return {"pool": pool, "table": table, "rows": rows, "page": page, "bounds": None, "most": int(rows.max())}


def _bounds_of(s, held, chunk=4096):
    """Bounds of all pages; `held` [batch, heads]: rows that are counted."""
    page, table = s["page"], s["table"]
    n = s["pool"].shape[0]
    bounds = torch.zeros((n, 2, D), dtype=torch.float16, device="cuda")
    left = held.unsqueeze(-1) - torch.arange(table.shape[2], device="cuda") * page
    ids, left = table[left > 0], left[left > 0]
    for at in range(0, ids.numel(), chunk):
        k = _pages(s["pool"], ids[at:at + chunk], page)[0]
        out = (torch.arange(page, device="cuda") >= left[at:at + chunk].unsqueeze(1)).unsqueeze(-1)
        bounds[ids[at:at + chunk].long(), 0] = k.masked_fill(out, math.inf).amin(1).half()
        bounds[ids[at:at + chunk].long(), 1] = k.masked_fill(out, -math.inf).amax(1).half()
    return bounds


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _state(case, gen, seed)
    s.update(case=case, dtype=TYPES[case["dtype"]])
    B, H = case["batch"], case["H"]
    if case["op"] == "append":
        new = torch.tensor(_new(case))
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
        N = int(offsets[-1])
        s["bounds"] = _bounds_of(s, s["rows"] - new.cuda().unsqueeze(1))
        s["offsets"], s["max_new"], s["tokens"] = offsets.int().cuda(), int(new.max()), N
        # K and V lie side by side in the output of one projection, as a model has them
        qkv = _randn(gen, N, 2 * H + 2, D)
        qkv[:, :, 5::29] *= 4.0
        s["qkv"] = qkv.to(s["dtype"])
        s["k"], s["v"] = s["qkv"][:, 1:1 + H], s["qkv"][:, 2 + H:]
        # a token's position is its place in the sequence, which compression does not change
        seq = torch.repeat_interleave(torch.arange(B), new)
        at = torch.arange(N) - offsets[seq]
        first = s["rows"].cpu().long()[:, 0] - new
        s["positions"] = (at + first[seq]).int().cuda()
        s["seq"], s["at"] = seq.cuda(), at.cuda()
        s["cos"] = s["sin"] = None
        if case["rope"] != "none":
            half = case["rot"] // 2
            angle = torch.arange(int(s["positions"].max()) + 1).double().unsqueeze(1) * 10000.0 ** (
                -torch.arange(half).double() / half)
            s["cos"], s["sin"] = angle.cos().float().cuda(), angle.sin().float().cuda()
    else:
        s["q"] = (_randn(gen, B, case["T"], H * case["G"], D) * 1.5).to(s["dtype"])
        if case["op"] == "sparse":
            s["bounds"] = _bounds_of(s, s["rows"])
    if own:
        from paper_2510_20707_b200 import binding
        s["binding"] = binding
        s["pages"] = binding.Pages(pool=s["pool"], table=s["table"], rows=s["rows"], page_rows=s["page"],
                                   bounds=s["bounds"], k_scale=K_SCALE, v_scale=V_SCALE)
        if case["op"] != "append":   # a server keeps the workspace from step to step
            s["ws"] = binding.paged_workspace(s["pages"], s["q"], s["most"])
    return s


# -------------------------------------------------------------------------------------------- one pass
def _plain_append(s):
    case, page = s["case"], s["page"]
    H, per = case["H"], page // TILE
    k, v = s["k"].float(), s["v"].float()
    if case["rope"] != "none":
        p = s["positions"].long()
        k = _rotate(k, s["cos"][p].unsqueeze(1), s["sin"][p].unsqueeze(1), case["rope"], case["rot"])
    kc, ks = _quantise(k, K_SCALE)
    vc, vs = _quantise(v, V_SCALE)
    # where every (token, head) goes
    n = (s["offsets"][1:] - s["offsets"][:-1]).long()
    row = s["rows"].long()[s["seq"]] - n[s["seq"]].unsqueeze(1) + s["at"].unsqueeze(1)
    pid = s["table"].long()[s["seq"].unsqueeze(1), torch.arange(H, device="cuda"), row // page]
    tile, r = pid * per + row % page // TILE, row % TILE
    a, j, b = r // 4, r // 2 % 2, r % 2
    span = lambda m: torch.arange(m, device="cuda")
    at_k = 512 * j + 64 * (2 * a + b)
    at_v = 1024 + 512 * j + 16 * a + 8 * b
    at_ks = 2048 + 16 * (2 * a + b) + 2 * j
    at_vs = 2176 + r
    flat, base = s["pool"].view(-1), (tile * TILE_BYTES).unsqueeze(-1)
    flat[base + at_k.unsqueeze(-1) + span(64)] = _pack(kc)
    flat[base + at_v.unsqueeze(-1) + 64 * (span(64) // 8) + span(64) % 8] = _pack(vc)
    flat[base + at_ks.unsqueeze(-1) + 4 * (span(8) // 2) + span(8) % 2] = ks
    flat[base + at_vs.unsqueeze(-1) + 16 * span(8)] = vs
    # bounds of the pages that got rows: what was there before counts, unless the page begins here
    val = _values(kc, ks).half().reshape(-1, D)
    lo, hi = s["bounds"][:, 0], s["bounds"][:, 1]
    fresh = (row % page == 0).reshape(-1)
    begun = pid.reshape(-1)[fresh]
    lo[begun], hi[begun] = math.inf, -math.inf
    where = pid.reshape(-1, 1).expand(-1, D)
    lo.copy_(lo.float().scatter_reduce(0, where, val.float(), "amin").half())
    hi.copy_(hi.float().scatter_reduce(0, where, val.float(), "amax").half())
    # and back
    t = s["pool"].view(-1, TILE_BYTES)[tile.reshape(-1)]
    kc, ks, vc, vs = _untile(t)
    pick = torch.arange(t.shape[0], device="cuda"), r.reshape(-1)
    shape = (s["tokens"], H, D)
    return {"k": (_values(kc[pick], ks[pick]) * K_SCALE).to(s["dtype"]).view(shape),
            "v": (_values(vc[pick], vs[pick]) * V_SCALE).to(s["dtype"]).view(shape), "bounds": s["bounds"]}


def _softmax_rows(q, K, V, seen):
    """q [u, r, 128], K, V [u, rows, 128], seen [u, r, rows] -> [u, r, 128]; a row that sees nothing is zero."""
    logit = (q @ K.transpose(1, 2)) * (K_SCALE / math.sqrt(D))
    logit = logit.masked_fill(~seen, -math.inf)
    most = logit.amax(-1, keepdim=True)
    w = torch.exp(logit - torch.where(torch.isinf(most), torch.zeros_like(most), most))
    total = w.sum(-1, keepdim=True)
    return (w @ V) * V_SCALE / torch.where(total > 0, total, torch.ones_like(total))


def _queries(s):
    """q as [sequence and head, token and head of the group, 128], fp32."""
    c = s["case"]
    return (s["q"].float().view(c["batch"], c["T"], c["H"], c["G"], D).transpose(1, 2)
            .reshape(c["batch"] * c["H"], c["T"] * c["G"], D))


def _back(s, o):
    c = s["case"]
    return (o.view(c["batch"], c["H"], c["T"], c["G"], D).transpose(1, 2)
            .reshape(c["batch"], c["T"], c["H"] * c["G"], D).to(s["dtype"]))


def _attend(s, ids, first_row):
    """Attention over pages ids [u, n] whose rows begin at first_row [u, n] of their sequence (ids below 0: none)."""
    c, page = s["case"], s["page"]
    u = ids.shape[0]
    K, V = _pages(s["pool"], ids.clamp(min=0), page)
    row = (first_row.unsqueeze(-1) + torch.arange(page, device="cuda")).view(u, 1, -1)
    last = s["rows"].view(u, 1) - c["T"] + torch.arange(c["T"], device="cuda").repeat_interleave(c["G"])
    seen = (row <= last.unsqueeze(-1)) & (ids >= 0).repeat_interleave(page, 1).unsqueeze(1)
    gone = (row >= s["rows"].view(u, 1, 1)).view(u, -1, 1)      # nothing was ever written there
    K, V = (x.view(u, -1, D).masked_fill(gone, 0.0) for x in (K, V))
    return _back(s, _softmax_rows(_queries(s), K, V, seen))


def _pair(x):
    return x[..., 0::2] + x[..., 1::2]


def _plain_select(s):
    c, page = s["case"], s["page"]
    u, P, top = c["batch"] * c["H"], s["table"].shape[2], c["top"]
    ids = s["table"].view(u, P).clamp(min=0).long()
    lo, hi = s["bounds"][ids, 0].float().unsqueeze(1), s["bounds"][ids, 1].float().unsqueeze(1)
    q = _queries(s).unsqueeze(2)
    x = torch.maximum(q * lo, q * hi)                            # [u, rows, pages, 128]; the products are exact
    score = _pair(_pair(_pair(_pair(_pair(_pair(_pair(x))))))).squeeze(-1).amax(1)
    n = ((s["rows"].view(u, 1) + page - 1) // page)
    p = torch.arange(P, device="cuda")
    score = score.masked_fill((p < c["first"]) | (p >= n - c["last"]), math.inf).masked_fill(p >= n, -math.inf)
    order = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :top]
    count = n.clamp(max=top)
    taken = torch.arange(order.shape[1], device="cuda") < count
    picked = torch.sort(torch.where(taken, order, P), dim=1).values
    lists = torch.full((u, top), -1, dtype=torch.int32, device="cuda")
    lists[:, :order.shape[1]] = torch.where(picked < P, picked, -1).int()
    return lists.view(c["batch"], c["H"], top), count.int().view(c["batch"], c["H"])


def _plain_sparse(s):
    c = s["case"]
    lists, counts = _plain_select(s)
    flat = lists.view(-1, c["top"]).long()
    ids = torch.where(flat >= 0, s["table"].view(flat.shape[0], -1).long().gather(1, flat.clamp(min=0)), -1)
    return {"out": _attend(s, ids, flat.clamp(min=0) * s["page"]), "pages": lists, "counts": counts}


def _plain_attend(s):
    c = s["case"]
    u = c["batch"] * c["H"]
    ids = s["table"].view(u, -1).long()
    return _attend(s, ids, torch.arange(ids.shape[1], device="cuda").expand(u, -1) * s["page"])


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "sparse": _plain_sparse}[op](s)
    c, b = s["case"], s["binding"]
    if op == "append":
        b.paged_append(s["pages"], s["k"], s["v"], offsets=s["offsets"], max_new=s["max_new"], cos=s["cos"],
                       sin=s["sin"], positions=s["positions"], interleaved=c["rope"] == "pairs")
        k, v = b.paged_read(s["pages"], s["tokens"], s["dtype"], offsets=s["offsets"], max_new=s["max_new"])
        return {"k": k, "v": v, "bounds": s["bounds"]}
    if op == "attend":
        return b.paged_attention(s["pages"], s["q"], s["most"], workspace=s["ws"])
    out, lists, counts = b.paged_sparse_attention(s["pages"], s["q"], c["top"], s["most"], keep_first=c["first"],
                                                  keep_last=c["last"], workspace=s["ws"])
    return {"out": out, "pages": lists, "counts": counts}


# ---------------------------------------------------------------------------------------------- floors
def work(case):
    rows = [n for seq in _rows(case) for n in seq]
    row = TILE_BYTES // TILE
    if case["op"] == "append":
        new, H, page = _new(case), case["H"], case["page"]
        N = sum(new)
        pages = sum((r[0] - 1) // page - (r[0] - n) // page + 1 for r, n in zip(_rows(case), new)) * H
        rot = 0 if case["rope"] == "none" else case["rot"] * 4 + 4
        # inputs, table and rows; the 4-bit rows written; the dense rows handed back; the bounds
        return {"bytes": N * H * (512 + row + 512) + N * rot + pages * (2 * D * 2 + 4) + 8 * len(rows),
                "flops": N * H * 2.0 * (3 * D + 3 * case["rot"] / 2)}
    R = case["T"] * case["G"]
    io = len(rows) * R * D * 4
    if case["op"] == "attend":
        return {"bytes": sum(rows) * row + io + sum(-(-n // case["page"]) * 4 for n in rows), "flops": 4.0 * D * R * sum(rows)}
    pages = [-(-n // case["page"]) for n in rows]
    read = sum(min(n, case["top"] * case["page"]) for n in rows)
    return {"bytes": sum(pages) * (2 * D * 2 + 4) + read * row + io + len(rows) * (case["top"] + 1) * 4,
            "flops": 4.0 * D * R * read + 3.0 * D * R * sum(pages)}


# --------------------------------------------------------------------- the definition, in 64 bits
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_rows(pool, table, page, first, n):
    """Rows first .. first + n - 1 of one head, K and V without the calls' scales."""
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), dtype=torch.float64, device="cuda")
    r = torch.arange(first, first + n, device="cuda")
    tile, w = table[r // page].long() * (page // 16) + r % page // 16, r % 16
    bytes_ = pool.view(-1, TILE_BYTES)
    d = torch.arange(D, device="cuda")
    w_, t_ = w.unsqueeze(1), tile.unsqueeze(1)
    kb = bytes_[t_, (w_ // 2 % 2) * 512 + (w_ // 4 * 2 + w_ % 2) * 64 + d // 2]
    vb = bytes_[t_, 1024 + (w_ // 2 % 2) * 512 + d // 16 * 64 + w_ // 4 * 16 + w_ % 2 * 8 + d % 16 // 2]
    ks = bytes_[t_, 2048 + (w_ // 4 * 2 + w_ % 2) * 16 + d // 32 * 4 + (w_ // 2 % 2) * 2 + d // 16 % 2]
    vs = bytes_[t_, 2176 + d // 16 * 16 + w_]
    value = lambda b, s: grid[((b >> (4 * (d % 2)).to(torch.uint8)) & 15).long()] * s.contiguous().view(torch.float8_e4m3fn).double()
    return value(kb, ks), value(vb, vs)


def _exact_quantise(x, scale):
    b = x.view(*x.shape[:-1], 8, 16)
    s = (b.abs().amax(-1, keepdim=True) / (6 * scale)).clamp(max=448).float().to(torch.float8_e4m3fn).double() * scale
    grid = torch.tensor(_GRID, dtype=torch.float64, device="cuda")
    y = torch.where(s > 0, b / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(b))
    code = torch.zeros_like(y, dtype=torch.int64)
    for i in range(7):
        mid = (grid[i] + grid[i + 1]) / 2
        code += (y.abs() > mid) | ((y.abs() == mid) & (i % 2 == 1))
    return (grid[code] * y.sign() * s).view(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    B, H, page = case["batch"], case["H"], case["page"]
    if case["op"] == "append":
        k, v = s["k"].double(), s["v"].double()
        if case["rope"] != "none":
            m = case["rot"] // 2
            c, n = s["cos"][s["positions"].long()].double(), s["sin"][s["positions"].long()].double()
            z = torch.complex(c, n).unsqueeze(1)
            first, second = (slice(0, m), slice(m, 2 * m)) if case["rope"] == "halves" else (slice(0, 2 * m, 2), slice(1, 2 * m, 2))
            turned = torch.complex(k[..., first], k[..., second]) * z
            k = k.clone()
            k[..., first], k[..., second] = turned.real, turned.imag
        k, v = _exact_quantise(k, K_SCALE), _exact_quantise(v, V_SCALE)
        bounds, off = s["bounds"].double(), s["offsets"].tolist()
        for b in range(B):
            n, total = off[b + 1] - off[b], int(s["rows"][b, 0])
            for p in range((total - n) // page, (total - 1) // page + 1):
                lo, hi = max(p * page, total - n), min((p + 1) * page, total)
                part = k[off[b] + lo - total + n:off[b] + hi - total + n] / K_SCALE
                ids = s["table"][b, :, p].long()
                low, high = part.amin(0), part.amax(0)
                if lo > p * page:
                    low, high = torch.minimum(low, bounds[ids, 0]), torch.maximum(high, bounds[ids, 1])
                bounds[ids, 0], bounds[ids, 1] = low, high
        return {"k": k, "v": v, "bounds": bounds}
    T, G, HG = case["T"], case["G"], H * case["G"]
    out = torch.zeros((B, T, HG, D), dtype=torch.float64, device="cuda")
    lists = torch.full((B, H, case.get("top", 0)), -1, dtype=torch.int32, device="cuda")
    counts = torch.zeros((B, H), dtype=torch.int32, device="cuda")
    for b in range(B):
        for h in range(H):
            n = int(s["rows"][b, h])
            q = s["q"][b, :, h * G:(h + 1) * G].double()
            K, V = _exact_rows(s["pool"], s["table"][b, h], page, 0, n)
            row = torch.arange(n, device="cuda")
            if case["op"] == "sparse":
                have = -(-n // page)
                ids = s["table"][b, h, :have].long()
                lo, hi = s["bounds"][ids, 0].double(), s["bounds"][ids, 1].double()
                score = (q.clamp(min=0).reshape(-1, D) @ hi.T + q.clamp(max=0).reshape(-1, D) @ lo.T).amax(0)
                score[:case["first"]] = math.inf
                score[max(0, have - case["last"]):] = math.inf
                best = torch.sort(score, descending=True, stable=True).indices[:case["top"]].sort().values
                counts[b, h] = best.numel()
                lists[b, h, :best.numel()] = best.int()
                row = (best.unsqueeze(1) * page + torch.arange(page, device="cuda")).view(-1)
                row = row[row < n]
                K, V = K[row], V[row]
            logit = (q @ K.T) * (K_SCALE / math.sqrt(D))
            see = row.unsqueeze(0) <= (n - T + torch.arange(T, device="cuda")).unsqueeze(1)
            w = torch.softmax(logit.masked_fill(~see.unsqueeze(1), -math.inf), -1)
            out[b, :, h * G:(h + 1) * G] = torch.nan_to_num(w) @ V * V_SCALE
    return out if case["op"] == "attend" else {"out": out, "pages": lists, "counts": counts}
