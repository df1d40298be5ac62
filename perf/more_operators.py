"""The paged 8-bit KV cache that keeps count of attention: the cases it is measured on, its plain form, and its definition
in 64 bits.

Kinds of case (``"op"``):
  append  new rows of K and V are rounded to 8 bits and written to their pages, and the blocks they went to are read back
  attend  attention of one token, or of the few tokens of a draft, over its sequence's pages: over all rows, or over a
          sliding window and a few first rows; if asked, what every row got of the softmax's weight is added to its mass
  evict   of every head the rows of the largest mass, its first and its last rows are kept: written to other pages, and read back

The cache.  A page holds ``page`` rows of one KV head, in tiles of 16 rows (4112 bytes): the K codes, the V codes, an fp32 scale
for K and one for V.  A tile is a block: a value is code (8 bits, int8 or e4m3) times its block's scale.  Row r of a tile has
dimension d at byte 128 r + 16 ((d / 16) ^ (r % 8)) + d % 16.  ``table`` [batch, heads, pages] says which page of the pool
holds a head's rows p * page and on, ``rows`` [batch, heads] how many rows there are, the call's own included.  ``mass``
[pages, page] holds a row's accumulated weight.
"""
import math
import random

import torch

own = False

D = 128
TILE = 16
TILE_BYTES = 4112
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
LARGEST = {"int8": 127.0, "e4m3": 448.0}
SMALLEST = 2.0 ** -126    # a scale below is zero


# ------------------------------------------------------------------------------------------------- cases
def listed():
    add = dict(op="append", dtype="bf16", code="int8", batch=1, H=4, page=64, new_lo=1, new_hi=1)
    one = dict(op="attend", dtype="bf16", code="int8", batch=1, H=4, G=7, T=1, page=64, window=0, sinks=0, mass=False,
               heads="even")
    out = dict(op="evict", dtype="bf16", code="int8", batch=1, H=4, page=64, first=4, last=32, own=False)
    return [
        # the step of one answer that has just begun: what a launch and the host cost
        dict(add, name="append_step", lo=520, hi=520),
        # a long video's prompt, as the benchmark's default workload has it
        dict(add, name="append_prompt", lo=32768, hi=32768, new_lo=32768, new_hi=32768),
        # chunks of odd lengths behind odd numbers of rows
        dict(add, name="append_chunks", dtype="f16", code="e4m3", batch=8, H=8, page=32, lo=2051, hi=7334, new_lo=517,
             new_hi=2049),
        # one sequence's step over a cache of the size the paper's budgets leave, weights counted
        dict(one, name="attend_step", lo=512, hi=512, mass=True),
        # one sequence of a text model with a long context, nothing thrown away
        dict(one, name="attend_long", code="e4m3", H=8, G=4, lo=131072, hi=131072),
        # the step of a served batch, lengths spread widely, weights counted: the largest call
        dict(one, name="attend_batch", batch=32, H=8, G=4, lo=1021, hi=16384, mass=True),
        # a draft of five tokens checked at once
        dict(one, name="attend_draft", dtype="f16", batch=8, T=5, lo=2051, hi=7334),
        # a served batch that streams: the first four rows and the last 4096
        dict(one, name="attend_window", code="e4m3", batch=16, H=8, G=4, lo=4001, hi=65536, window=4096, sinks=4),
        # heads of unlike length, as adaptive budgets leave them, weights counted while a draft is checked
        dict(one, name="attend_own", dtype="f16", batch=64, T=2, page=16, lo=70, hi=1639, heads="own", mass=True),
        # one answer that has outgrown its budget by a few pages
        dict(out, name="evict_step", lo=640, hi=640, budget=512),
        # a batch of long prompts cut down to a budget
        dict(out, name="evict_batch", batch=16, H=8, lo=6001, hi=16384, budget=2048),
        # budgets of their own for the heads, a context too long for one block's shared memory
        dict(out, name="evict_long", dtype="f16", code="e4m3", H=8, page=128, lo=131072, hi=131072, budget=32768, own=True),
    ]


MOST_ROWS = 32 * 8 * 8704   # rows of all heads of the largest listed call


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(("append", "attend", "attend", "evict"))
    H = rng.choice((1, 2, 3, 4, 8))
    case = dict(op=op, dtype=rng.choice(("bf16", "bf16", "f16")), code=rng.choice(("int8", "e4m3")), H=H,
                page=rng.choice((16, 32, 64, 64, 128)), batch=_log(rng, 1, 64))
    if op == "append":
        most = max(1, min(32768, 32768 * 4 // (case["batch"] * H)))
        hi = 1 if rng.random() < 0.4 else _log(rng, 1, most)
        old = _log(rng, 1, 8000)
        return dict(case, lo=hi + old // 3, hi=hi + old, new_lo=rng.randint(1, hi), new_hi=hi)
    if op == "attend":
        T = rng.choice((1, 1, 1, 1, 2, 3, 4, 5, 8))
        hi = _log(rng, 64, min(131072, MOST_ROWS // (case["batch"] * H * T)))
        window = rng.choice((0, 0, _log(rng, 16, 8192)))
        return dict(case, G=rng.choice((1, 2, 4, 4, 5, 7, 7, 8, 12, 16)), T=T, lo=rng.randint(max(T, hi // 8), hi), hi=hi,
                    window=window, sinks=rng.choice((0, 1, 4, 64)) if window else 0, mass=rng.random() < 0.5,
                    heads=rng.choice(("even", "even", "own")))
    hi = _log(rng, 128, min(131072, MOST_ROWS // (2 * case["batch"] * H)))
    first, last = rng.choice((0, 1, 4)), rng.choice((0, 8, 32))
    return dict(case, lo=rng.randint(hi // 8, hi), hi=hi, first=first, last=last, own=rng.random() < 0.4,
                budget=max(first + last + 1, int(hi * rng.uniform(0.05, 0.7))))


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


def _budgets(case):
    """Budget of every (sequence, head)."""
    n = case["batch"] * case["H"]
    return _spread(n, max(case["first"] + case["last"], case["budget"] // 3), case["budget"]) if case["own"] else [case["budget"]] * n


# ------------------------------------------------------------------------------- the cache's plain form
def _at():
    """Byte of every (row, dimension) of a tile's K codes [16, 128]."""
    r, d = torch.arange(TILE, device="cuda").unsqueeze(1), torch.arange(D, device="cuda")
    return 128 * r + 16 * ((d // 16) ^ (r % 8)) + d % 16


def _as_codes(b, code):
    """Bytes as the numbers their codes stand for, fp32."""
    return b.view(torch.int8 if code == "int8" else torch.float8_e4m3fn).float()


def _scale_of(x, code):
    """Scale of blocks x [..., 16, 128] fp32 (rows that are not there: zeros): [...]."""
    s = x.abs().amax((-2, -1)) * (1.0 / LARGEST[code])
    return torch.where(s < SMALLEST, torch.zeros_like(s), s)


def _encode(x, scale, code):
    """Bytes of x [..., 16, 128] fp32 under the blocks' scales [...]."""
    by = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))[..., None, None]
    y = x * by
    if code == "int8":
        return y.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _split(tiles, code):
    """Codes of K and V [n, 16, 128] as fp32 numbers, and their scales [n]: of tiles [n, 4112]."""
    at, s = _at(), tiles[:, 4096:4104].contiguous().view(torch.float32)
    return (_as_codes(tiles[:, :2048][:, at], code), s[:, 0], _as_codes(tiles[:, 2048:4096][:, at], code), s[:, 1])


def _pack(kb, ks, vb, vs):
    """Tiles [n, 4112] of bytes [n, 16, 128] and scales [n]."""
    n = kb.shape[0]
    t = torch.zeros((n, TILE_BYTES), dtype=torch.uint8, device="cuda")
    at = _at().view(-1)
    t[:, at], t[:, 2048 + at] = kb.reshape(n, -1), vb.reshape(n, -1)
    t[:, 4096:4104] = torch.stack([ks, vs], 1).view(torch.uint8)
    return t


def _values(pool, tile, code):
    """K and V values [..., 16, 128] fp32 of tiles tile [...] of the pool."""
    kc, ks, vc, vs = _split(pool.view(-1, TILE_BYTES)[tile.reshape(-1)], code)
    shape = (*tile.shape, TILE, D)
    return (kc * ks[:, None, None]).view(shape), (vc * vs[:, None, None]).view(shape)


# ---------------------------------------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _filled(gen, tiles, offset, code):
    """`tiles` tiles of random rows; K has its head's offset [tiles, 128] and a few dimensions of large values."""
    got, loud = [], torch.ones(D, device="cuda")
    loud[5::29] = 4.0
    for at in range(0, tiles, 8192):
        n = min(8192, tiles - at)
        k, v = (_randn(gen, n, TILE, D) + offset[at:at + n].unsqueeze(1)) * loud, _randn(gen, n, TILE, D)
        ks, vs = _scale_of(k, code), _scale_of(v, code)
        got.append(_pack(_encode(k, ks, code), ks, _encode(v, vs, code), vs))
    return torch.cat(got)


def _table(rows, page, seed, spare=3):
    """Pages in no order for rows [batch, heads]: the table, and the head of every page."""
    count = (rows + page - 1) // page
    most, total = int(count.max()), int(count.sum())
    here = torch.arange(most).view(1, 1, most) < count.unsqueeze(-1)
    order = torch.randperm(total + spare, generator=torch.Generator().manual_seed(seed))
    table = torch.full((*rows.shape, most), -1, dtype=torch.int32)
    table[here] = order[:total].int()
    head = torch.zeros(total + spare, dtype=torch.int64)
    head[order[:total]] = torch.arange(rows.numel()).view(*rows.shape, 1).expand(*rows.shape, most)[here]
    return table.cuda(), head.cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, H, page, code = case["batch"], case["H"], case["page"], case["code"]
    rows = torch.tensor(_rows(case))
    table, head = _table(rows, page, seed)
    per = page // TILE
    pool = _filled(gen, head.numel() * per, (_randn(gen, B * H, D) * 0.7)[head.repeat_interleave(per)], code)
    s = {"case": case, "dtype": TYPES[case["dtype"]], "pool": pool.view(-1, per * TILE_BYTES), "table": table,
         "rows": rows.int().cuda(), "page": page, "code": code, "most": int(rows.max()), "mass": None}
    if case["op"] == "append":
        new = torch.tensor(_new(case))
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).int().cuda()
        s["max_new"], N = int(new.max()), int(new.sum())
        # K and V lie side by side in the output of one projection, as a model has them
        qkv = _randn(gen, N, 2 * H + 2, D)
        qkv[:, :, 5::29] *= 4.0
        s["qkv"] = qkv.to(s["dtype"])
        s["k"], s["v"] = s["qkv"][:, 1:1 + H], s["qkv"][:, 2 + H:]
        # what is read back: the new rows and those that share the first block with them
        back = new + (rows[:, 0] - new) % TILE
        s["back"] = torch.cat([torch.zeros(1, dtype=torch.int64), back.cumsum(0)]).int().cuda()
        s["max_back"], s["tokens"] = int(back.max()), int(back.sum())
    elif case["op"] == "attend":
        s["q"] = (_randn(gen, B, case["T"], H * case["G"], D) * 1.5).to(s["dtype"])
        if case["mass"]:
            s["mass"] = torch.rand((head.numel(), page), generator=gen, device="cuda")
    else:
        # a few rows carry most of the weight, and what has just come has none
        s["mass"] = torch.exp(2.0 * _randn(gen, head.numel(), page))
        s["mass"][torch.rand((head.numel(), page), generator=gen, device="cuda") < 0.1] = 0.0
        budget = torch.tensor(_budgets(case)).view(B, H)
        kept = torch.minimum(rows, budget)
        s["budgets"] = budget.int().cuda() if case["own"] else None
        s["into_table"], pages = _table(kept, page, seed + 1)
        s["into_pool"] = torch.zeros((pages.numel(), per * TILE_BYTES), dtype=torch.uint8, device="cuda")
        s["into_mass"] = torch.zeros((pages.numel(), page), device="cuda")
        s["into_rows"] = torch.zeros((B, H), dtype=torch.int32, device="cuda")
        s["back"] = torch.cat([torch.zeros(1, dtype=torch.int64), kept.view(-1).cumsum(0)]).int().cuda()
        s["max_back"], s["tokens"] = int(kept.max()), int(kept.sum())
    if own:
        from paper_2510_20707_b200 import binding
        s["binding"] = binding
        s["cache"] = binding.Cache8(pool=s["pool"], table=table, rows=s["rows"], page_rows=page, code=code, mass=s["mass"])
        if case["op"] == "attend":   # a server keeps the workspace from step to step
            s["ws"] = binding.cache8_workspace(s["cache"], s["q"], s["most"], window=case["window"], sinks=case["sinks"],
                                               accumulate=case["mass"])
        if case["op"] == "evict":
            s["into"] = binding.Cache8(pool=s["into_pool"], table=s["into_table"], rows=s["into_rows"], page_rows=page,
                                       code=code, mass=s["into_mass"])
    return s


# -------------------------------------------------------------------------------------------- one pass
def _runs(count):
    """For runs of count [n] things: which run each thing is of, and its place in it."""
    run = torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count)
    return run, torch.arange(run.numel(), device="cuda") - (count.cumsum(0) - count)[run]


def _read(pool, table, rows, back, page, code, dtype):
    """The last back[i + 1] - back[i] rows of every unit (offsets a unit), dense [tokens, 128]: K and V."""
    n = (back[1:] - back[:-1]).long()
    u, i = _runs(n)
    row = rows.view(-1).long()[u] - n[u] + i
    tile = table.view(n.numel(), -1).long()[u, row // page] * (page // TILE) + row % page // TILE
    k, v = _values(pool, tile, code)
    pick = torch.arange(tile.numel(), device="cuda"), row % TILE
    return k[pick].to(dtype), v[pick].to(dtype)


def _plain_append(s):
    c, page, code = s["case"], s["page"], s["code"]
    B, H, per = c["batch"], c["H"], page // TILE
    n = s["rows"].view(-1).long()
    new = (s["offsets"][1:] - s["offsets"][:-1]).long().repeat_interleave(H)
    first = n - new
    u, i = _runs((n - 1) // TILE - first // TILE + 1)        # the tiles that get rows
    t = first[u] // TILE + i
    tile = s["table"].view(B * H, -1).long()[u, t // per] * per + t % per
    row = t.unsqueeze(1) * TILE + torch.arange(TILE, device="cuda")
    fresh = (row >= first[u].unsqueeze(1)) & (row < n[u].unsqueeze(1))
    token = (s["offsets"].long()[u // H].unsqueeze(1) + row - first[u].unsqueeze(1)).clamp(0, s["k"].shape[0] - 1)
    begun = (t * TILE >= first[u])                           # blocks that had no rows
    flat = s["pool"].view(-1, TILE_BYTES)
    old = flat[tile]
    codes = _split(old, code)
    got = []
    for x, c0, s0 in ((s["k"], codes[0], codes[1]), (s["v"], codes[2], codes[3])):
        x = x[token, (u % H).unsqueeze(1)].float() * fresh.unsqueeze(-1)
        s0 = torch.where(begun, torch.zeros_like(s0), s0)
        c0 = torch.where(begun[:, None, None], torch.zeros_like(c0), c0)
        scale = torch.maximum(s0, _scale_of(x, code))
        x = torch.where(fresh.unsqueeze(-1), x, c0 * s0[:, None, None])
        got += [_encode(x, scale, code), scale]
    flat[tile] = _pack(*got)
    k, v = _read(s["pool"], s["table"], s["rows"], _per_head(s["back"], H), page, code, s["dtype"])
    return {"k": _by_token(k, s["back"], H), "v": _by_token(v, s["back"], H)}


def _per_head(offsets, H):
    n = (offsets[1:] - offsets[:-1]).long().repeat_interleave(H)
    return torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), n.cumsum(0)])


def _by_token(x, offsets, H):
    """Rows [units of a sequence's heads, one after the other] as [tokens, heads, 128]."""
    n = (offsets[1:] - offsets[:-1]).long()
    b, i = _runs(n)
    at = (offsets[:-1].long()[b] * H + i).unsqueeze(1) + torch.arange(H, device="cuda") * n[b].unsqueeze(1)
    return x[at]


def _queries(s):
    """q as [sequence and head, token and head of the group, 128], fp32."""
    c = s["case"]
    return (s["q"].float().view(c["batch"], c["T"], c["H"], c["G"], D).transpose(1, 2)
            .reshape(c["batch"] * c["H"], c["T"] * c["G"], D))


def _plain_attend(s):
    c, page, u = s["case"], s["page"], s["case"]["batch"] * s["case"]["H"]
    ids = s["table"].view(u, -1).long()
    per = page // TILE
    tile = (ids.clamp(min=0) * per).unsqueeze(-1) + torch.arange(per, device="cuda")
    K, V = _values(s["pool"], tile, s["code"])
    K, V = K.view(u, -1, D), V.view(u, -1, D)
    row = torch.arange(K.shape[1], device="cuda").view(1, 1, -1)
    at = (s["rows"].view(u, 1) - c["T"] + torch.arange(c["T"], device="cuda").repeat_interleave(c["G"])).unsqueeze(-1)
    seen = row <= at
    if c["window"]:
        seen &= (row < c["sinks"]) | (row > at - c["window"])
    logit = (_queries(s) @ K.transpose(1, 2)) * (1.0 / math.sqrt(D))
    logit = logit.masked_fill(~seen, -math.inf)
    most = logit.amax(-1, keepdim=True)
    w = torch.exp(logit - torch.where(torch.isinf(most), torch.zeros_like(most), most))
    total = w.sum(-1, keepdim=True)
    w = w / torch.where(total > 0, total, torch.ones_like(total))
    o = (w @ V).view(c["batch"], c["H"], c["T"], c["G"], D).transpose(1, 2)
    o = o.reshape(c["batch"], c["T"], c["H"] * c["G"], D).to(s["dtype"])
    if not c["mass"]:
        return o
    here = (row.view(1, -1) < s["rows"].view(u, 1)) & (ids >= 0).repeat_interleave(page, 1)
    place = (ids.clamp(min=0) * page).repeat_interleave(page, 1) + row.view(1, -1) % page
    s["mass"].view(-1)[place[here]] += w.sum(1)[here]
    return {"out": o, "mass": s["mass"]}


def _plain_evict(s):
    c, page, code = s["case"], s["page"], s["code"]
    u, per = c["batch"] * c["H"], page // TILE
    ids, n = s["table"].view(u, -1).long(), s["rows"].view(u, 1).long()
    budget = s["budgets"].view(u, 1).long() if c["own"] else torch.full((u, 1), c["budget"], device="cuda")
    row = torch.arange(ids.shape[1] * page, device="cuda").unsqueeze(0)
    key = s["mass"][ids.clamp(min=0)].view(u, -1)
    key = key.masked_fill((row < c["first"]) | (row >= n - c["last"]), math.inf).masked_fill(row >= n, -math.inf)
    kept = torch.minimum(n, budget)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :c["budget"]]
    place = torch.arange(c["budget"], device="cuda").unsqueeze(0)
    past = key.shape[1]
    if order.shape[1] < c["budget"]:
        order = torch.nn.functional.pad(order, (0, c["budget"] - order.shape[1]), value=past)
    picked = torch.sort(torch.where(place < kept, order, past), dim=1).values
    idx = torch.where(place < kept, picked, -1).int()
    # the kept rows, as blocks of sixteen
    blocks = -(-c["budget"] // TILE)
    src = torch.nn.functional.pad(idx, (0, blocks * TILE - c["budget"]), value=-1).long()
    there, at = src >= 0, src.clamp(min=0)
    page_of = ids.gather(1, at // page)
    flat = s["pool"].view(-1, TILE_BYTES)
    from_tile, r = page_of * per + at % page // TILE, at % TILE
    byte = (128 * r).unsqueeze(-1) + 16 * ((torch.arange(D, device="cuda") // 16) ^ (r % 8).unsqueeze(-1)) + torch.arange(D, device="cuda") % 16
    scales = flat[:, 4096:4104].contiguous().view(torch.float32)
    into_t = torch.arange(blocks, device="cuda").unsqueeze(0).expand(u, -1)
    live = into_t * TILE < kept
    into_page = s["into_table"].view(u, -1).long().gather(1, (into_t // per).clamp(max=s["into_table"].shape[2] - 1))
    got = []
    for i in range(2):
        x = _as_codes(flat[from_tile.unsqueeze(-1), 2048 * i + byte], code) * scales[from_tile, i].unsqueeze(-1)
        x = (x * there.unsqueeze(-1)).view(u, blocks, TILE, D)[live]
        scale = _scale_of(x, code)
        got += [_encode(x, scale, code), scale]
    s["into_pool"].view(-1, TILE_BYTES)[(into_page * per + into_t % per)[live]] = _pack(*got)
    j = torch.arange(src.shape[1], device="cuda").unsqueeze(0).expand(u, -1)
    to = s["into_table"].view(u, -1).long().gather(1, (j // page).clamp(max=s["into_table"].shape[2] - 1)) * page + j % page
    s["into_mass"].view(-1)[to[there]] = s["mass"].view(-1)[(page_of * page + at % page)[there]]
    s["into_rows"].copy_(kept.view(c["batch"], c["H"]))
    k, v = _read(s["into_pool"], s["into_table"], s["into_rows"], s["back"], page, code, s["dtype"])
    return {"kept": idx.view(c["batch"], c["H"], -1), "rows": s["into_rows"], "mass": s["into_mass"], "k": k, "v": v}


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[c["op"]](s)
    b = s["binding"]
    if c["op"] == "append":
        b.cache8_append(s["cache"], s["k"], s["v"], offsets=s["offsets"], max_new=s["max_new"])
        k, v = b.cache8_read(s["cache"], s["tokens"], s["dtype"], offsets=s["back"], max_new=s["max_back"])
        return {"k": k, "v": v}
    if c["op"] == "attend":
        out = b.cache8_attention(s["cache"], s["q"], s["most"], window=c["window"], sinks=c["sinks"], accumulate=c["mass"],
                                 workspace=s["ws"])
        return {"out": out, "mass": s["mass"]} if c["mass"] else out
    kept = b.cache8_evict(s["cache"], s["into"], c["budget"], budgets=s["budgets"], keep_first=c["first"],
                          keep_last=c["last"], max_rows=s["most"])
    k, v = b.cache8_read(s["into"], s["tokens"], s["dtype"], offsets=s["back"], max_new=s["max_back"], compact=True)
    return {"kept": kept, "rows": s["into_rows"], "mass": s["into_mass"], "k": k, "v": v}


# ---------------------------------------------------------------------------------------------- floors
def work(case):
    rows = [n for seq in _rows(case) for n in seq]
    row, H, page = TILE_BYTES / TILE, case["H"], case["page"]
    if case["op"] == "append":
        total = news = 0
        for r, n in zip(_rows(case), _new(case)):
            back = n + (r[0] - n) % TILE
            blocks = (r[0] - 1) // TILE - (r[0] - n) // TILE + 1
            # inputs; the block that was begun, read; blocks written; read for what is handed back; the dense rows
            total += H * (n * 512 + (TILE_BYTES if (r[0] - n) % TILE else 0) + blocks * TILE_BYTES + back * 512)
            news += n
        return {"bytes": total + 8 * len(rows), "flops": news * H * 2.0 * 3 * D}
    if case["op"] == "attend":
        R, T, w = case["T"] * case["G"], case["T"], case["window"]
        seen = [n if not w else min(n, case["sinks"]) + max(0, min(n, w + T - 1, n - case["sinks"])) for n in rows]
        per = row + (8 if case["mass"] else 0)
        return {"bytes": sum(seen) * per + len(rows) * R * D * 4 + sum(-(-n // page) * 4 for n in seen),
                "flops": 4.0 * D * R * sum(seen)}
    kept = sum(min(n, b) for n, b in zip(rows, _budgets(case)))
    # every row's mass; kept rows read and written, with their mass; the list; the dense rows handed back
    return {"bytes": sum(rows) * 4 + kept * (2 * row + 4 + 512) + len(rows) * case["budget"] * 4,
            "flops": kept * 2.0 * 4 * D + sum(rows)}


# --------------------------------------------------------------------- the definition, in 64 bits
_E4M3 = [((m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)]


def _exact_tile(pool, tile, code):
    """K and V [n, 16, 128] of tiles tile [n], each value from its byte."""
    b = pool.view(-1, TILE_BYTES)[tile]
    r, d = torch.meshgrid(torch.arange(TILE, device="cuda"), torch.arange(D, device="cuda"), indexing="ij")
    if code == "int8":
        number = torch.tensor([x - 256 if x > 127 else x for x in range(256)], dtype=torch.float64, device="cuda")
    else:
        number = torch.tensor(_E4M3 + [-x for x in _E4M3], dtype=torch.float64, device="cuda")
    scale = b[:, 4096:4104].contiguous().view(torch.float32).double()
    place = r * 128 + torch.bitwise_xor(torch.div(d, 16, rounding_mode="floor"), r % 8) * 16 + d % 16
    return tuple(number[b[:, 2048 * i:][:, place].long()] * scale[:, i].view(-1, 1, 1) for i in range(2))


def _exact_rows(pool, table, page, n, code):
    """Rows 0 .. n - 1 of one head, K and V."""
    t = torch.arange(-(-n // TILE), device="cuda")
    k, v = _exact_tile(pool, table[t * TILE // page].long() * (page // TILE) + t % (page // TILE), code)
    return k.reshape(-1, D)[:n], v.reshape(-1, D)[:n]


def _exact_round(x, scale, code):
    """x [n, 16, 128] to the codes of blocks of these scales [n], and back."""
    s = scale.view(-1, 1, 1)
    y = torch.where(s > 0, x / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(x))
    if code == "int8":
        return y.round().clamp(-127, 127) * s
    m = y.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(m.clamp(min=2.0 ** -6))).clamp(min=-6) - 3)
    return torch.round(m / step) * step * y.sign() * s


def _blocks(x):
    """Rows [n, 128] as blocks of sixteen, the last filled up with zeros."""
    return torch.nn.functional.pad(x, (0, 0, 0, -x.shape[0] % TILE)).view(-1, TILE, D)


def exact(case, seed):
    s = prepare(case, seed)
    B, H, page, code = case["batch"], case["H"], case["page"], case["code"]
    top = LARGEST[code]
    if case["op"] == "append":
        off, got = s["offsets"].tolist(), ([], [])
        for b in range(B):
            n, total = off[b + 1] - off[b], int(s["rows"][b, 0])
            held = total - n
            t = held // TILE
            for i, x in enumerate((s["k"], s["v"])):
                heads = []
                for h in range(H):
                    new = x[off[b]:off[b + 1], h].double()
                    had = held - t * TILE
                    old, s0 = new[:0], 0.0
                    if had:
                        tile = s["table"][b, h, held // page].long() * (page // TILE) + t % (page // TILE)
                        old = _exact_tile(s["pool"], tile.view(1), code)[i][0, :had]
                        s0 = float(s["pool"].view(-1, TILE_BYTES)[tile, 4096 + 4 * i:4100 + 4 * i].contiguous().view(torch.float32))
                    y = _blocks(torch.cat([old, new]))
                    fresh = _blocks(torch.cat([torch.zeros_like(old), new]))
                    scale = fresh.abs().amax((1, 2)) / top
                    scale[0] = max(float(scale[0]), s0)
                    heads.append(_exact_round(y, scale, code).view(-1, D)[:had + n])
                got[i].append(torch.stack(heads, 1))
        return {"k": torch.cat(got[0]), "v": torch.cat(got[1])}
    if case["op"] == "attend":
        T, G = case["T"], case["G"]
        out = torch.zeros((B, T, H * G, D), dtype=torch.float64, device="cuda")
        mass = s["mass"].double() if case["mass"] else None
        for b in range(B):
            for h in range(H):
                n = int(s["rows"][b, h])
                K, V = _exact_rows(s["pool"], s["table"][b, h], page, n, code)
                q = s["q"][b, :, h * G:(h + 1) * G].double()
                row = torch.arange(n, device="cuda").view(1, 1, n)
                p = torch.arange(n - T, n, device="cuda").view(T, 1, 1)
                see = row <= p
                if case["window"]:
                    see = see & ((row < case["sinks"]) | (p - row < case["window"]))
                w = torch.softmax(((q @ K.T) / math.sqrt(D)).masked_fill(~see, -math.inf), -1)
                w = torch.nan_to_num(w)
                out[b, :, h * G:(h + 1) * G] = w @ V
                if case["mass"]:
                    at = torch.arange(n, device="cuda")
                    mass[s["table"][b, h, at // page].long(), at % page] += w.sum((0, 1))
        return {"out": out, "mass": mass} if case["mass"] else out
    budgets = _budgets(case)
    kept = torch.full((B, H, case["budget"]), -1, dtype=torch.int32, device="cuda")
    rows, mass = torch.zeros((B, H), dtype=torch.int32, device="cuda"), s["into_mass"].double()
    ks, vs = [], []
    for b in range(B):
        for h in range(H):
            n = int(s["rows"][b, h])
            at = torch.arange(n, device="cuda")
            m = s["mass"][s["table"][b, h, at // page].long(), at % page].double()
            key = m.clone()
            key[:case["first"]] = math.inf
            key[max(0, n - case["last"]):] = math.inf
            pick = torch.sort(key, descending=True, stable=True).indices[:budgets[b * H + h]].sort().values
            k, v = _exact_rows(s["pool"], s["table"][b, h], page, n, code)
            for x, to in ((k, ks), (v, vs)):
                y = _blocks(x[pick])
                to.append(_exact_round(y, y.abs().amax((1, 2)) / top, code).view(-1, D)[:pick.numel()])
            kept[b, h, :pick.numel()] = pick.int()
            rows[b, h] = pick.numel()
            j = torch.arange(pick.numel(), device="cuda")
            mass[s["into_table"][b, h, j // page].long(), j % page] = m[pick]
    return {"kept": kept, "rows": rows, "mass": mass, "k": torch.cat(ks), "v": torch.cat(vs)}
