"""The paged 4-bit cache and the attention that reads it: cases to time, each operator in a plain form beside the
framework's own.

A cache page holds `page_rows` rows of every KV head: [KV head][page_rows / 16] tiles of 16 rows. A tile is, in this
order, the K codes (16 rows of D/2 bytes), the V codes, and for K and then V one 32-bit word per row and group of `group`
dimensions: bf16 scale in the low half, bf16 zero in the high half. Inside a row the codes lie in the order in which a
warp's matrix fragments take them: with W = D/8 words and u = group/32, word j (W/4) + g u + t of a K row holds the eight
dimensions from 8 (g group/8 + j u + t) on, low nibble first; 16-bit half i (D/32) + g u + t of a V row the four
dimensions from 4 (g group/4 + i u + t) on.

Quantisation of one group x, every step in IEEE single precision: zero = min(x) rounded down to bf16; scale =
(max(x) - zero) / 15 rounded up to bf16, 0 where that is below 2^-100; code = rint((x - zero) * (1 / scale)); the value a
code stands for is scale * code + zero. Where max(x) - zero is not finite the group is stored as NaN.
"""
import math

import torch

own = False

DEV = "cuda"
TILE = 16


# ------------------------------------------------------------------ cases

def listed():
    return [
        # one user, a short compressed context, one token of a 7B-shaped layer: latency
        dict(name="attn_one", op="attn", n=1, hq=32, hkv=32, d=128, group=64, page_rows=64, dtype="bf16", q_len=1, lo=385, hi=385),
        # a decode step of one 7B-shaped layer for 64 sequences of different lengths (prompt 2048 kept in part + generated rows)
        dict(name="attn_batch", op="attn", n=64, hq=32, hkv=32, d=128, group=64, page_rows=64, dtype="bf16", q_len=1, lo=64, hi=2176),
        # a decode step of one 70B-shaped grouped-query layer, prompts of 8192 at their early, long layers
        dict(name="attn_gqa", op="attn", n=16, hq=64, hkv=8, d=128, group=32, page_rows=128, dtype="bf16", q_len=1, lo=1000, hi=8704),
        # two very long contexts, grouped-query heads: few (sequence, head) pairs, so the rows have to be split
        dict(name="attn_far", op="attn", n=2, hq=64, hkv=8, d=128, group=128, page_rows=256, dtype="bf16", q_len=1, lo=100003, hi=131071),
        # the small fp32 model: four drafted tokens checked at once, small pages, an empty sequence among them
        dict(name="attn_draft_f32", op="attn", n=7, hq=4, hkv=4, d=64, group=32, page_rows=16, dtype="f32", q_len=4, lo=0, hi=272),
        # the new row of each of 64 sequences in one 7B-shaped layer, and read back
        dict(name="store_step", op="store", n=64, hkv=32, d=128, group=64, page_rows=64, dtype="bf16", src=1, rows=1, lists=0, ragged=False),
        # 13B-shaped prompts of 4096: the kept rows of each KV head go to pages, and are read back dense for the next chunk
        dict(name="store_prompt", op="store", n=8, hkv=40, d=128, group=64, page_rows=64, dtype="bf16", src=4096, rows=2005, lists=40, ragged=False),
        # the small fp32 model's prompts, sequences of different lengths, one kept set for all heads
        dict(name="store_f32", op="store", n=2, hkv=4, d=64, group=32, page_rows=16, dtype="f32", src=256, rows=144, lists=1, ragged=True),
        # sessions branched and the branch pruned in place, one kept set for all heads
        dict(name="branch_prune", op="branch", n=4, hkv=8, d=128, group=64, page_rows=64, rows_in=717, rows=301, lists=1, spare=64),
        # re-selection of a 7B-shaped layer's caches for 64 sequences, a kept set per KV head, into fresh pages
        dict(name="prune_batch", op="prune", n=64, hkv=32, d=128, group=64, page_rows=64, rows_in=2176, rows=1155, lists=32, spare=64),
        # a beam step: two prompts of four beams; losers dropped, winners forked, room for the next row made
        dict(name="beams_few", op="beams", n=8, hkv=32, d=128, group=64, page_rows=64, lo=500, hi=900, spare=300),
        # the same for 80 layers of 16 sequences in one call, grouped-query heads
        dict(name="beams_many", op="beams", n=1280, hkv=8, d=128, group=64, page_rows=64, lo=256, hi=640, spare=4000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "store", "store", "branch", "prune", "beams"])
    hkv, rep = rng.choice([(1, 5), (2, 3), (4, 1), (8, 8), (8, 4), (32, 1), (40, 1)])
    d = rng.choice([64, 128, 128, 128])
    group = rng.choice([g for g in (32, 64, 128) if g <= d])
    page_rows = rng.choice([16, 48, 64, 64, 128])
    case = dict(op=op, hkv=hkv, d=d, group=group, page_rows=page_rows)
    row_bytes = hkv * (d + 8 * (d // group))
    if op == "attn":
        hi = _log(rng, 1, 60000)
        q_len = rng.choice([1, 1, 1, 2, 5])
        n = min(_log(rng, 1, 96), max(1, 300_000_000 // (row_bytes * hi * -(-rep * q_len // 8))))
        case.update(n=n, hq=hkv * rep, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]) if hi * n * row_bytes * rep < 50_000_000 else "bf16",
                    q_len=q_len, lo=rng.randint(0, hi), hi=hi)
    elif op == "store":
        src = _log(rng, 1, 4096)
        rows = rng.randint(1, src)
        n = min(_log(rng, 1, 64), max(1, 60_000_000 // (row_bytes * src)))
        case.update(n=n, dtype=rng.choice(["bf16", "bf16", "f32"]), src=src, rows=rows, lists=rng.choice([0, 1, hkv]), ragged=rng.random() < 0.5)
        case["src"] = rows if case["lists"] == 0 else src
    elif op in ("branch", "prune"):
        rows_in = _log(rng, 2, 4096)
        n = min(_log(rng, 1, 64), max(1, 150_000_000 // (row_bytes * rows_in)))
        case.update(n=n, rows_in=rows_in, rows=rng.randint(1, rows_in), lists=rng.choice([1, hkv]), spare=rng.randint(0, 500))
    else:
        hi = _log(rng, 1, 700)
        n = min(_log(rng, 2, 1280), max(2, 150_000_000 // (hkv * (d + 8 * (d // group)) * max(hi, page_rows))))
        case.update(n=n, lo=rng.randint(1, hi), hi=hi, spare=rng.randint(0, 4000))
    return case


def _tile_bytes(c):
    return TILE * (c["d"] + 8 * (c["d"] // c["group"]))


def work(case):
    c = case
    row = c["hkv"] * (c["d"] + 8 * (c["d"] // c["group"]))
    if c["op"] == "attn":
        rows = sum(_lengths(c))
        eb = 2 if c["dtype"] == "bf16" else 4
        qo = c["n"] * c["q_len"] * c["hq"]
        return {"bytes": rows * row + qo * (2 * c["d"] * eb + 4), "flops": 4 * c["d"] * c["hq"] * c["q_len"] * rows}
    if c["op"] == "store":
        eb = 2 if c["dtype"] == "bf16" else 4
        rows = sum(_counts(c))
        dense = rows * c["hkv"] * 2 * c["d"] * eb
        return {"bytes": 2 * dense + 2 * rows * row + c["n"] * c["lists"] * c["rows"] * 4, "flops": 10 * rows * c["hkv"] * c["d"]}
    if c["op"] == "prune":
        return {"bytes": 2 * c["n"] * c["rows"] * row + c["n"] * c["lists"] * c["rows"] * 4, "flops": 0}
    if c["op"] == "branch":
        return {"bytes": 2 * c["n"] * (c["rows_in"] + c["rows"]) * row + c["n"] * c["lists"] * c["rows"] * 4 +
                4 * _pool_pages(c), "flops": 0}
    lens = _lengths(c)
    pages = sum(-(-x // c["page_rows"]) for x in lens)
    copied = sum(x % c["page_rows"] for x in lens)
    return {"bytes": 2 * copied * row + 4 * (_pool_pages(c) + 4 * pages), "flops": 0}


def _lengths(c):
    """Rows of each list, from lo to hi, spread by a fixed multiplicative walk (no two neighbours alike); the last is hi."""
    span = c["hi"] - c["lo"]
    return [c["lo"] + (span * ((i * 61803 + 29) % 100000)) // 100000 for i in range(c["n"] - 1)] + [c["hi"]]


def _counts(c):
    if not c["ragged"]:
        return [c["rows"]] * c["n"]
    return [(c["rows"] * ((i * 61803 + 29) % 100000)) // 100000 for i in range(c["n"] - 1)] + [c["rows"]]


def _ceil(a, b):
    return -(-a // b)


def _pool_pages(c):
    pr = c["page_rows"]
    if c["op"] == "attn":
        return sum(_ceil(x, pr) for x in _lengths(c)) + 3
    if c["op"] == "store":
        return c["n"] * _ceil(c["rows"], pr) + 3
    if c["op"] == "prune":
        return c["n"] * (_ceil(c["rows_in"], pr) + _ceil(c["rows"], pr)) + c["spare"]
    if c["op"] == "branch":
        return 2 * c["n"] * _ceil(c["rows_in"], pr) + c["spare"]
    return sum(_ceil(x, pr) for x in _lengths(c)) + c["n"] + c["spare"]


# ------------------------------------------------------------------ the format in plain operations

def _order(d, group, parts, width):
    """Dimension of each stored code: `parts` lanes own d / parts codes each, in runs of `width` dimensions."""
    u = group // 32
    i, g, t = torch.meshgrid(torch.arange(parts), torch.arange(d // group), torch.arange(u), indexing="ij")
    first = width * (g * (group // width) + i * u + t)
    return (first.reshape(-1, 1) + torch.arange(width)).reshape(-1)


def _orders(c):
    k = _order(c["d"], c["group"], 4, 8).to(DEV)
    v = _order(c["d"], c["group"], 8, 4).to(DEV)
    return {"k": k, "v": v, "k_inv": torch.argsort(k), "v_inv": torch.argsort(v)}


def _floor_bf16(x):
    b = x.view(torch.int32)
    low = b & 0xFFFF
    b = b - low + torch.where((x < 0) & (low != 0), 0x10000, 0).to(torch.int32)
    return b.view(torch.float32)


def _ceil_bf16(x):
    b = x.view(torch.int32)
    low = b & 0xFFFF
    return (b - low + torch.where(low != 0, 0x10000, 0).to(torch.int32)).view(torch.float32)


def _quantise(x, group, order):
    """[..., d] -> code bytes [..., d / 2] uint8 and (scale, zero) words [..., d / group] int32."""
    y = x.float().unflatten(-1, (-1, group))
    zero = _floor_bf16(y.amin(-1))
    span = y.amax(-1) - zero
    scale = _ceil_bf16(span / torch.full_like(span, 15.0))
    scale = torch.where(scale < 2.0 ** -100, 0.0, scale)
    inv = torch.where(scale > 0, torch.ones_like(scale) / scale, 0.0)
    code = torch.round((y - zero.unsqueeze(-1)) * inv.unsqueeze(-1))
    bad = ~torch.isfinite(span)
    code = torch.where(bad.unsqueeze(-1), 0.0, code).to(torch.uint8).flatten(-2)[..., order]
    sbits = torch.where(bad, 0x7FC0, (scale.view(torch.int32) >> 16) & 0xFFFF)
    zbits = torch.where(bad, 0x7FC0, (zero.view(torch.int32) >> 16) & 0xFFFF)
    return code[..., 0::2] | (code[..., 1::2] << 4), (sbits | (zbits << 16)).to(torch.int32)


def _dequantise(codes, words, group, inverse):
    """The values that codes stand for, [..., d] in fp32."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)[..., inverse]
    scale = ((words & 0xFFFF) << 16).view(torch.float32)
    zero = (words & -65536).view(torch.float32)
    return (c.float().unflatten(-1, (-1, group)) * scale.unsqueeze(-1) + zero.unsqueeze(-1)).flatten(-2)


def _fields(pool, c):
    """K codes, V codes, K words, V words as [page, head, tile, row, ...] views of the pool's bytes."""
    d, g = c["d"], c["d"] // c["group"]
    t = pool.view(pool.shape[0], c["hkv"], c["page_rows"] // TILE, _tile_bytes(c))
    half = TILE * d // 2
    kw, vw = t[..., 2 * half:2 * half + 64 * g], t[..., 2 * half + 64 * g:]
    return (t[..., :half].unflatten(-1, (TILE, d // 2)), t[..., half:2 * half].unflatten(-1, (TILE, d // 2)),
            kw.view(torch.int32).unflatten(-1, (TILE, g)), vw.view(torch.int32).unflatten(-1, (TILE, g)))


def _at(table, rows, hkv, page_rows):
    """Index of rows [n, r] (or [n, r, hkv]) of lists whose page tables are `table` [n, slots]: page, head, tile, row."""
    if rows.dim() == 2:
        rows = rows.unsqueeze(-1).expand(-1, -1, hkv)
    page = torch.gather(table, 1, (rows // page_rows).flatten(1).clamp_max(table.shape[1] - 1)).view_as(rows).long().clamp_min(0)
    return page, torch.arange(hkv, device=DEV), rows % page_rows // TILE, rows % TILE


def _plain_attn(s):
    c, table, lens = s["case"], s["table"], s["lens"].long()
    rows = torch.arange(max(c["hi"], 1), device=DEV).expand(c["n"], -1)
    at = _at(table, rows, c["hkv"], c["page_rows"])
    kc, vc, kw, vw = _fields(s["pool"], c)
    live = (rows < lens.unsqueeze(1)).view(c["n"], -1, 1, 1)
    k = torch.where(live, _dequantise(kc[at], kw[at], c["group"], s["order"]["k_inv"]), 0.0)
    n, t, hq, d = s["q"].shape
    q = s["q"].float().view(n, t, c["hkv"], -1, d).permute(0, 2, 1, 3, 4).flatten(2, 3)       # [n, hkv, t * rep, d]
    score = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(d)
    del k
    v = torch.where(live, _dequantise(vc[at], vw[at], c["group"], s["order"]["v_inv"]), 0.0)
    limit = lens.view(-1, 1) - (t - 1 - torch.arange(t, device=DEV))                            # rows that token t sees
    seen = rows.unsqueeze(1) < limit.unsqueeze(2)
    seen = seen.repeat_interleave(hq // c["hkv"], 1).unsqueeze(1)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    den = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v.transpose(1, 2)) / torch.where(den == 0, 1.0, den)
    lse = (top + torch.log(den)).squeeze(-1)
    out = out.view(n, c["hkv"], t, -1, d).permute(0, 2, 1, 3, 4).reshape(n, t, hq, d)
    return {"out": out.to(s["q"].dtype), "lse": lse.view(n, c["hkv"], t, -1).permute(0, 1, 3, 2).reshape(n, hq, t)}


def _plain_store(s):
    c = s["case"]
    k, v = s["k"], s["v"]
    if s["idx"] is not None:
        idx = s["idx"].long().transpose(1, 2)                                                   # [n, rows, lists]
        idx = idx.repeat_interleave(c["hkv"] // idx.shape[2], 2).unsqueeze(-1).expand(-1, -1, -1, c["d"])
        k, v = torch.gather(k, 1, idx), torch.gather(v, 1, idx)
    rows = torch.arange(c["rows"], device=DEV).expand(c["n"], -1)
    at = _at(s["table"], rows, c["hkv"], c["page_rows"])
    live = (rows < s["counts"].unsqueeze(1)).view(c["n"], -1, 1, 1)
    fields = _fields(s["pool"], c)
    order = s["order"]
    kq, vq = _quantise(k, c["group"], order["k"]), _quantise(v, c["group"], order["v"])
    fields[0][at] = torch.where(live, kq[0], fields[0][at])
    fields[1][at] = torch.where(live, vq[0], fields[1][at])
    fields[2][at] = torch.where(live, kq[1], fields[2][at])
    fields[3][at] = torch.where(live, vq[1], fields[3][at])
    s["lens"].copy_(torch.maximum(s["lens"], s["counts"]))
    ks, vs = s["k_out"], s["v_out"]
    ks.copy_(torch.where(live, _dequantise(fields[0][at], fields[2][at], c["group"], order["k_inv"]).to(ks.dtype), ks))
    vs.copy_(torch.where(live, _dequantise(fields[1][at], fields[3][at], c["group"], order["v_inv"]).to(vs.dtype), vs))
    return {"k": ks, "v": vs, "lens": s["lens"]}


def _plain_trim(s, lists):
    entry = s["table"][lists]
    held = entry >= 0
    s["refs"].index_add_(0, entry.clamp_min(0).flatten(), -held.flatten().to(torch.int32))
    s["table"][lists] = -1
    s["lens"][lists] = 0


def _plain_fork(s, src, dst):
    pr = s["case"]["page_rows"]
    lens = s["lens"][src]
    slot = torch.arange(s["table"].shape[1], device=DEV)
    held = slot < ((lens + pr - 1) // pr).unsqueeze(1)
    entry = torch.where(held, s["table"][src], -1)
    s["refs"].index_add_(0, entry.clamp_min(0).flatten(), held.flatten().to(torch.int32))
    s["table"][dst] = entry
    s["lens"][dst] = lens


def _plain_reserve(s, lists, rows):
    """Pages for `rows` more rows of each list, the lowest free page first, list by list and slot by slot; a part-filled last
    page that another list holds too is copied (its filled rows) to a page of the list's own."""
    c = s["case"]
    pr = c["page_rows"]
    lens = s["lens"][lists].long().unsqueeze(1)
    entry = s["table"][lists]
    slot = torch.arange(entry.shape[1], device=DEV)
    part = (slot == lens // pr) & (lens % pr != 0) & (entry >= 0)
    shared = part & (s["refs"][entry.clamp_min(0).long()] > 1)
    need = shared | ((slot * pr < lens + rows) & (entry < 0))
    free = torch.argsort((s["refs"] != 0).to(torch.int8), stable=True)
    rank = (torch.cumsum(need.flatten().long(), 0) - 1).view_as(entry)
    fresh = free[rank.clamp(0, free.numel() - 1)]
    new = torch.where(need, fresh.to(torch.int32), entry)
    tiles = s["pool"].view(s["pool"].shape[0], c["hkv"], pr // TILE, _tile_bytes(c))
    last = (lens // pr).clamp_max(entry.shape[1] - 1)
    old_page = torch.gather(entry, 1, last).squeeze(1).clamp_min(0).long()
    new_page = torch.gather(new, 1, last).squeeze(1).clamp_min(0).long()
    copies = torch.gather(shared, 1, last).view(-1, 1, 1, 1)
    filled = (lens % pr).view(-1, 1, 1, 1) > torch.arange(pr // TILE, device=DEV).view(1, 1, -1, 1) * TILE + s["byte_row"]
    # a list that copies nothing writes its own last page back as it is
    tiles[new_page] = torch.where(copies & filled, tiles[old_page], tiles[new_page])
    s["refs"].index_add_(0, new.clamp_min(0).flatten(), need.flatten().to(torch.int32))
    s["refs"].index_add_(0, entry.clamp_min(0).flatten(), -shared.flatten().to(torch.int32))
    s["table"][lists] = new


def _plain_compact(s, src, dst, idx, rows, in_place=False):
    c = s["case"]
    pr = c["page_rows"]
    to = torch.arange(rows, device=DEV).expand(c["n"], -1)
    fro = to if idx is None else idx.long().transpose(1, 2).repeat_interleave(c["hkv"] // idx.shape[1], 2)
    a, b = _at(s["table"][src], fro, c["hkv"], pr), _at(s["table"][dst], to, c["hkv"], pr)
    kc, vc, kw, vw = _fields(s["pool"], c)
    kc[b] = kc[a]
    vc[b] = vc[a]
    kw[b] = kw[a]
    vw[b] = vw[a]
    s["lens"][dst] = rows
    if in_place:
        entry = s["table"][dst]
        drop = (entry >= 0) & (torch.arange(entry.shape[1], device=DEV) >= -(-rows // pr))
        s["refs"].index_add_(0, entry.clamp_min(0).flatten(), -drop.flatten().to(torch.int32))
        s["table"][dst] = torch.where(drop, -1, entry)


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n, hkv, d, pr = c["n"], c["hkv"], c["d"], c["page_rows"]
    dtype = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    order = _orders(c)
    pages = _pool_pages(c)
    # pages lie in the pool in no order, as after hours of serving
    shuffled = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    pool = torch.zeros(pages, hkv * (pr // TILE) * _tile_bytes(c), dtype=torch.uint8, device=DEV)
    two = c["op"] in ("branch", "prune", "beams")
    n_lists = 2 * n if two else n
    if c["op"] in ("branch", "prune"):
        lens = [c["rows_in"]] * n
    elif c["op"] == "store":
        lens = [c["rows"]] * n
    else:
        lens = _lengths(c)
    slots = max(1, _ceil(max(lens) + (1 if c["op"] == "beams" else 0), pr))
    table = torch.full((n_lists, slots), -1, dtype=torch.int32, device=DEV)
    s = {"case": c, "pool": pool, "table": table, "order": order}
    used = 0
    fields = _fields(pool, c)
    centre_k = torch.randn(hkv, d, generator=g, device=DEV)        # keys have channels that stand off from zero
    for i, ln in enumerate(lens):
        held = _ceil(ln, pr)
        table[i, :held] = shuffled[used:used + held]
        used += held
        if c["op"] == "store" or ln == 0:
            continue
        k = torch.randn(ln, hkv, d, generator=g, device=DEV) + centre_k
        v = torch.randn(ln, hkv, d, generator=g, device=DEV)
        at = _at(table[i:i + 1], torch.arange(ln, device=DEV).unsqueeze(0), hkv, pr)
        at = tuple(x.squeeze(0) if x.dim() == 3 else x for x in at)
        kq, vq = _quantise(k.to(dtype), c["group"], order["k"]), _quantise(v.to(dtype), c["group"], order["v"])
        fields[0][at], fields[2][at] = kq
        fields[1][at], fields[3][at] = vq
    s["lens"] = torch.zeros(n_lists, dtype=torch.int32, device=DEV)
    if c["op"] == "attn":
        s["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        s["q"] = torch.randn(n, c["q_len"], c["hq"], d, generator=g, device=DEV).to(dtype)
    elif c["op"] == "store":
        s["k"] = (torch.randn(n, c["src"], hkv, d, generator=g, device=DEV) + centre_k).to(dtype)
        s["v"] = torch.randn(n, c["src"], hkv, d, generator=g, device=DEV).to(dtype)
        s["idx"] = None
        if c["lists"]:
            keys = torch.rand(n, c["lists"], c["src"], generator=g, device=DEV)
            s["idx"] = torch.sort(torch.topk(keys, c["rows"], dim=2).indices, dim=2).values.to(torch.int32).contiguous()
        s["counts"] = torch.tensor(_counts(c), dtype=torch.int32, device=DEV)
        s["first"] = torch.zeros(n, dtype=torch.int32, device=DEV)
        s["k_out"] = torch.zeros(n, c["rows"], hkv, d, dtype=dtype, device=DEV)
        s["v_out"] = torch.zeros_like(s["k_out"])
    else:
        s["lens"][:n] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["dst"] = torch.arange(n, 2 * n, dtype=torch.int32, device=DEV)
    if c["op"] in ("branch", "prune"):
        keys = torch.rand(n, c["lists"], c["rows_in"], generator=g, device=DEV)
        s["idx"] = torch.sort(torch.topk(keys, c["rows"], dim=2).indices, dim=2).values.to(torch.int32).contiguous()
        s["src"] = torch.arange(n, dtype=torch.int32, device=DEV)
    if c["op"] == "prune":
        held = _ceil(c["rows"], pr)
        table[n:, :held] = shuffled[used:used + n * held].view(n, held)
    if c["op"] == "beams":
        s["src"] = torch.randint(0, n, (n,), generator=g, device=DEV).to(torch.int32)
    if c["op"] in ("branch", "beams"):
        groups = d // c["group"]
        byte = torch.arange(_tile_bytes(c), device=DEV)
        half = TILE * d // 2
        s["byte_row"] = torch.where(byte < 2 * half, byte % half // (d // 2), (byte - 2 * half) % (64 * groups) // (4 * groups))
    held = table[table >= 0].long()
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV).index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    s["lists"] = torch.arange(n, dtype=torch.int32, device=DEV)
    if own:
        from paper_2405_12532_b200 import binding
        p = binding.PyrPages(n_kv_heads=hkv, head_dim=d, group=c["group"], page_rows=pr, n_pages=pages, n_lists=n_lists, max_pages=slots)
        for name in ("pool", "table", "lens", "refs"):
            view = getattr(p, name)
            view.copy_(s[name])
            s[name] = view
        s["pages"] = p
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    s = state
    c = s["case"]
    if own:
        p = s["pages"]
        if c["op"] == "attn":
            out, lse = p.attn(s["q"], s["lists"], lse=True)
            return {"out": out, "lse": lse}
        if c["op"] == "store":
            p.write(s["k"], s["v"], s["lists"], first=s["first"], idx=s["idx"], counts=s["counts"])
            p.read(s["k_out"], s["v_out"], s["lists"], first=s["first"], counts=s["counts"])
            return {"k": s["k_out"], "v": s["v_out"], "lens": p.lens}
        if c["op"] == "prune":
            p.compact(s["src"], s["dst"], idx=s["idx"])
        elif c["op"] == "branch":
            p.trim(s["dst"])
            p.reserve(s["dst"], c["rows_in"])
            p.compact(s["src"], s["dst"], n_rows=c["rows_in"])
            p.compact(s["dst"], s["dst"], idx=s["idx"])
        else:
            p.trim(s["dst"])
            p.fork(s["src"], s["dst"])
            p.reserve(s["dst"], 1)
        return {"pool": p.pool, "table": p.table, "lens": p.lens, "refs": p.refs}
    if c["op"] == "attn":
        return _plain_attn(s)
    if c["op"] == "store":
        return _plain_store(s)
    if c["op"] == "prune":
        _plain_compact(s, s["src"], s["dst"], s["idx"], c["rows"])
    elif c["op"] == "branch":
        _plain_trim(s, s["dst"])
        _plain_reserve(s, s["dst"], c["rows_in"])
        _plain_compact(s, s["src"], s["dst"], None, c["rows_in"])
        _plain_compact(s, s["dst"], s["dst"], s["idx"], c["rows"], in_place=True)
    else:
        _plain_trim(s, s["dst"])
        _plain_fork(s, s["src"], s["dst"])
        _plain_reserve(s, s["dst"], 1)
    return {"pool": s["pool"], "table": s["table"], "lens": s["lens"], "refs": s["refs"]}


# ------------------------------------------------------------------ in 64 bits

def _cell(tile, c, what, row, dim):
    """Code, scale and zero of one plane ("k" or "v") at rows and dimensions of tiles [..., tile bytes], in fp64."""
    d, group = c["d"], c["group"]
    u, g = group // 32, d // group
    which, within = dim // group, dim % group
    if what == "k":
        word, nib = within // 8, within % 8
        nibble = 8 * ((word // u) * (d // 32) + which * u + word % u) + nib
        base = 0
    else:
        half, nib = within // 4, within % 4
        nibble = 4 * ((half // u) * (d // 32) + which * u + half % u) + nib
        base = 8 * d
    byte = tile[..., base + row * (d // 2) + nibble // 2].to(torch.int64)
    code = torch.where(nibble % 2 == 0, byte % 16, byte // 16).to(torch.float64)
    word_at = 16 * d + (0 if what == "k" else 64 * g) + 4 * (row * g + which)

    def bf16(at):
        bits = tile[..., at].to(torch.int64) + 256 * tile[..., at + 1].to(torch.int64)
        return (torch.where(bits >= 32768, bits - 65536, bits) * 65536).to(torch.int32).view(torch.float32).to(torch.float64)

    return code * bf16(word_at) + bf16(word_at + 2)


def exact(case, seed):
    c = case
    if c["op"] in ("prune", "branch", "beams") or work(c)["bytes"] > 1_000_000_000:
        return None
    s = prepare(c, seed)
    d, hkv, pr = c["d"], c["hkv"], c["page_rows"]
    if c["op"] == "attn":
        row, dim = torch.meshgrid(torch.arange(TILE, device=DEV), torch.arange(d, device=DEV), indexing="ij")
        n, t, hq, _ = s["q"].shape
        out = torch.zeros(n, t, hq, d, dtype=torch.float64, device=DEV)
        lse = torch.full((n, hq, t), -math.inf, dtype=torch.float64, device=DEV)
        tiles = s["pool"].view(-1, hkv, pr // TILE, _tile_bytes(c))
        for i, ln in enumerate(_lengths(c)):
            if ln == 0:
                continue
            ids = s["table"][i, :_ceil(ln, pr)].long()
            for h in range(hkv):
                mine = tiles[ids, h].flatten(0, 1)
                k = _cell(mine, c, "k", row, dim).flatten(0, 1)[:ln]
                v = _cell(mine, c, "v", row, dim).flatten(0, 1)[:ln]
                rep = hq // hkv
                for tok in range(t):
                    see = ln - (t - 1 - tok)
                    if see <= 0:
                        continue
                    z = s["q"][i, tok, h * rep:(h + 1) * rep].double() @ k[:see].T / math.sqrt(d)
                    lse[i, h * rep:(h + 1) * rep, tok] = torch.logsumexp(z, -1)
                    out[i, tok, h * rep:(h + 1) * rep] = torch.softmax(z, -1) @ v[:see]
        return {"out": out, "lse": lse}
    # store: the codes by their definition (single precision), the values they stand for in 64 bits
    counts = _counts(c)
    res = []
    for name in ("k", "v"):
        got = torch.zeros(c["n"], c["rows"], hkv, d, dtype=torch.float64, device=DEV)
        for i in range(c["n"]):
            for h in range(hkv):
                x = s[name][i, :, h]
                if s["idx"] is not None:
                    x = x[s["idx"][i, h * c["lists"] // hkv].long()]
                x = x[:counts[i]].float().reshape(-1, c["group"])
                lo = x.min(1, keepdim=True).values
                near = lo.to(torch.bfloat16).float()
                zero = torch.where(near > lo, _next_bf16(near, -1), near)
                want = (x.max(1, keepdim=True).values - zero) / torch.tensor(15.0, device=DEV)
                near = want.to(torch.bfloat16).float()
                scale = torch.where(near < want, _next_bf16(near, 1), near)
                scale = torch.where(scale < 2.0 ** -100, torch.zeros_like(scale), scale)
                inverse = torch.where(scale == 0, torch.zeros_like(scale), scale.reciprocal())
                code = ((x - zero) * inverse).double().round()
                got[i, :counts[i], h] = (code * scale.double() + zero.double()).reshape(-1, d)
        res.append(got)
    return {"k": res[0], "v": res[1], "lens": None}


def _next_bf16(x, way):
    """The bf16 number after x in the direction `way`, for x held in single precision."""
    bits = (x.view(torch.int32) >> 16).to(torch.int64) & 0xFFFF
    key = torch.where(bits >= 0x8000, 0x8000 - bits, bits) + way
    back = torch.where(key < 0, 0x8000 - key, key)
    return torch.where(back >= 0x8000, back - 0x10000, back).mul(65536).to(torch.int32).view(torch.float32)
