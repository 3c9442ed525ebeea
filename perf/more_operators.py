"""The paged cache held in 8 bits: rows stored with their rotation, attention over all rows, and attention over the pages that a
cheap score selects for each query. Cases to time, each operator in a plain form beside the framework's own.

A page holds `page_rows` rows of every KV head. For each head it is a header of 2 D + 16 bytes, the smallest and the largest
code of each dimension (signed bytes), then the K scale and the V scale (fp32) and 8 bytes of nothing, and behind it
page_rows / 16 tiles of 16 rows. A tile is 16 D bytes of K codes, 16 D bytes of V codes, the two scales once more and 8 bytes of
nothing. A code lies as the byte code + 128. K: row r's 16-byte chunk x (dimensions 16 x ..) at r D + 16 (x xor 4 (r & 1)) for D =
128, 16 x for D = 64. V: with j = (r & 7) / 2, b = 2 (r & 1) + r / 8, e = D / 8 and w = d mod e, the byte at 4 D j + 4 e (d / e) +
16 ((w / 4) xor (j mod (e / 4))) + 4 (w mod 4) + b.

Storing, every step in IEEE single precision: the scale of (page, head), for K and for V, is s = max(s_old, amax / 127) with amax
the largest magnitude among the rows to be stored there and s_old the scale before if other rows of the list stay in that page, else 0;
amax / 127 below 2^-100 counts as 0, and an amax that is not finite makes s NaN. Codes are rint(x * (1 / s)); codes of rows that stay
become rint(code * (s_old / s)). A code stands for s * code. The header's extrema are those of the codes stored since the
page held no other rows.
"""
import math

import torch

own = False

DEV = "cuda"
TILE = 16


# ------------------------------------------------------------------ cases

def listed():
    return [
        # a decode step of a 7B-shaped layer: one new row for each of 64 sequences, its keys and queries rotated on the way
        dict(name="append_step", op="append", n=64, hq=32, hkv=32, d=128, page_rows=64, dtype="bf16", src=1, rows=1, lists=0, lo=64, hi=2176, ragged=False),
        # 13B-shaped prompts of 4096: the kept rows of each KV head, stored at their original positions' rotation, and read back
        dict(name="append_prompt", op="append", n=8, hq=0, hkv=40, d=128, page_rows=64, dtype="bf16", src=4096, rows=2005, lists=40, lo=0, hi=0, ragged=False),
        # a chunk of up to 512 prompt tokens behind contexts that end inside a page, grouped-query heads
        dict(name="append_chunk", op="append", n=4, hq=64, hkv=8, d=128, page_rows=128, dtype="bf16", src=512, rows=512, lists=0, lo=900, hi=5000, ragged=True),
        # the small fp32 model's prompts, sequences of different lengths, one kept set for all heads
        dict(name="append_f32", op="append", n=2, hq=0, hkv=4, d=64, page_rows=16, dtype="f32", src=256, rows=144, lists=1, lo=0, hi=40, ragged=True),
        # one user, a short compressed context, one token of a 7B-shaped layer: latency
        dict(name="attn_one", op="attn", n=1, hq=32, hkv=32, d=128, page_rows=64, dtype="bf16", q_len=1, lo=385, hi=385),
        # a decode step of one 7B-shaped layer for 64 sequences of different lengths
        dict(name="attn_batch", op="attn", n=64, hq=32, hkv=32, d=128, page_rows=64, dtype="bf16", q_len=1, lo=64, hi=2176),
        # a decode step of one 70B-shaped grouped-query layer, prompts of 8192 at their early, long layers
        dict(name="attn_gqa", op="attn", n=16, hq=64, hkv=8, d=128, page_rows=32, dtype="bf16", q_len=1, lo=1000, hi=8704),
        # two very long contexts, grouped-query heads: few (sequence, head) pairs, so the rows have to be split
        dict(name="attn_far", op="attn", n=2, hq=64, hkv=8, d=128, page_rows=128, dtype="bf16", q_len=1, lo=100003, hi=131071),
        # the small fp32 model: four drafted tokens checked at once, small pages, an empty sequence among them
        dict(name="attn_draft_f32", op="attn", n=7, hq=4, hkv=4, d=64, page_rows=16, dtype="f32", q_len=4, lo=0, hi=272),
        # one user behind a long context: 4096 of 32 100 rows read for the token
        dict(name="sparse_one", op="sparse", n=1, hq=64, hkv=8, d=128, page_rows=64, dtype="bf16", q_len=1, lo=32100, hi=32100, slots=64, first=1, last=2, append=False),
        # 32 sequences of different lengths, grouped-query heads, two tokens each: 2048 rows read for every token
        dict(name="sparse_batch", op="sparse", n=32, hq=64, hkv=8, d=128, page_rows=64, dtype="bf16", q_len=2, lo=4000, hi=32768, slots=32, first=1, last=1, append=False),
        # a whole decode step of one layer's attention: rows rotated and stored, pages selected, the selected ones attended
        dict(name="sparse_step", op="sparse", n=64, hq=32, hkv=32, d=128, page_rows=32, dtype="bf16", q_len=1, lo=64, hi=2176, slots=16, first=1, last=2, append=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "append", "append", "sparse", "sparse"])
    hkv, rep = rng.choice([(1, 5), (2, 3), (4, 1), (8, 8), (8, 4), (32, 1), (40, 1)])
    d = rng.choice([64, 128, 128, 128])
    page_rows = rng.choice([16, 32, 48, 64, 64, 128])
    case = dict(op=op, hq=hkv * rep, hkv=hkv, d=d, page_rows=page_rows)
    row_bytes = 2 * hkv * d
    small = lambda n, rows: n * rows * row_bytes * rep < 50_000_000  # noqa: E731
    if op == "attn":
        hi = _log(rng, 1, 60000)
        q_len = rng.choice([1, 1, 1, 2, 5])
        n = min(_log(rng, 1, 96), max(1, 300_000_000 // (row_bytes * hi * -(-rep * q_len // 8))))
        case.update(n=n, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]) if small(n, hi) else "bf16", q_len=q_len, lo=rng.randint(0, hi), hi=hi)
    elif op == "append":
        src = _log(rng, 1, 4096)
        rows = rng.randint(1, src)
        n = min(_log(rng, 1, 64), max(1, 50_000_000 // (row_bytes * src)))
        lists = rng.choice([0, 1, hkv])
        hi = _log(rng, 1, 1000)
        case.update(n=n, dtype=rng.choice(["bf16", "bf16", "f32"]), src=src if lists else rows, rows=rows, lists=lists, lo=rng.randint(0, hi), hi=hi,
                    ragged=rng.random() < 0.5)
        if lists or rng.random() < 0.3:
            case["hq"] = 0
    else:
        hi = _log(rng, 16, 60000)
        q_len = rng.choice([1, 1, 2, 3])
        n = min(_log(rng, 1, 64), max(1, 200_000_000 // (row_bytes * hi)))
        slots = _log(rng, 2, max(2, min(64, 3000 // page_rows)))
        first = rng.randint(0, 1)
        case.update(n=n, dtype=rng.choice(["bf16", "bf16", "f32"]) if small(n, hi) else "bf16", q_len=q_len, lo=rng.randint(0, hi), hi=hi, slots=slots, first=first,
                    last=rng.randint(0, slots - first), append=rng.random() < 0.3)
    return case


def work(case):
    c = case
    eb = 2 if c["dtype"] == "bf16" else 4
    row = 2 * c["hkv"] * c["d"]
    if c["op"] == "append":
        rows = sum(_counts(c))
        dense = rows * row * eb
        q = 2 * rows * c["hq"] * c["d"] * eb
        return {"bytes": 2 * dense + 2 * rows * row + q + 4 * rows * c["d"] + c["n"] * c["lists"] * c["rows"] * 8,
                "flops": rows * (13 * c["hkv"] + 3 * c["hq"]) * c["d"]}
    lens = _lengths(c)
    qo = c["n"] * c["q_len"] * c["hq"] * 2 * c["d"] * eb
    if c["op"] == "attn":
        return {"bytes": sum(lens) * row + 8 * c["hkv"] * sum(_ceil(x, c["page_rows"]) for x in lens) + qo + 4 * c["n"] * c["q_len"] * c["hq"],
                "flops": 4 * c["d"] * c["hq"] * c["q_len"] * sum(lens)}
    more = c["q_len"] if c["append"] else 0
    pages = [_ceil(x + more, c["page_rows"]) for x in lens]
    read = sum(min(p * c["page_rows"], c["slots"] * c["page_rows"], x + more) for p, x in zip(pages, lens))
    scored = sum(p for p in pages if p > c["slots"])
    stored = c["n"] * more * row * (eb + 1)
    return {"bytes": scored * c["hkv"] * (2 * c["d"] + 4) + c["q_len"] * (read * row + 4 * c["n"] * c["hkv"] * c["slots"]) + qo + stored,
            "flops": c["q_len"] * c["hq"] * c["d"] * (4 * read + 4 * scored)}


def _lengths(c):
    """Rows that each list holds before the pass, from lo to hi, spread by a fixed multiplicative walk; the last is hi."""
    span = c["hi"] - c["lo"]
    return [c["lo"] + (span * ((i * 61803 + 29) % 100000)) // 100000 for i in range(c["n"] - 1)] + [c["hi"]]


def _counts(c):
    if not c["ragged"]:
        return [c["rows"]] * c["n"]
    return [(c["rows"] * ((i * 61803 + 29) % 100000)) // 100000 for i in range(c["n"] - 1)] + [c["rows"]]


def _ceil(a, b):
    return -(-a // b)


def _new_rows(c):
    return c["rows"] if c["op"] == "append" else (c["q_len"] if c.get("append") else 0)


# ------------------------------------------------------------------ the format in plain operations

def _places(d):
    """Byte of a tile at which the code of (row, dimension) lies, for K and for V: [16, d]."""
    r, x = torch.meshgrid(torch.arange(TILE), torch.arange(d), indexing="ij")
    k = r * d + 16 * ((x // 16) ^ (4 * (r & 1) if d == 128 else 0)) + x % 16
    e = d // 8
    j, b, w = (r & 7) // 2, 2 * (r & 1) + r // 8, x % e
    v = 16 * d + 4 * d * j + 4 * e * (x // e) + 16 * ((w // 4) ^ (j % (e // 4))) + 4 * (w % 4) + b
    return {"k": k.to(DEV), "v": v.to(DEV)}


def _head_bytes(c):
    return 2 * c["d"] + 16 + c["page_rows"] // TILE * (32 * c["d"] + 16)


def _split(pool, c):
    """Headers [page, head, 2 D + 16] and tiles [page, head, tile, bytes] as views of the pool's bytes."""
    heads = pool.view(pool.shape[0], c["hkv"], _head_bytes(c))
    at = 2 * c["d"] + 16
    return heads[..., :at], heads[..., at:].unflatten(-1, (c["page_rows"] // TILE, 32 * c["d"] + 16))


def _codes(tiles, place):
    """[..., tile, bytes] -> codes [..., rows, D] in fp32."""
    return (tiles[..., place].to(torch.float32) - 128.0).flatten(-3, -2)


def _scales(header, d):
    return header[..., 2 * d:2 * d + 8].contiguous().view(torch.float32)


def _page_of(table, slot):
    """Page ids of slots [n, ...] of the lists whose tables are `table` [n, slots]."""
    return torch.gather(table, 1, slot.flatten(1).clamp(0, table.shape[1] - 1)).view_as(slot).long().clamp_min(0)


def _rotate(x, cs):
    half = x.shape[-1] // 2
    c, s, a, b = cs[..., :half], cs[..., half:], x[..., :half], x[..., half:]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def _store(header, tiles, place, d, x, new, kept, at):
    """One plane ("k": at = 0, "v": at = 1) of pages whose bytes are `header` and `tiles` [..., heads, ...]: rows x [..., heads, rows, D]
    stored where `new`, those of `kept` brought to the new scale. Changes the bytes; returns the codes' extrema over the new rows
    and the kept extrema's factor."""
    new, kept, held = new.unsqueeze(-2).unsqueeze(-1), kept.unsqueeze(-2).unsqueeze(-1), kept.any(-1).unsqueeze(-1)
    top = torch.where(new, x.abs(), 0.0).amax((-2, -1))
    before = torch.where(held, _scales(header, d)[..., at], 0.0)
    scale = top / torch.full_like(top, 127.0)
    scale = torch.maximum(before, torch.where(scale < 2.0 ** -100, 0.0, scale))
    scale = torch.where(torch.isfinite(top), scale, math.nan)
    factor = torch.where(scale > 0, before / scale, 0.0)
    inverse = torch.where(scale > 0, torch.ones_like(scale) / scale, 0.0)
    old = torch.round(_codes(tiles, place) * factor[..., None, None])
    code = torch.where(new, torch.round(x * inverse[..., None, None]), torch.where(kept, old, 0.0))
    code = torch.where(torch.isnan(scale)[..., None, None], 0.0, code)
    tiles[..., place] = (code + 128.0).to(torch.uint8).unflatten(-2, (-1, TILE))
    tail = scale.unsqueeze(-1).contiguous().view(torch.uint8)
    header[..., 2 * d + 4 * at:2 * d + 4 * at + 4] = tail
    tiles[..., 32 * d + 4 * at:32 * d + 4 * at + 4] = tail.unsqueeze(-2)
    return torch.where(new, code, 127.0).amin(-2), torch.where(new, code, -127.0).amax(-2), factor, held


def _plain_append(s):
    c, d, pr = s["case"], s["case"]["d"], s["case"]["page_rows"]
    k, v, n, rows = s["k"].float(), s["v"].float(), s["case"]["n"], _new_rows(s["case"])
    if s["idx"] is not None:
        idx = s["idx"].long().transpose(1, 2)
        idx = idx.repeat_interleave(c["hkv"] // idx.shape[2], 2).unsqueeze(-1).expand(-1, -1, -1, d)
        k, v = torch.gather(k, 1, idx), torch.gather(v, 1, idx)
    angle = s["rope"][s["pos"].long()].transpose(1, 2)                                  # [n, rows, lists, d]
    k = _rotate(k, angle.repeat_interleave(c["hkv"] // angle.shape[2], 2))
    start, count, lens = s["at"].long().view(-1, 1, 1), s["counts"].long().view(-1, 1, 1), s["lens"].long().view(-1, 1, 1)
    slot = s["at"].long().view(-1, 1) // pr + torch.arange((rows + pr - 2) // pr + 1, device=DEV)
    row = slot.unsqueeze(-1) * pr + torch.arange(pr, device=DEV)                        # [n, slots, rows of a page]
    x = row - start
    new = (x >= 0) & (x < count)
    kept = (row < lens) & ~new
    page = torch.where(new.any(-1), _page_of(s["table"], slot), s["pool"].shape[0] - 1)  # (the pool's last page is in no table)
    x = x.clamp(0, rows - 1).flatten(1)
    pick = lambda t: t[torch.arange(n, device=DEV).view(-1, 1), x].unflatten(1, (-1, pr)).transpose(2, 3)  # noqa: E731
    headers, all_tiles = _split(s["pool"], c)
    header, tiles = headers[page], all_tiles[page]                                      # [n, slots, heads, ...]
    mn, mx, factor, held = _store(header, tiles, s["place"]["k"], d, pick(k), new, kept, 0)
    _store(header, tiles, s["place"]["v"], d, pick(v), new, kept, 1)
    old = torch.round(header[..., :2 * d].contiguous().view(torch.int8).float() * factor.unsqueeze(-1))
    held = held.unsqueeze(-1)
    mn = torch.where(held, torch.minimum(mn, old[..., :d]), mn)
    mx = torch.where(held, torch.maximum(mx, old[..., d:]), mx)
    header[..., :2 * d] = torch.cat((mn, mx), -1).to(torch.int8).view(torch.uint8)
    headers[page] = header
    all_tiles[page] = tiles
    s["lens"].copy_(torch.maximum(s["lens"], s["at"] + s["counts"]))
    if s["q"] is None:
        return None
    live = (torch.arange(rows, device=DEV) < s["counts"].view(-1, 1)).view(n, -1, 1, 1)     # (queries of rows that are not stored pass as they are)
    return torch.where(live, _rotate(s["q"].float(), angle).to(s["q"].dtype), s["q"])


def _plain_read(s):
    c, pr = s["case"], s["case"]["page_rows"]
    x = torch.arange(c["rows"], device=DEV)
    row = s["at"].long().view(-1, 1) + x
    page = _page_of(s["table"], row // pr).unsqueeze(-1)
    live = (x < s["counts"].view(-1, 1)).view(c["n"], -1, 1, 1)
    head, tile, within = torch.arange(c["hkv"], device=DEV), (row % pr // TILE).unsqueeze(-1), (row % TILE)
    headers, tiles = _split(s["pool"], c)
    mine = tiles[page, head, tile]                                                       # [n, rows, heads, bytes]
    scale = _scales(headers[page, head], c["d"])
    for_row = lambda name: torch.gather(mine, 3, s["place"][name][within].unsqueeze(2).expand(-1, -1, c["hkv"], -1)).float() - 128.0  # noqa: E731
    ko, vo = s["k_out"], s["v_out"]
    ko.copy_(torch.where(live, (for_row("k") * scale[..., :1]).to(ko.dtype), ko))
    vo.copy_(torch.where(live, (for_row("v") * scale[..., 1:]).to(vo.dtype), vo))
    return ko, vo


def _attend(score, seen, v):
    """softmax over the last dimension where `seen`, times v: outputs and the log of the denominators; zeros where nothing is seen."""
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    den = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(den == 0, 1.0, den), (top + torch.log(den)).squeeze(-1)


def _plain_attn(s):
    c, pr = s["case"], s["case"]["page_rows"]
    n, t, hq, d = s["q"].shape
    lens = s["lens"].long()
    slot = torch.arange(s["table"].shape[1], device=DEV).expand(n, -1)
    row = torch.arange(slot.shape[1] * pr, device=DEV)
    headers, tiles = _split(s["pool"], c)
    page = _page_of(s["table"], slot)
    scale = _scales(headers[page], d).transpose(1, 2).repeat_interleave(pr, 2)           # [n, heads, rows, 2]
    live = (row < lens.view(-1, 1)).view(n, 1, -1, 1)
    mine = tiles[page]
    values = lambda name, at: torch.where(live, _codes(mine, s["place"][name]).transpose(1, 2).flatten(2, 3) * scale[..., at:at + 1], 0.0)  # noqa: E731
    q = s["q"].float().view(n, t, c["hkv"], -1, d).permute(0, 2, 1, 3, 4).flatten(2, 3)       # [n, hkv, t * rep, d]
    score = torch.matmul(q, values("k", 0).transpose(2, 3)) / math.sqrt(d)
    limit = lens.view(-1, 1) - (t - 1 - torch.arange(t, device=DEV))                            # rows that token t sees
    seen = (row < limit.unsqueeze(2)).repeat_interleave(hq // c["hkv"], 1).unsqueeze(1)
    out, lse = _attend(score, seen, values("v", 1))
    out = out.view(n, c["hkv"], t, -1, d).permute(0, 2, 1, 3, 4).reshape(n, t, hq, d)
    return {"out": out.to(s["q"].dtype), "lse": lse.view(n, c["hkv"], t, -1).permute(0, 1, 3, 2).reshape(n, hq, t)}


def _plain_select(s, q):
    """The pages that each token of each KV head reads: [n, tokens, KV heads, slots], ascending, -1 behind them. A page's score is
    the largest, over the head's query heads, of s_q s_K sum_d max(qc min, qc max), an upper bound of q . K for its rows, with qc
    the query in 8 bits (scale s_q = largest magnitude / 127, as for rows)."""
    c = s["case"]
    n, t, hq, d = q.shape
    q = q.float()
    top = q.abs().amax(-1)
    sq = top / torch.full_like(top, 127.0)
    sq = torch.where(torch.isfinite(top), torch.where(sq < 2.0 ** -100, 0.0, sq), math.nan)
    inverse = torch.where(sq > 0, torch.ones_like(sq) / sq, 0.0)
    code = torch.where(torch.isnan(sq).unsqueeze(-1), 0.0, torch.round(q * inverse.unsqueeze(-1)))
    code = code.view(n, t, c["hkv"], -1, d).permute(0, 2, 1, 3, 4)                       # [n, hkv, t, rep, d]
    sq = sq.view(n, t, c["hkv"], -1).permute(0, 2, 1, 3).unsqueeze(-1)
    slot = torch.arange(s["table"].shape[1], device=DEV)
    header = _split(s["pool"], c)[0][_page_of(s["table"], slot.expand(n, -1))].transpose(1, 2)   # [n, hkv, slots, bytes]
    ends = header[..., :2 * d].contiguous().view(torch.int8).float().transpose(2, 3).unsqueeze(2)
    total = torch.matmul(code.clamp_min(0), ends[..., d:, :]) + torch.matmul(code.clamp_max(0), ends[..., :d, :])   # (whole numbers: exact)
    score = sq * _scales(header, d)[..., 0].unsqueeze(2).unsqueeze(2) * total
    score = score.amax(3).nan_to_num(nan=math.inf, posinf=math.inf, neginf=-math.inf)     # [n, hkv, t, slots]
    seen = s["lens"].long().view(-1, 1) - (t - 1 - torch.arange(t, device=DEV))
    pages = ((seen.clamp_min(0) + c["page_rows"] - 1) // c["page_rows"]).view(n, 1, t, 1)
    kind = torch.where((slot < c["first"]) | (slot >= pages - c["last"]), 0, 1)
    kind = torch.where(slot < pages, kind, 2).expand_as(score)
    order = torch.argsort(score, dim=-1, descending=True, stable=True)
    order = torch.gather(order, -1, torch.argsort(torch.gather(kind, -1, order), dim=-1, stable=True))[..., :c["slots"]]
    order = torch.where(torch.gather(kind, -1, order) == 2, slot.numel(), order).sort(-1).values
    order = torch.where(order == slot.numel(), -1, order).permute(0, 2, 1, 3)
    short = torch.full((n, t, c["hkv"], max(0, c["slots"] - order.shape[-1])), -1, device=DEV, dtype=order.dtype)
    return torch.cat((order, short), -1).to(torch.int32)


def _plain_blocks(s, q, slots):
    c, pr = s["case"], s["case"]["page_rows"]
    n, t, hq, d = q.shape
    page = _page_of(s["table"], slots.long())                                             # [n, t, hkv, slots]
    head = torch.arange(c["hkv"], device=DEV).view(-1, 1)
    headers, tiles = _split(s["pool"], c)
    row = (slots.long().unsqueeze(-1) * pr + torch.arange(pr, device=DEV)).flatten(3)
    limit = s["lens"].long().view(-1, 1) - (t - 1 - torch.arange(t, device=DEV))
    seen = (row < limit.view(n, t, 1, 1)) & (row >= 0)
    scale = _scales(headers[page, head], d).repeat_interleave(pr, 3)
    mine = tiles[page, head]
    values = lambda name, at: torch.where(seen.unsqueeze(-1), _codes(mine, s["place"][name]).flatten(3, 4) * scale[..., at:at + 1], 0.0)  # noqa: E731
    score = torch.matmul(q.float().view(n, t, c["hkv"], -1, d), values("k", 0).transpose(3, 4)) / math.sqrt(d)
    out, lse = _attend(score, seen.unsqueeze(3), values("v", 1))
    return out.reshape(n, t, hq, d).to(q.dtype), lse.reshape(n, t, hq).transpose(1, 2).contiguous()


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n, hkv, d, pr = c["n"], c["hkv"], c["d"], c["page_rows"]
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    lens, more = _lengths(c), _new_rows(c)
    held = [_ceil(x + more, pr) for x in lens]
    pages = sum(held) + 4
    # pages lie in the pool in no order, as after hours of serving; the last page of the pool is in no table
    shuffled = torch.randperm(pages - 1, generator=g, device=DEV).to(torch.int32)
    place = _places(d)
    pool = torch.zeros(pages, hkv * _head_bytes(c), dtype=torch.uint8, device=DEV)
    table = torch.full((n, max(1, max(held))), -1, dtype=torch.int32, device=DEV)
    headers, tiles = _split(pool, c)
    centre_k = torch.randn(hkv, 1, d, generator=g, device=DEV)        # keys have channels that stand off from zero
    used = 0
    for i, ln in enumerate(lens):
        table[i, :held[i]] = shuffled[used:used + held[i]]
        ids = table[i, :_ceil(ln, pr)].long()
        used += held[i]
        if ln == 0:
            continue
        there = (torch.arange(ids.numel() * pr, device=DEV) < ln).view(-1, pr)
        header, mine = headers[ids], tiles[ids]
        # what a page's keys have in common is what a score of pages can tell them apart by
        k = torch.randn(ids.numel(), hkv, pr, d, generator=g, device=DEV) + centre_k + 0.7 * torch.randn(ids.numel(), hkv, 1, d, generator=g, device=DEV)
        mn, mx, _, _ = _store(header, mine, place["k"], d, k, there, torch.zeros_like(there), 0)
        _store(header, mine, place["v"], d, torch.randn(ids.numel(), hkv, pr, d, generator=g, device=DEV), there, torch.zeros_like(there), 1)
        header[..., :2 * d] = torch.cat((mn, mx), -1).to(torch.int8).view(torch.uint8)
        headers[ids], tiles[ids] = header, mine
    s = {"case": c, "pool": pool, "table": table, "place": place, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    s["lists"] = torch.arange(n, dtype=torch.int32, device=DEV)
    if c["op"] != "append":
        s["q"] = torch.randn(n, c["q_len"], c["hq"], d, generator=g, device=DEV).to(dtype)
    if more:
        src = c["src"] if c["op"] == "append" else more
        s["k"] = (torch.randn(n, src, hkv, d, generator=g, device=DEV) + centre_k.transpose(0, 1)).to(dtype)
        s["v"] = torch.randn(n, src, hkv, d, generator=g, device=DEV).to(dtype)
        s["at"] = s["lens"].clone()
        s["counts"] = torch.tensor(_counts(c) if c["op"] == "append" else [more] * n, dtype=torch.int32, device=DEV)
        s["idx"] = None
        lists = c.get("lists", 0)
        # positions are those of the original sequence: behind what was there, or the kept rows' own
        pos = 3 * s["lens"].view(-1, 1, 1) + torch.arange(more, dtype=torch.int32, device=DEV)
        if lists:
            keys = torch.rand(n, lists, c["src"], generator=g, device=DEV)
            s["idx"] = torch.sort(torch.topk(keys, c["rows"], dim=2).indices, dim=2).values.to(torch.int32).contiguous()
            pos = 3 * s["lens"].view(-1, 1, 1) + s["idx"]
        s["pos"] = pos.contiguous()
        turn = torch.arange(3 * c["hi"] + c.get("src", more) + 1, device=DEV, dtype=torch.float64).unsqueeze(1) * (
            10000.0 ** (-torch.arange(d // 2, device=DEV, dtype=torch.float64) * 2 / d))
        s["rope"] = torch.cat((turn.cos(), turn.sin()), 1).float()
        if c["op"] == "append":
            s["q"] = torch.randn(n, c["rows"], c["hq"], d, generator=g, device=DEV).to(dtype) if c["hq"] else None
            s["k_out"] = torch.zeros(n, c["rows"], hkv, d, dtype=dtype, device=DEV)
            s["v_out"] = torch.zeros_like(s["k_out"])
    if own:
        from paper_2405_12532_b200 import binding
        p = binding.PyrPages(bits=8, n_kv_heads=hkv, head_dim=d, page_rows=pr, n_pages=pages, n_lists=n, max_pages=table.shape[1])
        for name in ("pool", "table", "lens"):
            view = getattr(p, name)
            view.copy_(s[name])
            s[name] = view
        p.refs.index_fill_(0, table[table >= 0].long(), 1)
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
        if c["op"] == "append":
            q = p.append(s["k"], s["v"], s["lists"], first=s["at"], pos=s["pos"], rope=s["rope"], q=s["q"], idx=s["idx"], counts=s["counts"])
            p.read(s["k_out"], s["v_out"], s["lists"], first=s["at"], counts=s["counts"])
            return {"k": s["k_out"], "v": s["v_out"], "lens": p.lens} | ({} if q is None else {"q": q})
        q = s["q"]
        if c["append"]:
            q = p.append(s["k"], s["v"], s["lists"], first=s["at"], pos=s["pos"], rope=s["rope"], q=q)
        slots = p.select(q, c["slots"], s["lists"], keep_first=c["first"], keep_last=c["last"])
        out, lse = p.attn_blocks(q, slots, s["lists"], lse=True)
        return {"out": out, "lse": lse, "slots": slots}
    if c["op"] == "attn":
        return _plain_attn(s)
    if c["op"] == "append":
        q = _plain_append(s)
        k, v = _plain_read(s)
        return {"k": k, "v": v, "lens": s["lens"]} | ({} if q is None else {"q": q})
    q = _plain_append(s) if c["append"] else s["q"]
    slots = _plain_select(s, q)
    out, lse = _plain_blocks(s, q, slots)
    return {"out": out, "lse": lse, "slots": slots}


# ------------------------------------------------------------------ in 64 bits

def _byte_of(d, row, dim, value):
    """Where a tile holds a code."""
    if not value:
        chunk = dim // 16
        if d == 128 and row % 2:
            chunk = (chunk + 4) % 8
        return row * d + chunk * 16 + dim % 16
    part, four = row % 8 // 2, 2 * (row % 2) + row // 8
    per = d // 8
    chunk = (dim % per // 4) ^ (part & (3 if d == 128 else 1))
    return 16 * d + part * 4 * d + dim // per * 4 * per + chunk * 16 + dim % 4 * 4 + four


def _bytes_of(d, value):
    return torch.tensor([[_byte_of(d, r, x, value) for x in range(d)] for r in range(TILE)], device=DEV)


def _whole_list(s, i, h, value, rows, where):
    """The values of one plane of one head of list i, its first `rows` rows, in 64 bits."""
    c = s["case"]
    d, pr = c["d"], c["page_rows"]
    ids = s["table"][i, :_ceil(rows, pr)].long()
    mine = s["pool"].view(-1, c["hkv"], _head_bytes(c))[ids, h]
    scale = mine[:, 2 * d + 4 * value:2 * d + 4 * value + 4].contiguous().view(torch.float32).double().view(-1, 1, 1)
    tile = mine[:, 2 * d + 16:].reshape(ids.numel(), pr // TILE, -1)
    return ((tile[:, :, where[value]].double() - 128).view(ids.numel(), pr, d) * scale).view(-1, d)[:rows]


def exact(case, seed):
    c = case
    if work(c)["bytes"] > 1_200_000_000 or (c["op"] == "sparse" and c["n"] * c["q_len"] * c["hkv"] > 2100):
        return None
    s = prepare(c, seed)
    n, hkv, d = c["n"], c["hkv"], c["d"]
    where = (_bytes_of(d, 0), _bytes_of(d, 1))
    if c["op"] == "attn":
        t, hq, rep = c["q_len"], c["hq"], c["hq"] // hkv
        out = torch.zeros(n, t, hq, d, dtype=torch.float64, device=DEV)
        lse = torch.full((n, hq, t), -math.inf, dtype=torch.float64, device=DEV)
        for i, ln in enumerate(_lengths(c)):
            for h in range(hkv if ln else 0):
                k, v = _whole_list(s, i, h, 0, ln, where), _whole_list(s, i, h, 1, ln, where)
                for tok in range(max(0, t - ln), t):
                    see = ln - (t - 1 - tok)
                    z = s["q"][i, tok, h * rep:(h + 1) * rep].double() @ k[:see].T / math.sqrt(d)
                    lse[i, h * rep:(h + 1) * rep, tok] = torch.logsumexp(z, -1)
                    out[i, tok, h * rep:(h + 1) * rep] = torch.softmax(z, -1) @ v[:see]
        return {"out": out, "lse": lse}
    if c["op"] == "sparse":
        # over the stored codes and the pages that the plain score names: which those are is a matter of whole numbers
        t, hq, rep, pr = c["q_len"], c["hq"], c["hq"] // hkv, c["page_rows"]
        q = _plain_append(s) if c["append"] else s["q"]
        slots = _plain_select(s, q)
        out = torch.zeros(n, t, hq, d, dtype=torch.float64, device=DEV)
        lse = torch.full((n, hq, t), -math.inf, dtype=torch.float64, device=DEV)
        for i, ln in enumerate(s["lens"].tolist()):
            for h in range(hkv if ln else 0):
                k, v = _whole_list(s, i, h, 0, ln, where), _whole_list(s, i, h, 1, ln, where)
                for tok in range(max(0, t - ln), t):
                    row = torch.arange(ln - (t - 1 - tok), device=DEV)
                    row = row[torch.isin(row // pr, slots[i, tok, h])]
                    z = q[i, tok, h * rep:(h + 1) * rep].double() @ k[row].T / math.sqrt(d)
                    lse[i, h * rep:(h + 1) * rep, tok] = torch.logsumexp(z, -1)
                    out[i, tok, h * rep:(h + 1) * rep] = torch.softmax(z, -1) @ v[row]
        return {"out": out, "lse": lse, "slots": None}
    # append: every stored row at its page's scale
    pr, counts, lens = c["page_rows"], _counts(c), _lengths(c)
    res = {"k": [], "v": []}
    turn = s["rope"].double()
    for name in ("k", "v"):
        got = torch.zeros(n, c["rows"], hkv, d, dtype=torch.float64, device=DEV)
        for i in range(n):
            if counts[i] == 0:
                continue
            x = s[name][i].double()
            angle = turn[s["pos"][i].long()]                             # [lists, rows, d]
            if s["idx"] is not None:
                by = s["idx"][i].long()
                x = torch.stack([x[by[h * by.shape[0] // hkv], h] for h in range(hkv)], 1)
            if name == "k":
                angle = torch.stack([angle[h * angle.shape[0] // hkv] for h in range(hkv)], 1)
                turned = torch.complex(x[..., :d // 2], x[..., d // 2:]) * torch.complex(angle[..., :d // 2], angle[..., d // 2:])
                x = torch.cat((turned.real, turned.imag), -1)
            x = x[:counts[i]]
            old = s["pool"].view(-1, hkv, _head_bytes(c))[s["table"][i, lens[i] // pr].long(), :, 2 * d:2 * d + 8].contiguous().view(torch.float32).double()
            done = 0
            while done < counts[i]:
                end = min(counts[i], done + pr - (lens[i] + done) % pr)
                part = x[done:end]
                scale = part.abs().amax((0, 2)) / 127
                if done == 0 and lens[i] % pr:
                    scale = torch.maximum(scale, old[:, int(name == "v")])
                scale = scale.view(1, -1, 1)
                got[i, done:end] = torch.where(scale > 0, (part / scale).round() * scale, torch.zeros_like(part))
                done = end
        res[name] = got
    res["lens"] = None
    if s["q"] is not None:
        q = s["q"].double()
        angle = turn[s["pos"].long()].transpose(1, 2)
        turned = torch.complex(q[..., :d // 2], q[..., d // 2:]) * torch.complex(angle[..., :d // 2], angle[..., d // 2:])
        live = (torch.arange(c["rows"], device=DEV) < s["counts"].view(-1, 1)).view(n, -1, 1, 1)
        res["q"] = torch.where(live, torch.cat((turned.real, turned.imag), -1), q)
    return res
