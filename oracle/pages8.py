"""The paged 8-bit cache by its definition (include/pyr.h), on the CPU: what a store makes of a page step by step in IEEE single
precision, the bytes in which codes lie, the score of a page, and attention in fp64 over what codes stand for. Shares nothing
with the library."""
from __future__ import annotations

import numpy as np

TILE = 16
F = np.float32


def k_byte(D, r, d):
    """Byte of a tile that holds the K code of row r, dimension d."""
    chunk = d // 16
    if D == 128 and r % 2 == 1:
        chunk = chunk + 4 if chunk < 4 else chunk - 4
    return r * D + chunk * 16 + d % 16


def v_byte(D, r, d):
    """Byte of a tile that holds the V code of row r, dimension d."""
    lane = (r % 8) // 2
    byte = {(0, 0): 0, (0, 1): 1, (1, 0): 2, (1, 1): 3}[(r % 2, r // 8)]
    eighth, word = divmod(d, D // 8)
    chunk, within = divmod(word, 4)
    swapped = [c for c in range(D // 32) if (c ^ (lane % (D // 32))) == chunk][0]
    return 16 * D + lane * 4 * D + eighth * (D // 2) + swapped * 16 + within * 4 + byte


def head_bytes(D, page_rows):
    return 2 * D + 16 + page_rows // TILE * (32 * D + 16)


def unpack(pool, table_row, length, H, D, page_rows):
    """One list's codes K, V [length, H, D] (int), the tiles' scales K, V [length, H], and by page [pages, H, ...]: extrema and scales."""
    hb = head_bytes(D, page_rows)
    heads = pool.reshape(pool.shape[0], H, hb)
    pages = -(-length // page_rows)
    kmap = np.array([[k_byte(D, r, d) for d in range(D)] for r in range(TILE)])
    vmap = np.array([[v_byte(D, r, d) for d in range(D)] for r in range(TILE)])
    K, V = np.zeros((length, H, D), np.int64), np.zeros((length, H, D), np.int64)
    ks, vs = np.zeros((length, H), F), np.zeros((length, H), F)
    mn, mx = np.zeros((pages, H, D), np.int64), np.zeros((pages, H, D), np.int64)
    ps = np.zeros((pages, H, 2), F)
    for p in range(pages):
        b = heads[int(table_row[p])]
        mn[p], mx[p] = b[:, :D].copy().view(np.int8), b[:, D:2 * D].copy().view(np.int8)
        ps[p] = b[:, 2 * D:2 * D + 8].copy().view(F)
        for t in range(page_rows // TILE):
            r0 = p * page_rows + t * TILE
            n = min(TILE, length - r0)
            if n <= 0:
                break
            tile = b[:, 2 * D + 16 + t * (32 * D + 16):2 * D + 16 + (t + 1) * (32 * D + 16)]
            K[r0:r0 + n] = tile[:, kmap].astype(np.int64).transpose(1, 0, 2)[:n] - 128
            V[r0:r0 + n] = tile[:, vmap].astype(np.int64).transpose(1, 0, 2)[:n] - 128
            tail = tile[:, 32 * D:32 * D + 8].copy().view(F)
            ks[r0:r0 + n], vs[r0:r0 + n] = tail[:, 0], tail[:, 1]
    return K, V, ks, vs, mn, mx, ps


def rotate(x, cs):
    """x [..., D] fp32 turned by cs [..., D] (cosines, sines), every product and sum rounded."""
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h].astype(F), x[..., h:].astype(F), cs[..., :h].astype(F), cs[..., h:].astype(F)
    with np.errstate(all="ignore"):
        return np.concatenate([(a * c).astype(F) - (b * s).astype(F), (b * c).astype(F) + (a * s).astype(F)], -1).astype(F)


def scale_of(amax, before):
    """(scale, factor of codes that stay, inverse) for arrays of largest magnitudes and scales before."""
    with np.errstate(all="ignore"):
        want = (amax.astype(F) / F(127)).astype(F)
        want = np.where(want < F(2.0 ** -100), F(0), want)
        s = np.where(np.isfinite(amax) & ~np.isnan(before), np.fmax(before, want), F(np.nan)).astype(F)
        factor = np.where(s > 0, (before / s).astype(F), F(0)).astype(F)
        inverse = np.where(s > 0, (F(1) / s).astype(F), F(0)).astype(F)
    return s, factor, inverse


class List8:
    """One list's contents. Rows are given as fp32 numbers (after rotation)."""

    def __init__(self, H, D, page_rows, cap):
        self.pr, self.len = page_rows, 0
        slots = -(-cap // page_rows)
        self.code = np.zeros((2, slots * page_rows, H, D), np.int64)
        self.scale = np.zeros((2, slots, H), F)
        self.mn, self.mx = np.zeros((slots, H, D), np.int64), np.zeros((slots, H, D), np.int64)

    def store(self, first, K, V):
        n, pr = K.shape[0], self.pr
        for p in range(first // pr, -(-(first + n) // pr) if n else 0):
            a, b = max(first, p * pr), min(first + n, (p + 1) * pr)
            there = range(p * pr, min(self.len, (p + 1) * pr))
            stay = [r for r in there if r < first or r >= first + n]
            for i, X in enumerate((K, V)):
                x = X[a - first:b - first].astype(F)
                with np.errstate(all="ignore"):
                    amax = np.abs(x).max((0, 2))                     # (NaN goes through)
                    before = self.scale[i, p] if stay else np.zeros_like(self.scale[i, p])
                    s, factor, inverse = scale_of(amax, before)
                    new = np.where(np.isnan(s)[:, None], 0, np.rint((x * inverse[:, None]).astype(F))).astype(np.int64)
                again = lambda c: np.rint((c.astype(F) * factor[:, None]).astype(F)).astype(np.int64)  # noqa: E731
                if stay:
                    self.code[i, stay] = again(self.code[i, stay])
                if i == 0:
                    lo, hi = new.min(0), new.max(0)
                    self.mn[p] = np.minimum(lo, again(self.mn[p])) if stay else lo
                    self.mx[p] = np.maximum(hi, again(self.mx[p])) if stay else hi
                self.code[i, a:b] = new
                self.scale[i, p] = s
        self.len = max(self.len, first + n)

    def copy(self):
        c = object.__new__(List8)
        c.pr, c.len = self.pr, self.len
        c.code, c.scale, c.mn, c.mx = (x.copy() for x in (self.code, self.scale, self.mn, self.mx))
        return c

    def values(self):
        """K, V [len, H, D] in fp64."""
        page = np.arange(self.len) // self.pr
        return [self.code[i, :self.len].astype(np.float64) * self.scale[i, page][:, :, None].astype(np.float64) for i in (0, 1)]


def select(q, mn, mx, k_scale, rows, page_rows, n_slots, first, last):
    """Page slots [H, n_slots] of one token that sees `rows` rows; q [Hq, D] fp32, extrema [pages, H, D], K scales [pages, H]."""
    pages = -(-rows // page_rows) if rows > 0 else 0
    H, rep = mn.shape[1], q.shape[0] // mn.shape[1]
    out = np.full((H, n_slots), -1, np.int64)
    with np.errstate(all="ignore"):
        sq, _, inverse = scale_of(np.abs(q).max(-1), np.zeros(q.shape[0], F))
        code = np.where(np.isnan(sq)[:, None], 0, np.rint((q.astype(F) * inverse[:, None]).astype(F))).astype(np.int64)
        for h in range(H):
            score = np.full(pages, -np.inf, F)
            for g in range(h * rep, (h + 1) * rep):
                total = np.maximum(code[g] * mn[:pages, h], code[g] * mx[:pages, h]).sum(-1)
                one = ((sq[g] * k_scale[:pages, h]).astype(F) * total.astype(F)).astype(F)
                score = np.where(np.isnan(one) | np.isnan(score), F(np.nan), np.maximum(score, one))
            score = np.where(np.isnan(score), F(np.inf), score)
            forced = [p for p in range(pages) if p < first or p >= pages - last] if pages > n_slots else list(range(pages))
            rest = sorted((p for p in range(pages) if p not in forced), key=lambda p: (-float(score[p]), p))
            take = sorted(forced + rest[:n_slots - len(forced)])
            out[h, :len(take)] = take
    return out


def attention(q, K, V, seen, scale):
    """q [T, Hq, D] over K, V [n, H, D]; seen [T, H, n]. out [T, Hq, D], lse [Hq, T], and for tolerances sum p |v| [T, Hq, D] and the
    largest sum |q| |k| scale over the rows seen [T, Hq]."""
    T, Hq, D = q.shape
    n, H, _ = K.shape
    out, mass, size = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    lse = np.full((Hq, T), -np.inf)
    for t in range(T):
        for g in range(Hq):
            h = g // (Hq // H)
            at = np.flatnonzero(seen[t, h])
            if at.size == 0:
                continue
            s = K[at, h] @ q[t, g] * scale
            m = s.max()
            p = np.exp(s - m)
            out[t, g] = p @ V[at, h] / p.sum()
            mass[t, g] = p @ np.abs(V[at, h]) / p.sum()
            size[t, g] = (np.abs(K[at, h]) @ np.abs(q[t, g])).max() * scale
            lse[g, t] = m + np.log(p.sum())
    return out, lse, mass, size
