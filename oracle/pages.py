"""The paged 4-bit cache by its definition (include/pyr.h), on the CPU: quantisation step by step in IEEE single precision,
the values that codes stand for and attention over them in fp64, and the bookkeeping of pages as plain Python. Shares
nothing with the library."""
from __future__ import annotations

import numpy as np

TILE = 16


def _to_bf16(x, up: bool):
    """fp32 array rounded up / down to the neighbouring bf16 number (exact ones stay)."""
    x = np.asarray(x, np.float32)
    bits = x.view(np.uint32)
    cut = (bits & np.uint32(0xFFFF0000))
    inexact = (bits & np.uint32(0xFFFF)) != 0
    away = inexact & ((x > 0) if up else (x < 0))
    with np.errstate(over="ignore"):
        return (cut + np.where(away, np.uint32(0x10000), np.uint32(0))).astype(np.uint32).view(np.float32)


def quantise(x, group: int):
    """[..., D] -> codes [..., D] (0 .. 15), scale and zero [..., D / group] as fp32 holding bf16 numbers."""
    y = np.asarray(x, np.float32).reshape(*x.shape[:-1], x.shape[-1] // group, group)
    with np.errstate(all="ignore"):
        zero = _to_bf16(y.min(-1), up=False)
        span = (y.max(-1) - zero).astype(np.float32)
        scale = _to_bf16((span / np.float32(15)).astype(np.float32), up=True)
        scale = np.where(scale < np.float32(2.0 ** -100), np.float32(0), scale)
        inv = np.where(scale > 0, np.float32(1) / scale, np.float32(0)).astype(np.float32)
        t = ((y - zero[..., None]).astype(np.float32) * inv[..., None]).astype(np.float32)
        codes = np.rint(t)
    bad = ~np.isfinite(span)
    codes = np.where(bad[..., None], 0, codes).astype(np.int64)
    nan = np.float32(np.nan)
    return codes.reshape(x.shape), np.where(bad, nan, scale), np.where(bad, nan, zero)


def values(codes, scale, zero):
    """What codes stand for, in fp64."""
    group = codes.shape[-1] // scale.shape[-1]
    y = codes.reshape(*codes.shape[:-1], scale.shape[-1], group).astype(np.float64)
    return (y * scale[..., None].astype(np.float64) + zero[..., None].astype(np.float64)).reshape(codes.shape)


def _word_of_k(D, group, d):
    """Nibble position inside a stored K row of dimension d."""
    u, g, r = group // 32, d // group, d % group
    w, nib = r // 8, r % 8
    return 8 * ((w // u) * (D // 32) + g * u + w % u) + nib


def _half_of_v(D, group, d):
    u, g, r = group // 32, d // group, d % group
    h, nib = r // 4, r % 4
    return 4 * ((h // u) * (D // 32) + g * u + h % u) + nib


def tile_bytes(D, group):
    return TILE * (D + 8 * (D // group))


def unpack(tile, D, group):
    """One tile's bytes -> K codes, K scale, K zero, V codes, V scale, V zero of its 16 rows."""
    G, half = D // group, TILE * D // 2
    out = []
    for plane, place in ((0, _word_of_k), (1, _half_of_v)):
        b = tile[plane * half:(plane + 1) * half].reshape(TILE, D // 2)
        nib = np.stack([b & 15, b >> 4], -1).reshape(TILE, D)
        codes = nib[:, [place(D, group, d) for d in range(D)]].astype(np.int64)
        w = tile[2 * half + plane * TILE * G * 4: 2 * half + (plane + 1) * TILE * G * 4].copy().view(np.uint32).reshape(TILE, G)
        out += [codes, (w << np.uint32(16)).view(np.float32), (w & np.uint32(0xFFFF0000)).view(np.float32)]
    return out


def list_values(pool, table_row, length, Hkv, D, group, page_rows):
    """K, V values [length, Hkv, D] in fp64 of one list, from the pool's bytes."""
    tb = tile_bytes(D, group)
    tiles = pool.reshape(pool.shape[0], Hkv, page_rows // TILE, tb)
    K, V = np.zeros((length, Hkv, D)), np.zeros((length, Hkv, D))
    for r0 in range(0, length, TILE):
        page = int(table_row[r0 // page_rows])
        n = min(TILE, length - r0)
        for h in range(Hkv):
            kc, ks, kz, vc, vs, vz = unpack(tiles[page, h, r0 % page_rows // TILE], D, group)
            K[r0:r0 + n, h], V[r0:r0 + n, h] = values(kc, ks, kz)[:n], values(vc, vs, vz)[:n]
    return K, V


def attention(q, K, V, scale):
    """q [T, Hq, D] over K, V [n, Hkv, D]: token t sees the first n - (T - 1 - t) rows. out [T, Hq, D], lse [Hq, T]."""
    T, Hq, D = q.shape
    n, Hkv, _ = K.shape
    out, lse = np.zeros((T, Hq, D)), np.full((Hq, T), -np.inf)
    for t in range(T):
        see = n - (T - 1 - t)
        if see <= 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = K[:see, g] @ q[t, h] * scale
            m = s.max()
            p = np.exp(s - m)
            out[t, h] = p @ V[:see, g] / p.sum()
            lse[h, t] = m + np.log(p.sum())
    return out, lse


class Book:
    """Tables, lengths and reference counts as the calls are defined to leave them. A refused call or entry returns False and
    changes nothing. Moves of rows are reported as (list, destination row, source list, source row) copies."""

    def __init__(self, n_pages, n_lists, max_pages, page_rows):
        self.refs = np.zeros(n_pages, np.int64)
        self.lens = np.zeros(n_lists, np.int64)
        self.table = np.full((n_lists, max_pages), -1, np.int64)
        self.pr, self.max_pages = page_rows, max_pages

    def _pages(self, rows):
        return -(-int(rows) // self.pr)

    def reserve(self, lists, rows):
        """Returns the (old page, new page, rows) copies, or None where the call is refused."""
        if len(set(lists)) != len(lists) or any(r < 0 for r in rows):
            return None
        refs0 = self.refs.copy()
        free = iter(np.flatnonzero(refs0 == 0).tolist())
        todo, copies = [], []
        try:
            for l, r in zip(lists, rows):
                if r == 0:
                    continue
                ln = int(self.lens[l])
                if ln + r > self.max_pages * self.pr:
                    return None
                if ln % self.pr:
                    old = int(self.table[l, ln // self.pr])
                    if refs0[old] > 1:
                        new = next(free)
                        todo.append((l, ln // self.pr, old, new))
                        copies.append((old, new, ln % self.pr))
                for s in range(self._pages(ln), self._pages(ln + r)):
                    if self.table[l, s] < 0:
                        todo.append((l, s, -1, next(free)))
        except StopIteration:
            return None
        for l, s, old, new in todo:
            self.table[l, s] = new
            self.refs[new] = 1
            if old >= 0:
                self.refs[old] -= 1
        return copies

    def fork(self, src, dst):
        done = []
        for i, (s, d) in enumerate(zip(src, dst)):
            alone = d not in src and list(dst).count(d) == 1
            done.append(alone and self.lens[d] == 0 and self.table[d, 0] < 0)
        for s, d, ok in zip(src, dst, done):
            if ok:
                k = self._pages(self.lens[s])
                self.table[d, :k] = self.table[s, :k]
                np.add.at(self.refs, self.table[s, :k], 1)
                self.lens[d] = self.lens[s]
        return done

    def trim(self, lists, rows):
        for l, r in zip(lists, rows):
            self.lens[l] = min(self.lens[l], r)
            self.drop(l)

    def drop(self, l):
        k = self._pages(self.lens[l])
        tail = self.table[l, k:]
        np.add.at(self.refs, tail[tail >= 0], -1)
        tail[:] = -1
