"""The paged 8-bit cache on the GPU against its definition (oracle/pages8.py): stored codes, scales and extrema, page selection, and
attention in fp64 over what the codes stand for."""
import math

import numpy as np
import pytest
import torch

from oracle import pages8 as o8
from paper_2405_12532_b200 import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def _ids(*x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def _np(t):
    return t.detach().cpu().float().numpy()


def _rand(*shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).to(DEV)


def _pages(H, D, pr, n_pages, n_lists, max_pages, bits=8):
    p = pb.PyrPages(bits=bits, n_kv_heads=H, head_dim=D, page_rows=pr, n_pages=n_pages, n_lists=n_lists, max_pages=max_pages)
    p.pool.fill_(0xFF)               # stale bytes: every scale a NaN
    return p


def _unpack(p, l):
    c = p.cfg
    return o8.unpack(p.pool.cpu().numpy(), p.table[l].cpu().numpy(), int(p.lens[l]), c.n_kv_heads, c.head_dim, c.page_rows)


def _check(p, l, want):
    """List l holds exactly what the definition says: codes, both copies of the scales, extrema."""
    assert int(p.lens[l]) == want.len
    K, V, ks, vs, mn, mx, ps = _unpack(p, l)
    page, n = np.arange(want.len) // want.pr, -(-want.len // want.pr)
    for got, i, s in ((K, 0, ks), (V, 1, vs)):
        nan = np.isnan(want.scale[i, page])[:, :, None]
        np.testing.assert_array_equal(np.where(nan, 0, got), np.where(nan, 0, want.code[i, :want.len]))
        np.testing.assert_array_equal(s, want.scale[i, page])
        np.testing.assert_array_equal(ps[:, :, i], want.scale[i, :n])
    nan = np.isnan(want.scale[0, :n])[:, :, None]
    np.testing.assert_array_equal(np.where(nan, 0, mn), np.where(nan, 0, want.mn[:n]))
    np.testing.assert_array_equal(np.where(nan, 0, mx), np.where(nan, 0, want.mx[:n]))


def _state(p):
    return [t.clone() for t in (p.pool, p.table, p.lens, p.refs)]


def _unchanged(p, state):
    return all(torch.equal(a, b) for a, b in zip((p.pool, p.table, p.lens, p.refs), state))


def _filled(H, D, pr, lens, seed, spare=2, dtype=BF, kscale=1.0, vscale=1.0):
    """Lists of the given lengths, written in one go, pages in the pool's order turned round."""
    cap = max(max(lens), 1) + spare
    slots = -(-cap // pr)
    p = _pages(H, D, pr, len(lens) * slots + 3, len(lens), slots)
    order = list(range(len(lens)))[::-1]
    if order:
        p.reserve(_ids(*order), cap)
    k, v = _rand(len(lens), max(max(lens), 1), H, D, seed=seed, dtype=dtype, scale=kscale), _rand(len(lens), max(max(lens), 1), H, D, seed=seed + 1, dtype=dtype, scale=vscale)
    p.write(k, v, counts=_ids(*lens))
    want = []
    for i, n in enumerate(lens):
        w = o8.List8(H, D, pr, slots * pr)
        w.store(0, _np(k[i, :n]), _np(v[i, :n]))
        want.append(w)
    assert p.status() == 0
    return p, want


# ------------------------------------------------------------------ storing

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,pr", [(64, 16), (64, 80), (128, 16), (128, 48), (128, 128)])
def test_rows_are_stored_as_defined_wherever_they_begin(D, pr, dtype):
    """Chunks of many sizes behind one another, of growing and shrinking magnitude: codes that stay go to the new scales."""
    H, lists, cap = 3, (2, 0, 3), 300
    p = _pages(H, D, pr, 80, 4, 24)
    p.reserve(_ids(*lists), cap)
    want = {l: o8.List8(H, D, pr, 24 * pr) for l in lists}
    for step, (rows, scale) in enumerate([(5, 1.0), (40, 0.3), (1, 2.0), (16, 3.0), (2, 0.01), (1, 40.0), (33, 4.0), (150, 1.0)]):
        k, v = _rand(3, rows, H, D, seed=step, dtype=dtype, scale=scale), _rand(3, rows, H, D, seed=50 + step, dtype=dtype, scale=5 * scale)
        counts = [rows, max(0, rows - 3), rows]
        p.write(k, v, _ids(*lists), counts=_ids(*counts))
        for i, l in enumerate(lists):
            want[l].store(want[l].len, _np(k[i, :counts[i]]), _np(v[i, :counts[i]]))
            _check(p, l, want[l])
    assert p.status() == 0 and int(p.lens[1]) == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_one_by_one(D, dtype):
    """The decode step's form: every scale grows, falls behind and grows again within a page; and rows in the middle stored anew."""
    H, pr = 9, 32                    # more heads than a CTA has warps
    p = _pages(H, D, pr, 8, 2, 3)
    p.reserve(_ids(1), 70)
    want = o8.List8(H, D, pr, 96)
    for r in range(70):
        scale = (1.0, 0.2, 1.5, 8.0, 0.1)[r % 5] * (1 + r // 20)
        k, v = _rand(1, 1, H, D, seed=r, dtype=dtype, scale=scale), _rand(1, 1, H, D, seed=100 + r, dtype=dtype, scale=1 / scale)
        p.write(k, v, _ids(1))
        want.store(want.len, _np(k[0]), _np(v[0]))
        if r in (0, 1, 15, 16, 31, 32, 33, 50, 69):
            _check(p, 1, want)
    for first, scale in ((3, 30.0), (31, 1.0), (32, 90.0), (69, 5.0), (0, 0.5), (64, 200.0)):
        k, v = _rand(1, 1, H, D, seed=first + 300, dtype=dtype, scale=scale), _rand(1, 1, H, D, seed=first + 400, dtype=dtype, scale=scale)
        p.write(k, v, _ids(1), first=_ids(first))
        want.store(first, _np(k[0]), _np(v[0]))
        _check(p, 1, want)
    for first, n in ((10, 20), (0, 32), (30, 38), (64, 6)):                # ranges, with rows before and behind them in their pages
        k, v = _rand(1, n, H, D, seed=first + 500, dtype=dtype, scale=first + 1.0), _rand(1, n, H, D, seed=first + 600, dtype=dtype)
        p.write(k, v, _ids(1), first=_ids(first))
        want.store(first, _np(k[0]), _np(v[0]))
        _check(p, 1, want)
    assert p.status() == 0


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("rows", [1, 37])
def test_kept_rows_at_their_positions(groups, rows):
    """Gathered rows (an index list a sequence or a head, from head-major tensors), keys turned by positions of their own."""
    H, D, pr, n, src = 4, 128, 32, 3, 60
    p = _pages(H, D, pr, 30, 5, 4)
    lists, counts = (4, 0, 2), ([rows, rows - 9, 0] if rows > 1 else [1, 1, 0])
    p.reserve(_ids(*lists), 100)
    base_k, base_v = _rand(n, 21, H, D, seed=1, dtype=BF), _rand(n, 21, H, D, seed=2, dtype=BF)
    p.write(base_k, base_v, _ids(*lists))
    k, v = (_rand(n, H, src, D, seed=s, dtype=BF, scale=2.0).transpose(1, 2) for s in (3, 4))
    g = torch.Generator().manual_seed(5)
    idx = torch.randint(0, src, (n, groups, rows), generator=g).to(torch.int32).to(DEV)
    pos = torch.randint(0, 500, (n, groups, rows), generator=g).to(torch.int32).to(DEV)
    rope = pb.glue_rope_table(500, D)
    p.append(k, v, _ids(*lists), pos=pos, rope=rope, idx=idx, counts=_ids(*counts))
    assert p.status() == 0
    table = _np(rope)
    for i, l in enumerate(lists):
        want = o8.List8(H, D, pr, 128)
        want.store(0, _np(base_k[i]), _np(base_v[i]))
        ks, vs = np.zeros((counts[i], H, D), np.float32), np.zeros((counts[i], H, D), np.float32)
        for h in range(H):
            at = idx[i, h % groups, :counts[i]].cpu().numpy()
            ks[:, h] = o8.rotate(_np(k[i])[at, h], table[pos[i, h % groups, :counts[i]].cpu().numpy()])
            vs[:, h] = _np(v[i])[at, h]
        if counts[i]:
            want.store(21, ks, vs)
        _check(p, l, want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,hq", [(1, 40), (6, 10)])
def test_queries_are_turned_beside_the_rows(rows, hq, D, dtype):
    """q_out, in place and apart, strided, and queries of rows that are not stored as they are. Keys equal those turned beforehand."""
    H, pr, n = 2, 16, 3
    rope = pb.glue_rope_table(90000, D, base=500000.0)
    pos = torch.tensor([[[7]], [[89990]], [[400]]], dtype=torch.int32, device=DEV) + torch.arange(rows, dtype=torch.int32, device=DEV)
    k, v = _rand(n, rows, H, D, seed=1, dtype=dtype), _rand(n, rows, H, D, seed=2, dtype=dtype)
    q = _rand(n, hq, rows, D, seed=3, dtype=dtype).transpose(1, 2)
    counts = [rows, rows - 1, rows]
    p = _pages(H, D, pr, 10, 3, 2)
    p.reserve(_ids(0, 1, 2), rows)
    out = p.append(k, v, pos=pos, rope=rope, q=q, counts=_ids(*counts))
    want = o8.rotate(_np(q), _np(rope)[pos.cpu().numpy()[:, 0]][:, :, None])
    want = torch.from_numpy(want).to(dtype).float().numpy()
    want[1, rows - 1] = _np(q)[1, rows - 1]
    np.testing.assert_array_equal(_np(out), want)
    for i in range(n):
        w = o8.List8(H, D, pr, 32)
        w.store(0, o8.rotate(_np(k[i, :counts[i]]), _np(rope)[pos[i, 0, :counts[i]].cpu().numpy()][:, None]), _np(v[i, :counts[i]]))
        if counts[i]:
            _check(p, i, w)
    mine = q.clone()
    p.trim(_ids(0, 1, 2), _ids(0, 0, 0))
    p.reserve(_ids(0, 1, 2), rows)
    assert p.append(k, v, pos=pos, rope=rope, q=mine, q_out=mine, counts=_ids(*counts)) is mine
    np.testing.assert_array_equal(_np(mine), want)
    assert p.status() == 0


def test_rope_table():
    """Cosines and sines in double, rounded: half a step of fp32 at 1, 2^-25, and the double's own error at angles up to 2^31."""
    for first, n, D, base in ((0, 700, 128, 10000.0), (2_000_000_000, 64, 64, 500000.0)):
        got = _np(pb.glue_rope_table(n, D, base=base, first=first)).astype(np.float64)
        ang = (first + np.arange(n, dtype=np.float64))[:, None] * base ** (-2.0 * np.arange(D // 2) / D)
        tol = 2.0 ** -25 + 2.0 ** -51 * (first + n)
        assert np.abs(got[:, :D // 2] - np.cos(ang)).max() <= tol and np.abs(got[:, D // 2:] - np.sin(ang)).max() <= tol


@pytest.mark.parametrize("rows", [1, 20])
def test_values_that_cannot_be_stored_and_very_small_ones(rows):
    """Inf, NaN and what lies out of range make a page's rows of that head NaN, the others stay; magnitudes below 127 * 2^-100 are 0; a page
    filled anew is free of all that."""
    H, D, pr = 5, 128, 32
    p = _pages(H, D, pr, 6, 2, 2)
    p.reserve(_ids(0), 64)
    want = o8.List8(H, D, pr, 64)
    k0, v0 = _rand(1, 8, H, D, seed=1), _rand(1, 8, H, D, seed=2)
    p.write(k0, v0, _ids(0))
    want.store(0, _np(k0[0]), _np(v0[0]))
    k, v = _rand(1, rows, H, D, seed=3), _rand(1, rows, H, D, seed=4)
    k[0, 0, 0, 5], v[0, 0, 1, 127], k[0, -1, 2, 64] = math.inf, math.nan, -math.inf
    k[0, :, 3] *= 2.0 ** -120
    v[0, :, 4] *= 1e37
    p.write(k, v, _ids(0))
    want.store(8, _np(k[0]), _np(v[0]))
    _check(p, 0, want)
    assert np.isnan(want.scale[0, 0, 0]) and np.isnan(want.scale[1, 0, 1]) and np.isnan(want.scale[0, 0, 2]) and want.scale[1, 0, 4] > 1e34
    ko, vo = torch.zeros(1, 8 + rows, H, D, device=DEV), torch.zeros(1, 8 + rows, H, D, device=DEV)
    p.read(ko, vo, _ids(0))
    assert ko[0, :, 0].isnan().all() and vo[0, :, 1].isnan().all() and vo[0, :, 0].isfinite().all() and ko[0, :, 1].isfinite().all()
    p.trim(_ids(0), _ids(0))
    p.reserve(_ids(0), 64)
    for x in (2.0 ** -100, 2.0 ** -120, 0.0):                 # a page of very small rows: a scale of 0
        k = torch.full((1, rows, H, D), x, device=DEV)
        p.write(k, k, _ids(0), first=_ids(0))
        want = o8.List8(H, D, pr, 64)
        want.store(0, _np(k[0]), _np(k[0]))
        _check(p, 0, want)
        assert (want.scale[0, 0] == 0).all()
    assert p.status() == 0


@pytest.mark.parametrize("rows", [1, 3])
def test_refused_entries_are_left_as_they_were(rows):
    """A list twice, first beyond the end, counts and ids out of range, no page, a shared page: that entry only, and it is reported. Rows
    whose source or position is out of range are stored as NaN."""
    H, D, pr = 2, 64, 16
    p, want = _filled(H, D, pr, [20, 20, 20, 20], seed=1, spare=rows)
    k, v = _rand(4, rows, H, D, seed=8), _rand(4, rows, H, D, seed=9)
    rope, pos = pb.glue_rope_table(50, D), torch.zeros(4, 1, rows, dtype=torch.int32, device=DEV)
    q = _rand(4, rows, 4, D, seed=10)

    def left(changed, **kw):
        old = _state(p)
        got = p.append(k, v, pos=pos, rope=rope, q=q, **kw)
        assert p.status() == pb.PYR_ERR_INVALID and p.status() == 0
        for l in range(4):
            if l in changed:
                assert int(p.lens[l]) == 20 + rows
            else:
                assert int(p.lens[l]) == 20
                _check(p, l, want[l])
        for t, o in zip((p.pool, p.table, p.lens, p.refs), old):
            t.copy_(o)
        return got

    left([3], lists=_ids(1, 1, 3, 7))
    out = left([0, 3], lists=_ids(0, 1, 2, 3), first=_ids(20, 21, -1, 20))
    assert torch.equal(out[1:3], q[1:3])
    left([0, 2], counts=_ids(rows, rows + 1, rows, -1))
    p.fork(_ids(0), _ids(0))                                   # refused: its own source
    assert p.status() == pb.PYR_ERR_INVALID
    p.trim(_ids(3))
    p.fork(_ids(0), _ids(3))
    want[3] = want[0].copy()
    left([1, 2], lists=_ids(0, 1, 2, 3))                       # lists 0 and 3 share the page that ends inside
    p.table[2, 1] = 1 << 20
    old = p.table.clone()
    p.write(k, v, _ids(2, 1, 0, 3))
    assert p.status() == pb.PYR_ERR_INVALID and int(p.lens[2]) == 20 and int(p.lens[1]) == 20 + rows
    assert torch.equal(p.table, old)
    bad = torch.full((1, 1, rows), 50, dtype=torch.int32, device=DEV)
    for kw in (dict(pos=bad, rope=rope, q=q[:1]), dict(idx=bad), dict(pos=-bad, rope=rope)):
        first = int(p.lens[1])
        p.reserve(_ids(1), rows)
        out = p.append(k[:1], v[:1], _ids(1), **kw)
        assert p.status() == pb.PYR_ERR_INVALID and int(p.lens[1]) == first + rows
        ko, vo = torch.zeros(1, rows, H, D, device=DEV), torch.zeros(1, rows, H, D, device=DEV)
        p.read(ko, vo, _ids(1), first=_ids(first))
        assert ko.isnan().all() and vo.isnan().all() and (out is None or out.isnan().all())


def test_reading_leaves_the_rest():
    """Windows that begin and end inside tiles, head-major and padded outputs, bf16 and fp32: values are scale * code rounded, rows behind
    a list's end stay."""
    H, D, pr = 3, 128, 48
    p, want = _filled(H, D, pr, [100, 7, 0], seed=4)
    for dtype in (BF, F32):
        k = torch.full((3, H, 41, D + 8), -9.0, dtype=dtype, device=DEV)[..., :D].transpose(1, 2)
        v = torch.full((3, H, 41, D + 8), -9.0, dtype=dtype, device=DEV)[..., :D].transpose(1, 2)
        first, counts = [63, 5, 0], [41, 1, 41]
        p.read(k, v, first=_ids(*first), counts=_ids(*counts))
        for i in range(3):
            n = max(0, min(want[i].len - first[i], counts[i]))
            for t, w in zip((k, v), want[i].values()):
                x = torch.from_numpy(w[first[i]:first[i] + n].astype(np.float32)).to(dtype).float().numpy()
                np.testing.assert_array_equal(_np(t[i, :n]), x)
                assert (t[i, n:] == -9).all()
    assert p.status() == 0


def test_branches_share_pages_and_part_with_them():
    """A fork's rows are the original's; after room is made on the branch both grow on their own, scales and extrema included."""
    H, D, pr = 2, 128, 64
    p, want = _filled(H, D, pr, [90, 0], seed=7, spare=30)
    p.trim(_ids(1))
    p.trim(_ids(0), _ids(85))
    want[0].len = 85
    p.fork(_ids(0), _ids(1))
    want[1] = want[0].copy()
    p.reserve(_ids(1), 3)
    p.reserve(_ids(0), 3)
    for i, scale in ((1, 9.0), (0, 0.5)):
        k, v = _rand(1, 3, H, D, seed=20 + i, scale=scale), _rand(1, 3, H, D, seed=30 + i, scale=scale)
        p.write(k, v, _ids(i))
        want[i].store(85, _np(k[0]), _np(v[0]))
    _check(p, 0, want[0])
    _check(p, 1, want[1])
    assert p.status() == 0


# ------------------------------------------------------------------ attention

def _tolerances(dtype, out, mass, size, lse):
    """What the roundings make of an output, with mass = sum p |v| and size = sum |q| |k| scale: the output's own half step, 2^-8 of it in bf16;
    weights as f16, 2^-11 (fp32: two f16, 2^-22, the exponential's 2^-22 and the sums of a few hundred terms a lane). Scores: products
    summed by the instruction in 8 steps that lose 2^-22 of their size each, fp32 queries as two f16 (2^-22), three products rounded: 2^-19
    (fp32: 2^-18) in all; an error of a score goes into a weight and into the denominator."""
    score = size * (2.0 ** -19 if dtype == BF else 2.0 ** -18)
    rel = (2.0 ** -11 + 2.0 ** -19 if dtype == BF else 2.0 ** -19) + 2 * score
    last = 2.0 ** -8 if dtype == BF else 2.0 ** -22
    return last * np.abs(out) + rel[..., None] * mass + 1e-30, score.T + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(np.isinf(lse), 0, lse))


def _compare(dtype, got, got_lse, want):
    out, lse, mass, size = want
    tol, ltol = _tolerances(dtype, out, mass, size, lse)
    err = np.abs(got.astype(np.float64) - out)
    assert np.all(err <= tol), (err - tol).max()
    inf = np.isinf(lse)
    np.testing.assert_array_equal(np.isinf(got_lse), inf)
    assert np.all(np.abs(np.where(inf, 0, got_lse - np.where(inf, 0, lse))) <= ltol)


def _dense(n, T, H, page_rows=None, slots=None):
    """Which rows each token and KV head sees, [T, H, n]: causal over the last T rows, in the chosen pages if slots [T, H, m] are given."""
    row = np.arange(n)
    seen = np.broadcast_to(row < (n - (T - 1 - np.arange(T)))[:, None, None], (T, H, n)).copy()
    if slots is not None:
        for t in range(T):
            for h in range(H):
                seen[t, h] &= np.isin(row // page_rows, slots[t, h][slots[t, h] >= 0])
    return seen


LENGTHS = [1, 0, 15, 16, 17, 31, 33, 47, 48, 49, 64, 100, 129, 300]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,pr,H,rep,T", [(128, 64, 2, 1, 1), (128, 16, 1, 5, 1), (128, 48, 2, 8, 2), (128, 128, 1, 12, 3), (64, 32, 3, 1, 4),
                                          (64, 16, 1, 3, 1), (64, 112, 2, 4, 5)])
def test_attention_over_lists_of_any_length(D, pr, H, rep, T, dtype):
    p, want = _filled(H, D, pr, LENGTHS, seed=11, dtype=dtype)
    q = _rand(len(LENGTHS), T, H * rep, D, seed=13, dtype=dtype, scale=1.5)
    out, lse = p.attn(q, lse=True)
    assert p.status() == 0
    for i, n in enumerate(LENGTHS):
        K, V = want[i].values()
        _compare(dtype, _np(out[i]), _np(lse[i]), o8.attention(_np(q[i]).astype(np.float64), K, V, _dense(n, T, H), 1 / math.sqrt(D)))
    # some lists, one of them twice, one that does not exist; outputs of another order and in head-major tensors
    some = [9, 3, 9, 99]
    qs = _rand(4, H * rep, T, D, seed=14, dtype=dtype).transpose(1, 2)
    buf = torch.full((4, H * rep, T, D), 7.0, dtype=dtype, device=DEV).transpose(1, 2)
    p.attn(qs, _ids(*some), out=buf, softmax_scale=0.3)
    assert p.status() == pb.PYR_ERR_INVALID and (buf[3] == 7).all()
    for i, l in enumerate(some[:3]):
        K, V = want[l].values()
        want_out = o8.attention(_np(qs[i]).astype(np.float64), K, V, _dense(LENGTHS[l], T, H), 0.3)
        tol, _ = _tolerances(dtype, want_out[0], want_out[2], want_out[3], want_out[1])
        assert np.all(np.abs(_np(buf[i]) - want_out[0]) <= tol)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_over_pages_whose_scales_are_far_apart(dtype):
    """Scales of V (and of K) from 1e-25 to 1e20 in one list, pages of zeros, and scores that make the small ones count: sums follow
    the weights times scales, not the weights."""
    H, D, pr = 1, 128, 16
    p = _pages(H, D, pr, 16, 1, 12)
    p.reserve(_ids(0), 12 * 16)
    want = o8.List8(H, D, pr, 192)
    for page, (ks, vs) in enumerate([(1, 1), (3, 1e-25), (0.1, 1e-3), (1, 0), (0, 1), (4, 1e-6), (1, 30.0), (2, 1e-12), (5, 1e-20), (1, 1e-25), (3, 1e-2), (1, 0)]):
        k, v = _rand(1, 16, H, D, seed=page, dtype=dtype, scale=ks), _rand(1, 16, H, D, seed=page + 40, dtype=dtype, scale=vs)
        p.write(k, v, _ids(0))
        want.store(16 * page, _np(k[0]), _np(v[0]))
    K, V = want.values()
    for seed, scale in ((1, 0.0884), (2, 0.5), (3, 3.0)):
        q = _rand(1, 1, 6, D, seed=seed, dtype=dtype)
        out, lse = p.attn(q, lse=True, softmax_scale=scale)
        _compare(dtype, _np(out[0]), _np(lse[0]), o8.attention(_np(q[0]).astype(np.float64), K, V, _dense(192, 1, H), scale))
    big = _pages(H, D, pr, 4, 1, 2)
    big.reserve(_ids(0), 32)
    want = o8.List8(H, D, pr, 32)
    for page, vs in enumerate((1e20, 1e-20)):
        k, v = _rand(1, 16, H, D, seed=page, scale=1e-15), _rand(1, 16, H, D, seed=page + 40, scale=vs)
        big.write(k, v)
        want.store(16 * page, _np(k[0]), _np(v[0]))
    K, V = want.values()
    q = _rand(1, 1, 2, D, seed=6, dtype=dtype, scale=1e15)
    out, lse = big.attn(q, lse=True)
    _compare(dtype, _np(out[0]), _np(lse[0]), o8.attention(_np(q[0]).astype(np.float64), K, V, _dense(32, 1, H), 1 / math.sqrt(D)))


def test_attention_over_many_rows_of_little_weight():
    """One row of much weight before 40 000 of little (2^-17 and 2^-22 of it): f16 weights far below the largest keep their bits. The error of
    a sum of rows is that of one, 2^-11, at most."""
    H, D, pr, n = 1, 128, 128, 40000
    for far in (17.0, 22.0):
        p = _pages(H, D, pr, 330, 1, 320)
        p.reserve(_ids(0), n)
        k = torch.zeros(1, n, H, D, device=DEV)
        k[0, 0, 0, 0] = far * math.log(2.0)
        v = torch.rand(1, n, H, D, generator=torch.Generator().manual_seed(1)).to(DEV) + 0.5
        p.write(k, v)
        want = o8.List8(H, D, pr, 313 * 128)
        want.store(0, _np(k[0]), _np(v[0]))
        K, V = want.values()
        for dtype in (BF, F32):
            q = torch.zeros(1, 1, 1, D, dtype=dtype, device=DEV)
            q[..., 0] = 1.0
            out, lse = p.attn(q, lse=True, softmax_scale=1.0)
            _compare(dtype, _np(out[0]), _np(lse[0]), o8.attention(_np(q[0]).astype(np.float64), K, V, _dense(n, 1, H), 1.0))


def test_what_is_not_finite_shows_where_it_is_seen_and_nowhere_else():
    """A page of NaN reaches the tokens that see it (and its head, and its plane's outputs); rows behind the end and unseen pages do not."""
    H, D, pr = 2, 64, 16
    p, want = _filled(H, D, pr, [40], seed=3, spare=24)
    nan = torch.full((1, 1, H, D), math.nan, device=DEV)
    one = torch.ones(1, 1, H, D, device=DEV)
    row = nan.clone()
    row[:, :, 1] = 1.0
    q = _rand(1, 2, 4, D, seed=5, dtype=BF)
    clean, clean_lse = p.attn(q, lse=True)
    p.append(one, row, _ids(0))                                 # V of head 0: rows 32 .. 40 are NaN
    p.trim(_ids(0), _ids(32))
    first, _ = p.attn(q, lse=True)
    assert first.isfinite().all()
    p.reserve(_ids(0), 20)
    p.append(row, one, _ids(0))                                 # a page begun anew: K of head 0 is NaN from row 32 on
    out, lse = p.attn(q, lse=True)
    assert out[0, 1, :2].isnan().all() and lse[0, :2, 1].isnan().all()          # the last token sees row 32
    assert out[0, 0].isfinite().all() and lse[0, :, 0].isfinite().all()         # the one before sees rows 0 .. 31
    assert out[0, 1, 2:].isfinite().all() and clean.isfinite().all() and clean_lse.isfinite().all()
    # a query row that is not finite
    q[0, 0, 1, 3] = math.inf
    out = p.attn(q)
    assert not out[0, 0, 1].isfinite().any() and out[0, 0, 0].isfinite().all() and out[0, 0, 2:].isfinite().all()
    assert p.status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_far_from_zero(dtype):
    """Scores up to 2^33: the weights are those of the largest. (Where products round, neighbouring rows' scores are 2^10 apart.)"""
    H, D, pr, n = 1, 128, 64, 70
    p = _pages(H, D, pr, 3, 1, 2)
    p.reserve(_ids(0), n)
    k, v = torch.zeros(1, n, H, D, device=DEV), _rand(1, n, H, D, seed=2)
    k[0, :, 0, 0] = torch.linspace(-127, 127, n).round().to(DEV)
    p.write(k, v)
    want = o8.List8(H, D, pr, 128)
    want.store(0, _np(k[0]), _np(v[0]))
    q = torch.zeros(1, 1, 2, D, dtype=dtype, device=DEV)
    q[0, 0, 0, 0], q[0, 0, 1, 0] = 2.0 ** 26, -(2.0 ** 26)
    out, lse = p.attn(q, lse=True, softmax_scale=1.0)
    K, V = want.values()
    for head, row in ((0, n - 1), (1, 0)):
        last = 2.0 ** -8 if dtype == BF else 2.0 ** -20
        assert np.all(np.abs(_np(out[0, 0, head]) - V[row, 0]) <= last * np.abs(V[row, 0]) + 2.0 ** -20)
        assert abs(float(lse[0, head, 0]) / (127 * 2.0 ** 26) - 1) <= 2.0 ** -20


def test_attention_splits_long_lists():
    """A list over the whole machine beside short and empty ones: states that cross CTAs, one and many heads of queries."""
    H, D, pr, lens = 2, 128, 64, [30000, 5, 0, 900]
    p, want = _filled(H, D, pr, lens, seed=21, spare=1)
    for rep, T in ((1, 1), (8, 1), (3, 3)):
        q = _rand(4, T, H * rep, D, seed=22, dtype=BF)
        out, lse = p.attn(q, lse=True)
        again, lse2 = p.attn(q, lse=True)
        assert torch.equal(out, again) and torch.equal(lse, lse2)              # bit-reproducible
        for i, n in enumerate(lens):
            K, V = want[i].values()
            _compare(BF, _np(out[i]), _np(lse[i]), o8.attention(_np(q[i]).astype(np.float64), K, V, _dense(n, T, H), 1 / math.sqrt(D)))
    assert p.status() == 0


def _sampled(p, want_of, out, lse, q, lists, rep, T, dtype, at, H, pr, slots=None):
    for i in at:
        w = want_of(lists[i])
        K, V = w.values()
        seen = _dense(w.len, T, H, pr, None if slots is None else slots[i].cpu().numpy())
        _compare(dtype, _np(out[i]), _np(lse[i]), o8.attention(_np(q[i]).astype(np.float64), K, V, seen, 1 / math.sqrt(q.shape[-1])))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_long_list_in_hundreds_of_pieces(dtype):
    """A list of 60 001 rows: every head's states come from hundreds of ranges, and are merged in three rounds; one and nine query heads."""
    H, D, pr, n = 8, 128, 128, 60001
    p, want = _filled(H, D, pr, [n, 3], seed=81, spare=1)
    for rep in (1, 9):
        q = _rand(2, 1, H * rep, D, seed=82, dtype=dtype)
        out, lse = p.attn(q, lse=True)
        for _ in range(2):
            again, lse2 = p.attn(q, lse=True)
            assert torch.equal(out, again) and torch.equal(lse, lse2)              # bit-reproducible
        _sampled(p, lambda l: want[l], out, lse, q, [0, 1], rep, 1, dtype, (0, 1), H, pr)
    assert p.status() == 0


def test_hundreds_of_ragged_lists():
    """More work than warps by far, over lists from none to 1200 rows, one that does not exist among them; more entries than a CTA has threads, and
    more than it has a table for; dense and over chosen pages."""
    H, D, pr, rep, n = 8, 128, 64, 2, 300
    lens = [(i * 7919) % 1201 if i % 13 else 0 for i in range(n)]
    p, want = _filled(H, D, pr, lens, seed=83, spare=2)
    sample = [0, 1, 13, 57, 100, 255, 256, 257, 299]
    q = _rand(n, 2, H * rep, D, seed=84, dtype=BF)
    out, lse = p.attn(q, lse=True)
    _sampled(p, lambda l: want[l], out, lse, q, list(range(n)), rep, 2, BF, sample, H, pr)
    slots = p.select(q, 6, keep_first=1, keep_last=1)
    blocks, blse = p.attn_blocks(q, slots, lse=True)
    _sampled(p, lambda l: want[l], blocks, blse, q, list(range(n)), rep, 2, BF, sample, H, pr, slots)
    for i in sample:
        np.testing.assert_array_equal(slots[i].cpu().numpy(), _slots_of(want[i], _np(q[i]), lens[i], pr, 6, 1, 1))
    again, blse2 = p.attn_blocks(q, slots, lse=True)
    assert torch.equal(blocks, again) and torch.equal(blse, blse2) and p.status() == 0
    lists = [(i * 37) % n for i in range(1100)]
    lists[500] = n + 5
    many = _rand(1100, 1, H * rep, D, seed=85, dtype=BF)
    for count in (900, 1100):
        out = torch.full((count, 1, H * rep, D), 3.0, dtype=BF, device=DEV)
        _, lse = p.attn(many[:count], _ids(*lists[:count]), out=out, lse=True)
        assert p.status() == pb.PYR_ERR_INVALID and (out[500] == 3).all()
        _sampled(p, lambda l: want[l], out, lse, many, lists, rep, 1, BF, [0, 1, 2, 499, 501, count - 1], H, pr)


def test_pages_beyond_32_bits():
    """A pool of 5 GB: rows in its last pages are stored, read, selected and attended where they lie."""
    H, D, pr = 40, 128, 128
    page = H * o8.head_bytes(D, pr)
    n_pages = (5 << 30) // page
    p = pb.PyrPages(bits=8, n_kv_heads=H, head_dim=D, page_rows=pr, n_pages=n_pages, n_lists=2, max_pages=4)
    p.refs.fill_(1)
    p.refs[-4:] = 0
    p.reserve(_ids(1), 500)
    assert p.status() == 0 and p.table[1].tolist() == list(range(n_pages - 4, n_pages))
    k, v = _rand(1, 500, H, D, seed=1, dtype=BF), _rand(1, 500, H, D, seed=2, dtype=BF)
    p.write(k[:, :499], v[:, :499], _ids(1))
    p.write(k[:, 499:], v[:, 499:], _ids(1))
    want = o8.List8(H, D, pr, 512)
    want.store(0, _np(k[0, :499]), _np(v[0, :499]))
    want.store(499, _np(k[0, 499:]), _np(v[0, 499:]))
    ko, vo = torch.zeros_like(k).float(), torch.zeros_like(v).float()
    p.read(ko, vo, _ids(1))
    for t, w in zip((ko, vo), want.values()):
        np.testing.assert_array_equal(_np(t[0]), w.astype(np.float32))
    q = _rand(1, 1, H, D, seed=3, dtype=BF)
    slots = p.select(q, 2, _ids(1), keep_last=1)
    np.testing.assert_array_equal(slots[0, 0].cpu().numpy(), o8.select(_np(q[0, 0]), want.mn, want.mx, want.scale[0], 500, pr, 2, 0, 1))
    out, lse = p.attn_blocks(q, slots, _ids(1), lse=True)
    K, V = want.values()
    _compare(BF, _np(out[0]), _np(lse[0]), o8.attention(_np(q[0]).astype(np.float64), K, V, _dense(500, 1, H, pr, slots[0].cpu().numpy()), 1 / math.sqrt(D)))
    assert p.status() == 0


# ------------------------------------------------------------------ chosen pages

def _slots_of(want, q, n, pr, n_slots, first, last):
    T = q.shape[0]
    return np.stack([o8.select(q[t], want.mn, want.mx, want.scale[0], n - (T - 1 - t), pr, n_slots, first, last) for t in range(T)])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,pr,H,rep,T,n_slots,first,last", [(128, 16, 2, 1, 1, 5, 1, 1), (128, 32, 1, 8, 2, 3, 0, 0), (128, 16, 1, 12, 1, 4, 0, 2),
                                                             (64, 16, 3, 3, 3, 6, 2, 4), (64, 48, 2, 5, 1, 1, 0, 1), (64, 16, 1, 20, 1, 7, 0, 0)])
def test_pages_are_chosen_and_attended_as_defined(D, pr, H, rep, T, n_slots, first, last, dtype):
    lens = [0, 1, 16, 17, 100, 333, 800]
    p, want = _filled(H, D, pr, lens, seed=31, dtype=dtype)
    q = _rand(len(lens), T, H * rep, D, seed=33, dtype=dtype, scale=2.0)
    slots = p.select(q, n_slots, keep_first=first, keep_last=last)
    out, lse = p.attn_blocks(q, slots, lse=True)
    assert p.status() == 0
    got = slots.cpu().numpy()
    for i, n in enumerate(lens):
        np.testing.assert_array_equal(got[i], _slots_of(want[i], _np(q[i]), n, pr, n_slots, first, last))
        K, V = want[i].values()
        _compare(dtype, _np(out[i]), _np(lse[i]), o8.attention(_np(q[i]).astype(np.float64), K, V, _dense(n, T, H, pr, got[i]), 1 / math.sqrt(D)))
    every = p.select(q, 64)
    all_out, all_lse = p.attn_blocks(q, every, lse=True)
    dense, dense_lse = p.attn(q, lse=True)
    for i, n in enumerate(lens):                                 # all pages: what attention over everything gives
        K, V = want[i].values()
        for o, s in ((all_out, all_lse), (dense, dense_lse)):
            _compare(dtype, _np(o[i]), _np(s[i]), o8.attention(_np(q[i]).astype(np.float64), K, V, _dense(n, T, H), 1 / math.sqrt(D)))


@pytest.mark.parametrize("n,n_lists", [(9000, 1), (20000, 2), (70000, 1)])
def test_selection_from_long_lists(n, n_lists):
    """Clusters of CTAs that share a list's scores, and one CTA that has more than a step of them."""
    H, D, pr, rep = 3, 64, 16, 4
    p, want = _filled(H, D, pr, [n] * n_lists, seed=41)
    for lists in ([0], list(range(n_lists)) * 20):
        q = _rand(len(lists), 1, H * rep, D, seed=len(lists), dtype=BF)
        slots = p.select(q, 100, _ids(*lists), keep_first=1, keep_last=3).cpu().numpy()
        for i in (0, len(lists) - 1):
            np.testing.assert_array_equal(slots[i], _slots_of(want[lists[i]], _np(q[i]), n, pr, 100, 1, 3))
    assert p.status() == 0


def test_ties_go_to_the_lower_page_and_nan_comes_first():
    H, D, pr = 1, 64, 16
    p = _pages(H, D, pr, 80, 2, 40)
    p.reserve(_ids(0, 1), 40 * 16)
    k = torch.ones(1, 16, 1, D, device=DEV).repeat(1, 40, 1, 1)
    k[0, 5 * 16:6 * 16], k[0, 9 * 16] = 2.0, 2.0
    p.write(k, k, _ids(0))
    q = torch.ones(1, 1, 2, D, dtype=BF, device=DEV)
    assert p.select(q, 6, _ids(0)).tolist() == [[[[0, 1, 2, 3, 5, 9]]]]
    assert p.select(q, 6, _ids(0), keep_last=2).tolist() == [[[[0, 1, 5, 9, 38, 39]]]]
    assert p.select(-q, 3, _ids(0)).tolist() == [[[[0, 1, 2]]]]          # 2 is the least now, and the rest is equal
    assert p.select(q * 0, 3, _ids(0), keep_first=1).tolist() == [[[[0, 1, 2]]]]
    k[0, 7 * 16 + 3, 0, 0], k[0, 30 * 16, 0, 1] = math.nan, math.inf
    p.write(k, k, _ids(1))
    assert p.select(q, 3, _ids(1)).tolist() == [[[[5, 7, 30]]]]
    assert p.select(q, 3, _ids(1), keep_last=2).tolist() == [[[[7, 38, 39]]]]
    q[0, 0, 0, 0] = math.nan                                             # every score is one
    assert p.select(q, 3, _ids(1)).tolist() == [[[[0, 1, 2]]]]
    assert p.status() == 0


def test_selection_and_attention_with_bad_lists_tables_and_slots():
    """Reported, and nothing but the page or entry concerned is affected."""
    H, D, pr = 2, 64, 16
    p, want = _filled(H, D, pr, [100, 100], seed=51)
    q = _rand(3, 1, 4, D, seed=52, dtype=BF)
    lists = _ids(0, 77, 1)
    slots = p.select(q, 3, lists)
    assert p.status() == pb.PYR_ERR_INVALID and (slots[1] == -1).all() and (slots[[0, 2]] >= 0).all()
    out = torch.full_like(q, 5.0)
    p.attn_blocks(q, slots, lists, out=out)
    assert p.status() == pb.PYR_ERR_INVALID and (out[1] == 5).all() and out[[0, 2]].isfinite().all()
    p.table[0, 2] = -5
    got = p.select(q[:1], 6, _ids(0)).cpu().numpy()[0, 0]
    assert p.status() == pb.PYR_ERR_INVALID and not (got == 2).any() and (got >= 0).all()
    K, V = want[0].values()
    # the caller's own slots: any order, -1 behind, one in no table, one out of range, one behind what the token sees
    mine = torch.tensor([[[[6, 0, 3, -1], [2, 1, 40, -7]]]], dtype=torch.int32, device=DEV)
    for slots, reported in ((mine, pb.PYR_ERR_INVALID), (mine.clamp(0, 6)[..., :1].contiguous(), pb.PYR_ERR_INVALID)):
        out, lse = p.attn_blocks(q[:1], slots, _ids(0), lse=True)
        assert p.status() == reported
        use = slots[0].cpu().numpy().copy()
        use[use == 2] = -1
        _compare(BF, _np(out[0]), _np(lse[0]), o8.attention(_np(q[0]).astype(np.float64), K, V, _dense(100, 1, H, pr, use), 1 / math.sqrt(D)))
    q2 = _rand(1, 5, 4, D, seed=53, dtype=BF)                            # of 5 tokens only the last sees a row of page 6
    six = torch.tensor([6, 1], dtype=torch.int32, device=DEV).expand(1, 5, 2, 2).contiguous()
    out, lse = p.attn_blocks(q2, six, _ids(1), lse=True)
    assert p.status() == 0
    K, V = want[1].values()
    _compare(BF, _np(out[0]), _np(lse[0]), o8.attention(_np(q2[0]).astype(np.float64), K, V, _dense(100, 5, H, pr, six[0].cpu().numpy()), 1 / math.sqrt(D)))
    none = torch.full((1, 1, H, 4), -1, dtype=torch.int32, device=DEV)
    out, lse = p.attn_blocks(q[:1], none, _ids(1), lse=True)
    assert p.status() == 0 and (out == 0).all() and torch.isneginf(lse).all()


# ------------------------------------------------------------------ together

def test_a_decode_step_is_captured_and_replayed_while_lists_grow():
    """Room, rows and queries turned and stored, pages chosen, attention over them and over all: one graph, replayed for every token, gives what
    eager calls on another handle give; on a stream of its own."""
    H, rep, D, pr, n = 2, 4, 128, 16, 3
    handles = [_filled(H, D, pr, [70, 5, 31], seed=61, spare=40)[0] for _ in range(2)]
    rope = pb.glue_rope_table(200, D)
    lists = _ids(2, 0, 1)
    k, v = torch.zeros(n, 1, H, D, dtype=BF, device=DEV), torch.zeros(n, 1, H, D, dtype=BF, device=DEV)
    q, qr = torch.zeros(n, 1, H * rep, D, dtype=BF, device=DEV), torch.zeros(n, 1, H * rep, D, dtype=BF, device=DEV)
    pos, slots = torch.zeros(n, 1, 1, dtype=torch.int32, device=DEV), torch.zeros(n, 1, H, 3, dtype=torch.int32, device=DEV)
    outs = [torch.zeros_like(q), torch.zeros_like(q)]

    def step(p, k, v, q, pos, qr, slots, outs):
        p.reserve(lists, 1)
        p.append(k, v, lists, pos=pos, rope=rope, q=q, q_out=qr)
        p.select(qr, 3, lists, keep_last=1, out=slots)
        p.attn_blocks(qr, slots, lists, out=outs[0])
        p.attn(qr, lists, out=outs[1])

    g, (graphed, eager) = torch.cuda.CUDAGraph(), handles
    state = _state(graphed)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(graphed, k, v, q, pos, qr, slots, outs)             # (a first call outside the capture)
    torch.cuda.current_stream().wait_stream(side)
    for t, o in zip((graphed.pool, graphed.table, graphed.lens, graphed.refs), state):
        t.copy_(o)
    with torch.cuda.graph(g):
        step(graphed, k, v, q, pos, qr, slots, outs)
    for t in range(38):
        for x, seed in ((k, 1), (v, 2), (q, 3)):
            x.copy_(_rand(*x.shape, seed=100 * t + seed, dtype=BF, scale=1 + t % 3))
        pos.copy_(torch.tensor([31, 70, 5], dtype=torch.int32).view(n, 1, 1) + t)
        g.replay()
        mine = [torch.zeros_like(x) for x in (qr, slots, *outs)]
        step(eager, k.clone(), v.clone(), q.clone(), pos.clone(), mine[0], mine[1], mine[2:])
        for a, b in zip((qr, slots, *outs), mine):
            assert torch.equal(a, b)
    assert eager.status() == 0 and graphed.status() == 0 and graphed.lens.tolist() == [108, 43, 69]
    assert all(torch.equal(a, b) for a, b in zip(_state(graphed)[1:], _state(eager)[1:]))


def test_calls_on_a_stream_of_the_callers():
    """Inputs and outputs used on the stream that is passed, results the same."""
    H, D, pr = 2, 128, 32
    p, _ = _filled(H, D, pr, [200], seed=71)
    q = _rand(1, 1, 8, D, seed=72, dtype=BF)
    want, ws = p.attn(q), p.select(q, 3)
    wb = p.attn_blocks(q, ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        slots = p.select(q, 3, stream=s)
        out, blocks = p.attn(q, stream=s), p.attn_blocks(q, slots, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want) and torch.equal(slots, ws) and torch.equal(blocks, wb)


def test_calls_that_a_format_does_not_have():
    p8, p4 = _pages(1, 64, 16, 4, 2, 2), pb.PyrPages(n_kv_heads=1, head_dim=64, n_pages=4, n_lists=2, max_pages=2)
    k = torch.zeros(1, 1, 1, 64, device=DEV)
    s = torch.zeros(1, 1, 1, 1, dtype=torch.int32, device=DEV)
    for call in (lambda: p8.compact(_ids(0), _ids(1), n_rows=1), lambda: p4.append(k, k), lambda: p4.select(k, 1), lambda: p4.attn_blocks(k, s)):
        with pytest.raises(pb.PyrError) as e:
            call()
        assert e.value.status == pb.PYR_ERR_UNSUPPORTED
    # no entries, no rows
    assert p8.attn(k[:0]).numel() == 0 and p8.select(k[:0], 2, _ids()).shape == (0, 1, 1, 2)
    p8.append(k[:0], k[:0], _ids())
    p8.append(k[:, :0], k[:, :0], _ids(0))
    assert p8.status() == 0 and p8.lens.tolist() == [0, 0]


def test_compiled_calls_and_the_binding_do_the_same():
    """The same arguments through both: results, errors, outputs that are passed in, empty and odd tensors."""
    H, D, pr = 2, 128, 16
    rope = pb.glue_rope_table(300, D)
    handles = [_filled(H, D, pr, [70, 5, 31], seed=91, spare=30)[0] for _ in range(2)]
    handles[1]._call = None
    assert handles[0]._call is not None
    got = []
    for p in handles:
        r = []
        k, v = _rand(3, 4, H, D, seed=1, dtype=BF), _rand(3, 4, H, D, seed=2, dtype=BF)
        q = _rand(3, 4, 3 * H, D, seed=3, dtype=BF)
        pos = (torch.arange(12, dtype=torch.int32, device=DEV) * 7).view(3, 1, 4)
        idx = torch.tensor([[[3, 1]], [[0, 0]], [[2, 3]]], dtype=torch.int32, device=DEV)
        r.append(p.append(k, v, _ids(2, 0, 1), pos=pos, rope=rope, q=q, counts=_ids(4, 3, 0)))
        out = torch.zeros_like(q)
        assert p.append(k, v, pos=pos, rope=rope, q=q, q_out=out) is out
        r.append(out)
        assert p.append(k, v, idx=idx, pos=pos[:, :, :2].contiguous(), rope=rope) is None
        assert p.append(k[:, :1], v[:, :1], first=_ids(3, 3, 3)) is None
        ko, vo = torch.zeros(3, 20, H, D, device=DEV), torch.zeros(3, 20, H, D, device=DEV)
        assert p.read(ko, vo, _ids(1, 0, 2), first=_ids(0, 60, 10), counts=_ids(20, 19, 1)) is None
        r += [ko, vo, *p.attn(q, lse=True), p.attn(q[:2], _ids(2, 1), out=out[:2], softmax_scale=1)]
        s = p.select(q, 3, _ids(0, 1, 2), keep_first=1)
        assert p.select(q, 3, out=s) is s
        r += [s, *p.attn_blocks(q, s, lse=True), p.attn_blocks(q[:, :1], s[:, :1].contiguous()), p.attn(q[:0], _ids())]
        for call in (lambda: p.attn(q, _ids(0)), lambda: p.attn(q.half()), lambda: p.attn(q, out=out.float()), lambda: p.select(q, 3, out=s[:1]),
                     lambda: p.attn_blocks(q, s.long()), lambda: p.append(k, v, pos=pos), lambda: p.append(k, v.float()), lambda: p.read(ko, vo[:, :3])):
            with pytest.raises(ValueError):
                call()
        for call in (lambda: p.attn(q[:, :, :3]), lambda: p.attn(q, softmax_scale=-1.0), lambda: p.select(q, 2, keep_first=1, keep_last=2), lambda: p.select(q, 0),
                     lambda: p.append(k.repeat(2, 1, 1, 1), v.repeat(2, 1, 1, 1)), lambda: p.read(ko[:, :1].expand(-1, 20, -1, -1), vo[:, :1].expand(-1, 20, -1, -1))):
            with pytest.raises(pb.PyrError):
                call()
        assert p.status() == 0
        got.append(r + [p.lens.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    p = handles[0]
    p.close()
    with pytest.raises(pb.PyrError):
        p.attn(_rand(3, 1, H, D, seed=1, dtype=BF))


@pytest.mark.parametrize("rows", [1, 19])
def test_more_entries_than_decide_for_themselves(rows):
    """640 ragged lists in one call, twice (the second in pages that hold rows already), queries beside them; a list twice and one that does not
    exist among them."""
    H, D, pr, hq, n, n_lists = 3, 64, 16, 5, 640, 700
    p = _pages(H, D, pr, 3 * n_lists, n_lists, 3)
    rope = pb.glue_rope_table(400, D)
    lists = [(i * 31) % n_lists for i in range(n)]
    lists[600] = lists[7]
    lists[77] = n_lists
    bad = {7, 600, 77}
    counts = [(i * 5) % (rows + 1) if i % 9 else rows for i in range(n)]
    p.reserve(torch.arange(n_lists, dtype=torch.int32, device=DEV), 40)
    assert p.status() == 0
    sample = [0, 1, 6, 76, 78, 333, 511, 512, 513, 599, 601, 639]
    want = {i: o8.List8(H, D, pr, 48) for i in sample}
    lens = [0] * n_lists
    for step in range(2):
        k, v = _rand(n, rows, H, D, seed=5 * step, dtype=BF, scale=1 + 3 * step), _rand(n, rows, H, D, seed=5 * step + 1, dtype=BF, scale=3 - 2 * step)
        q = _rand(n, rows, hq, D, seed=5 * step + 2, dtype=BF)
        pos = (torch.arange(n * rows, dtype=torch.int32, device=DEV) % 399 + step).view(n, 1, rows)
        out = p.append(k, v, _ids(*lists), pos=pos, rope=rope, q=q, counts=_ids(*counts))
        assert p.status() == pb.PYR_ERR_INVALID
        turned = torch.from_numpy(o8.rotate(_np(q), _np(rope)[pos.cpu().numpy()[:, 0]][:, :, None])).to(BF).float().numpy()
        for i in range(n):
            c = 0 if i in bad else counts[i]
            turned[i, c:] = _np(q[i, c:])
            if i not in bad:
                lens[lists[i]] += c
        np.testing.assert_array_equal(_np(out), turned)
        assert p.lens.tolist() == lens
        for i, w in want.items():
            c = counts[i]
            if c:
                w.store(w.len, o8.rotate(_np(k[i, :c]), _np(rope)[pos[i, 0, :c].cpu().numpy()][:, None]), _np(v[i, :c]))
                _check(p, lists[i], w)


def test_calls_under_inference_mode_and_beside_gradients():
    """A call asks for no gradient, whatever its tensors say, and gives the same in every mode."""
    H, D, pr = 2, 128, 16
    p, _ = _filled(H, D, pr, [100, 3], seed=95)
    q = _rand(2, 2, 4 * H, D, seed=96, dtype=BF)
    slots = p.select(q, 2)
    want = [*p.attn(q, lse=True), *p.attn_blocks(q, slots, lse=True), slots]
    leaf = q.clone().requires_grad_()
    got = [*p.attn(leaf, lse=True), *p.attn_blocks(leaf, p.select(leaf, 2), lse=True), p.select(leaf, 2)]
    assert not any(t.requires_grad for t in got) and all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.inference_mode():
        got = [*p.attn(q, lse=1), *p.attn_blocks(q, p.select(q, 2), lse=True), p.select(q, 2)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(RuntimeError):
        p.attn(q, lse=torch.zeros(2))                          # neither true nor false


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_chosen_pages_of_many_lists(D, dtype):
    """More work than a stage or two a warp, of every type: lists from none to 300 rows, two tokens each."""
    H, pr, rep, n, n_slots = 8, 16, 3, 70, 9
    lens = [(i * 53) % 301 if i % 11 else 0 for i in range(n)]
    p, want = _filled(H, D, pr, lens, seed=97, spare=2, dtype=dtype)
    q = _rand(n, 2, H * rep, D, seed=98, dtype=dtype)
    slots = p.select(q, n_slots, keep_last=1)
    out, lse = p.attn_blocks(q, slots, lse=True)
    sample = [0, 1, 2, 11, 33, 34, 69]
    _sampled(p, lambda l: want[l], out, lse, q, list(range(n)), rep, 2, dtype, sample, H, pr, slots)
    for i in sample:
        np.testing.assert_array_equal(slots[i].cpu().numpy(), _slots_of(want[i], _np(q[i]), lens[i], pr, n_slots, 0, 1))
    again, lse2 = p.attn_blocks(q, slots, lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2) and p.status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,n", [(64, 9000), (128, 9000), (64, 20000)])
def test_selection_with_one_query_head_a_kv_head(D, n, dtype):
    """Few and many entries over long lists: clusters of CTAs, one CTA, one warp a list; two tokens, which see different rows."""
    H, pr = 3, 16
    p, want = _filled(H, D, pr, [n, 700], seed=43, dtype=dtype)
    for count in (1, 20, 150, 600):
        lists = [1 if i % 5 == 4 else 0 for i in range(count)]
        q = _rand(count, 2, H, D, seed=count, dtype=dtype)
        slots = p.select(q, 40, _ids(*lists), keep_first=1, keep_last=3).cpu().numpy()
        for i in sorted({0, min(4, count - 1), count - 1}):
            l = lists[i]
            np.testing.assert_array_equal(slots[i], _slots_of(want[l], _np(q[i]), want[l].len, pr, 40, 1, 3))
    assert p.status() == 0


def test_ties_and_nan_with_one_query_head():
    H, D, pr = 1, 128, 16
    p = _pages(H, D, pr, 80, 2, 40)
    p.reserve(_ids(0, 1), 40 * 16)
    k = torch.ones(1, 16, 1, D, device=DEV).repeat(1, 40, 1, 1)
    k[0, 5 * 16:6 * 16], k[0, 9 * 16] = 2.0, 2.0
    p.write(k, k, _ids(0))
    q = torch.ones(1, 1, 1, D, dtype=BF, device=DEV)
    assert p.select(q, 6, _ids(0)).tolist() == [[[[0, 1, 2, 3, 5, 9]]]]
    assert p.select(-q, 3, _ids(0)).tolist() == [[[[0, 1, 2]]]]
    assert p.select(q * 0, 3, _ids(0), keep_first=1).tolist() == [[[[0, 1, 2]]]]
    k[0, 7 * 16 + 3, 0, 0], k[0, 30 * 16, 0, 1] = math.nan, math.inf
    p.write(k, k, _ids(1))
    assert p.select(q, 3, _ids(1), keep_last=1).tolist() == [[[[7, 30, 39]]]]
    q[0, 0, 0, 0] = math.nan
    assert p.select(q, 3, _ids(1)).tolist() == [[[[0, 1, 2]]]] and p.status() == 0
    p.table[1, 3] = 1 << 20                                              # a page out of range comes last
    q[0, 0, 0, 0] = 1
    assert p.select(q, 39, _ids(1)).tolist() == [[[[x for x in range(40) if x != 3]]]]
    assert p.status() == pb.PYR_ERR_INVALID
    assert p.select(q, 3, _ids(7)).tolist() == [[[[-1, -1, -1]]]] and p.status() == pb.PYR_ERR_INVALID
