"""The paged 4-bit cache on the GPU against its definition (oracle/pages.py): stored bytes, attention in fp64 over what the
bytes stand for, and the bookkeeping of pages."""
import numpy as np
import pytest
import torch

from oracle import pages as op
from paper_2405_12532_b200 import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda"
FORMATS = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]
BF, F32 = torch.bfloat16, torch.float32


def _ids(*x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def _wide(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _rand(*shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).to(DEV)


def _pages(hkv, D, group, page_rows, n_pages, n_lists, max_pages, poison=True):
    p = pb.PyrPages(n_kv_heads=hkv, head_dim=D, group=group, page_rows=page_rows, n_pages=n_pages, n_lists=n_lists, max_pages=max_pages)
    if poison:
        p.pool.fill_(0xFF)            # stale bytes: every scale and zero a NaN
    return p


def _book(p):
    b = op.Book(p.cfg.n_pages, p.cfg.n_lists, p.cfg.max_pages, p.cfg.page_rows)
    return b


def _same(p, b):
    assert p.status() == 0
    np.testing.assert_array_equal(p.table.cpu().numpy(), b.table)
    np.testing.assert_array_equal(p.lens.cpu().numpy(), b.lens)
    np.testing.assert_array_equal(p.refs.cpu().numpy(), b.refs)


def _state(p):
    return [t.clone() for t in (p.pool, p.table, p.lens, p.refs)]


def _unchanged(p, state):
    return all(torch.equal(a, b) for a, b in zip(_state(p), state))


def _list_values(p, l, length=None):
    c = p.cfg
    return op.list_values(p.pool.cpu().numpy(), p.table[l].cpu().numpy(), int(p.lens[l]) if length is None else length,
                          c.n_kv_heads, c.head_dim, c.group, c.page_rows)


def _quantised(x, group):
    """x [..., D] as the values its codes stand for, fp64."""
    return op.values(*op.quantise(x.detach().cpu().float().numpy(), group))


def _as(x, dtype):
    """fp64 -> fp32 -> dtype, the roundings that reading makes, as fp64."""
    return torch.from_numpy(x.astype(np.float32)).to(dtype).to(torch.float64).numpy()


# ------------------------------------------------------------------ store and read

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,group", FORMATS)
def test_write_stores_the_defined_codes_and_read_returns_their_values(D, group, dtype):
    hkv, pr, n, rows = 3, 32, 3, 45
    p = _pages(hkv, D, group, pr, 9, 4, 3)
    lists = _ids(2, 0, 3)
    p.reserve(lists, rows)
    k = _rand(n, rows, hkv, D, seed=1, dtype=dtype)
    v = _rand(n, rows, hkv, D, seed=2, dtype=dtype, scale=7.0)
    p.write(k, v, lists)
    assert p.status() == 0 and p.lens.tolist() == [rows, 0, rows, rows]
    kw, vw = _quantised(k, group), _quantised(v, group)
    ko, vo = torch.full_like(k, -9.0), torch.full_like(v, -9.0)
    p.read(ko, vo, lists)
    np.testing.assert_array_equal(_wide(ko), _as(kw, dtype))
    np.testing.assert_array_equal(_wide(vo), _as(vw, dtype))
    for i, l in enumerate(lists.tolist()):          # the bytes themselves, unpacked by the definition
        K, V = _list_values(p, l)
        np.testing.assert_array_equal(K, kw[i])
        np.testing.assert_array_equal(V, vw[i])


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_write_gathers_kept_rows_at_any_place_and_leaves_the_rest(dtype, groups):
    """Kept lists per sequence or per head, counts of their own (0 among them), first rows that end inside a tile, head-major
    source tensors, an index row longer than it needs to be: rows outside [first, first + count) keep their bytes."""
    hkv, D, group, pr, n, src = 4, 128, 64, 48, 4, 200
    rows = 61
    p = _pages(hkv, D, group, pr, 40, 6, 4)
    lists = _ids(5, 1, 2, 4)
    p.reserve(lists, 130)
    base_k, base_v = _rand(n, 70, hkv, D, seed=3, dtype=dtype), _rand(n, 70, hkv, D, seed=4, dtype=dtype)
    p.write(base_k, base_v, lists)
    k = _rand(n, hkv, src, D, seed=5, dtype=dtype).transpose(1, 2)            # [n, src, hkv, D], head-major
    v = _rand(n, hkv, src, D, seed=6, dtype=dtype).transpose(1, 2)
    g = torch.Generator().manual_seed(7)
    wide = torch.randint(0, src, (n, groups, rows), generator=g).to(torch.int32)
    idx = torch.cat([wide.flatten(1), torch.full((n, 5), -7, dtype=torch.int32)], 1).to(DEV)
    idx = torch.as_strided(idx, (n, groups, rows), (idx.shape[1], rows, 1))
    first, counts = [70, 3, 16, 69], [61, 29, 0, 1]
    before = [_list_values(p, l) for l in lists.tolist()]
    p.write(k, v, lists, first=_ids(*first), idx=idx, counts=_ids(*counts))
    assert p.status() == 0
    kq, vq = _quantised(k.contiguous(), group), _quantised(v.contiguous(), group)
    for i, l in enumerate(lists.tolist()):
        ln = max(70, first[i] + counts[i])
        assert int(p.lens[l]) == ln
        K, V = _list_values(p, l)
        wk, wv = np.zeros_like(K), np.zeros_like(V)
        wk[:70], wv[:70] = before[i]
        for h in range(hkv):
            rowsel = wide[i, h if groups == hkv else 0, :counts[i]].numpy()
            wk[first[i]:first[i] + counts[i], h] = kq[i, rowsel, h]
            wv[first[i]:first[i] + counts[i], h] = vq[i, rowsel, h]
        np.testing.assert_array_equal(K, wk)
        np.testing.assert_array_equal(V, wv)
    # reading from inside, with counts, into strided tensors: rows a list does not have stay as they are
    ko = torch.full((n, hkv, 40, D), -9.0, dtype=dtype, device=DEV).transpose(1, 2)
    vo = torch.full((n, hkv, 40, D), -9.0, dtype=dtype, device=DEV).transpose(1, 2)
    p.read(ko, vo, lists, first=_ids(100, 65, 40, 500), counts=_ids(40, 12, 0, 40))
    assert p.status() == 0
    for i, (f, c) in enumerate([(100, 40), (65, 12), (40, 0), (500, 40)]):
        K, V = _list_values(p, lists.tolist()[i])
        m = max(0, min(c, K.shape[0] - f))
        np.testing.assert_array_equal(_wide(ko[i, :m]), _as(K[f:f + m], dtype))
        np.testing.assert_array_equal(_wide(vo[i, :m]), _as(V[f:f + m], dtype))
        assert bool((ko[i, m:] == -9).all()) and bool((vo[i, m:] == -9).all())


def test_appending_single_rows_equals_writing_them_at_once():
    hkv, D, n, rows = 2, 128, 5, 50
    p, q = _pages(hkv, D, 64, 16, 30, n, 4), _pages(hkv, D, 64, 16, 30, n, 4)
    k, v = _rand(n, rows, hkv, D, seed=8, dtype=BF), _rand(n, rows, hkv, D, seed=9, dtype=BF)
    lists = _ids(*range(n))
    q.reserve(lists, rows)
    q.write(k, v)
    for t in range(rows):
        p.reserve(lists, 1)
        p.write(k[:, t:t + 1], v[:, t:t + 1])
    assert p.status() == 0 and q.status() == 0
    assert torch.equal(p.lens, q.lens)
    for l in range(n):
        for a, b in zip(_list_values(p, l), _list_values(q, l)):
            np.testing.assert_array_equal(a, b)


def test_values_that_cannot_be_quantised():
    """Constant groups come back exactly; an Inf, a NaN or a range beyond fp32 makes its group (and no other) NaN; rows with an
    offset much larger than their range, tiny rows and huge rows stay within half a step."""
    D, group = 128, 32
    p = _pages(1, D, group, 16, 2, 1, 2)
    x = torch.randn(12, 1, D, generator=torch.Generator().manual_seed(3))
    x[0] = 2.5
    x[1, 0, 5] = float("inf")
    x[2, 0, 40] = float("nan")
    x[3, 0, 70] = float("-inf")
    x[4, 0, 100] = -3.4e38
    x[5] = 1000 + 0.01 * x[5]
    x[6] *= 1e30
    x[7] *= 1e-25
    x[8] = 0.0
    x[9] = -0.0
    x[10] *= 1e-37
    k = x.unsqueeze(0).to(DEV)
    p.reserve(_ids(0), 12)
    p.write(k, -k)
    ko, vo = torch.zeros_like(k), torch.zeros_like(k)
    p.read(ko, vo)
    assert p.status() == 0
    np.testing.assert_array_equal(_wide(ko), _as(_quantised(k, group), F32))
    np.testing.assert_array_equal(_wide(vo), _as(_quantised(-k, group), F32))
    nan = torch.isnan(ko[0, :, 0]).view(12, 4, 32)
    assert [nan[r].any(-1).tolist() for r in range(1, 5)] == [[i == g for i in range(4)] for g in range(4)]
    assert bool(nan.any(-1).eq(nan.all(-1)).all()) and int(nan.any(-1).sum()) == 4
    assert bool((ko[0, 0] == 2.5).all()) and bool((ko[0, 8:10] == 0).all())


# ------------------------------------------------------------------ attention

def _fill(p, lens, seed, dtype=BF, kscale=1.0):
    """Lists 0 .. with the given lengths, written through the library in pages of shuffled order."""
    c = p.cfg
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(c.n_pages, generator=g)
    used = 0
    for l, ln in enumerate(lens):
        need = -(-ln // c.page_rows)
        p.table[l, :need] = order[used:used + need].to(torch.int32).to(DEV)
        p.refs[order[used:used + need].to(DEV)] = 1
        used += need
    m = max(max(lens), 1)
    k = _rand(len(lens), m, c.n_kv_heads, c.head_dim, seed=seed + 1, dtype=dtype, scale=kscale)
    k = k + _rand(1, 1, c.n_kv_heads, c.head_dim, seed=seed + 2, dtype=dtype)
    v = _rand(len(lens), m, c.n_kv_heads, c.head_dim, seed=seed + 3, dtype=dtype)
    p.write(k, v, counts=_ids(*lens))
    assert p.status() == 0


def _check_attn(p, q, lists, out, lse, scale):
    """Bounds derived term by term. Scores: products of a code, a query value and the row's (scale, zero), summed in fp32 - an
    error of at most (D + 8) 2^-23 times scale sum |q| (15 s + |zero|) - which moves a probability by that factor, as do the
    exponential (2^-21) and the fp32 sums (n 2^-23 with both sums). bf16: probabilities times scale are rounded to 8 bits
    or better before the product with the centred codes (|c - 8| <= 8), at most 2^-9 8 max(scale); the output is
    rounded once, 2^-9 |o|. lse: the scores' error and 2^-21 relative."""
    for i, l in enumerate(lists):
        K, V = _list_values(p, l)
        qw = _wide(q[i])
        want, wlse = op.attention(qw, K, V, scale)
        if K.shape[0] == 0:
            assert not _wide(out[i]).any()
            assert bool(torch.isneginf(lse[i]).all())
            continue
        n, D = K.shape[0], q.shape[3]
        rep = q.shape[2] // K.shape[1]
        big = 15 * (K.max(-1) - K.min(-1)) + np.abs(K).max(-1)                  # [n, Hkv], above 15 s + |zero|
        ds = (D + 8) * 2.0 ** -23 * scale * max(np.abs(qw[:, h * rep:(h + 1) * rep]).sum(-1).max() * big[:, h].max()
                                               for h in range(K.shape[1]))
        rel = 2 * ds + 2.0 ** -20 + n * 2.0 ** -22
        tol = rel * 2 * np.abs(V).max() * np.ones_like(want)
        if q.dtype == BF:
            step = (V.max() - V.min()) / 15 * (1 + 2.0 ** -6)
            tol += 2.0 ** -9 * 8 * step + 2.0 ** -9 * np.abs(want) * (1 + 2.0 ** -7)
        err = np.abs(_wide(out[i]) - want)
        assert (err <= tol).all(), f"list {l}: off by {err.max()} (bound there {tol.flat[err.argmax()]})"
        lerr = np.abs(lse[i].cpu().double().numpy() - wlse)
        seen = np.isfinite(wlse)
        assert np.array_equal(np.isneginf(lse[i].cpu().numpy()), ~seen)
        assert (lerr[seen] <= ds + 2.0 ** -21 * np.abs(wlse[seen]) + 2.0 ** -20 + n * 2.0 ** -23).all()


ATTN = [
    # D, group, page_rows, hq, hkv, q_len, lengths
    (128, 64, 64, 4, 4, 1, [1, 15, 16, 17, 64, 65, 200]),
    (128, 32, 32, 8, 2, 1, [100, 0, 33]),
    (128, 128, 16, 8, 1, 1, [77]),
    (64, 32, 16, 4, 4, 4, [0, 1, 3, 4, 5, 40]),
    (64, 64, 48, 6, 2, 2, [90, 2, 31]),
    (128, 64, 256, 5, 1, 3, [300, 10]),
    (128, 64, 64, 16, 1, 1, [500]),                # more query heads per KV head than a column group holds
    (128, 32, 64, 12, 4, 7, [70, 6, 129]),         # ragged column groups: 21 columns
    (128, 64, 64, 1, 1, 1, [5000]),                # one pair: split over many CTAs
    (128, 64, 16, 2, 2, 1, [1] * 300),             # more lists than a block has threads
    (64, 32, 16, 8, 2, 1, [2000, 0, 1, 999, 31]),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,group,page_rows,hq,hkv,q_len,lens", ATTN)
def test_attention_against_fp64(D, group, page_rows, hq, hkv, q_len, lens, dtype):
    slots = max(1, -(-max(lens) // page_rows))
    p = _pages(hkv, D, group, page_rows, sum(-(-x // page_rows) for x in lens) + 2, len(lens), slots)
    _fill(p, lens, seed=D + group, dtype=dtype)
    q = _rand(len(lens), q_len, hq, D, seed=5, dtype=dtype)
    state = _state(p)
    out, lse = p.attn(q, lse=True)
    again, lse2 = p.attn(q, lse=True)
    assert p.status() == 0
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert _unchanged(p, state)
    _check_attn(p, q, range(len(lens)), out, lse, D ** -0.5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[1408, 1, 0, 700], [1409, 1, 0, 700], [176, 176, 1408, 177], [16 * 8 * 11 - 1] * 3])
@pytest.mark.parametrize("entries", [4, 18, 19, 37, 38, 74])
def test_attention_on_both_sides_of_the_rules_that_deal_out_the_work(entries, lens, dtype):
    """About as many (entry, head, column group)s as a B200 has SMs (148), and lists about as long as a CTA takes whole; some
    entries name no list, and lists repeat."""
    hkv, hq, D, T = 4, 12, 64, 3                    # 9 columns: 2 groups (bf16), 3 (fp32)
    p = _pages(hkv, D, 32, 64, sum(-(-x // 64) for x in lens), len(lens), 23)
    _fill(p, lens, seed=26, dtype=dtype)
    q = _rand(entries, T, hq, D, seed=27, dtype=dtype)
    lists = [(7 * i) % len(lens) for i in range(entries)]
    named = list(lists)
    for i in range(3, entries, 16):
        named[i] = -1 if i % 32 == 3 else len(lens)
    out = torch.full_like(q, -5.0)
    got, lse = p.attn(q, _ids(*named), out=out, lse=True)
    assert p.status() == (pb.PYR_ERR_INVALID if named != lists else 0)
    first = {}
    for i in range(entries):
        if named[i] != lists[i]:
            assert bool((out[i] == -5).all())
        else:
            first.setdefault(lists[i], []).append(i)
    for l, at in first.items():
        at = sorted({at[0], at[len(at) // 2], at[-1]})
        _check_attn(p, q[at], [l] * len(at), out[at], lse[at], D ** -0.5)


@pytest.mark.parametrize("hq,q_len", [(2, 2), (4, 1), (2, 1), (6, 1)])
@pytest.mark.parametrize("D,group", FORMATS)
def test_fp32_attention_with_one_two_and_more_columns(D, group, hq, q_len):
    lens = [70, 3, 1, 0, 200]
    p = _pages(2, D, group, 32, 16, 5, 7)
    _fill(p, lens, seed=24, dtype=F32)
    q = _rand(5, q_len, hq, D, seed=25)
    out, lse = p.attn(q, lse=True)
    assert p.status() == 0
    _check_attn(p, q, range(5), out, lse, D ** -0.5)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_strides_lists_scale(dtype):
    """Lists in any order and more than once, token-major and head-major tensors, a scale of the caller's, scores that are far
    apart (a few rows take nearly all the weight), no lse."""
    hkv, hq, D, T = 2, 6, 128, 3
    lens = [150, 31, 64]
    p = _pages(hkv, D, 64, 32, 12, 3, 5)
    _fill(p, lens, seed=20, dtype=dtype, kscale=6.0)
    lists = [2, 0, 0, 1, 2]
    q = _rand(5, hq, T, D, seed=21, dtype=dtype, scale=2.0).transpose(1, 2)
    room = torch.full((5, T, hq, 2 * D), -9.0, dtype=dtype, device=DEV)
    out = room[..., :D]
    got, lse = p.attn(q, _ids(*lists), out=out, lse=True, softmax_scale=0.3)
    assert got is out
    _check_attn(p, q, lists, out, lse, 0.3)
    assert bool((room[..., D:] == -9).all())
    assert torch.equal(p.attn(q, _ids(*lists), softmax_scale=0.3), out)
    assert p.status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_shows_nan_rows_where_they_are_seen(dtype):
    """A row whose key group is NaN shows in its head's outputs, in no other head, and not in tokens that do not see it."""
    p = _pages(2, 128, 64, 16, 8, 2, 4)
    k, v = _rand(2, 40, 2, 128, seed=30, dtype=dtype), _rand(2, 40, 2, 128, seed=31, dtype=dtype)
    k[0, 39, 1, 7] = float("nan")
    p.reserve(_ids(0, 1), 40)
    p.write(k, v)
    q = _rand(2, 2, 4, 128, seed=32, dtype=dtype)
    out, lse = p.attn(q, lse=True)
    bad = torch.isnan(out).any(-1)
    want = torch.zeros(2, 2, 4, dtype=torch.bool)
    want[0, 1, 2:] = True                       # the second token sees row 39, the first does not; query heads 2, 3 share KV head 1
    assert torch.equal(bad.cpu(), want) and torch.equal(torch.isnan(lse).cpu(), want.transpose(1, 2))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_keeps_nan_values_from_tokens_that_do_not_see_them(dtype):
    """A NaN group of V in the last row: NaN in that group's dimensions for the token that sees the row, nothing elsewhere - also
    not through a probability of zero times NaN. Stale bytes behind a list's end (NaN scales) never count."""
    p = _pages(1, 128, 32, 16, 8, 2, 4)
    k, v = _rand(2, 37, 1, 128, seed=33, dtype=dtype), _rand(2, 37, 1, 128, seed=34, dtype=dtype)
    v[0, 36, 0, 70] = float("inf")
    p.reserve(_ids(0, 1), 37)
    p.write(k, v)
    q = _rand(2, 3, 5, 128, seed=35, dtype=dtype)
    out, lse = p.attn(q, lse=True)
    want = torch.zeros(2, 3, 5, 128, dtype=torch.bool)
    want[0, 2, :, 64:96] = True
    assert torch.equal(torch.isnan(out).cpu(), want) and not bool(torch.isnan(lse).any())
    clean = v.clone()
    clean[0, 36] = 0
    p.write(k, clean, first=_ids(0, 0))
    ref = p.attn(q)
    assert torch.equal(ref[0, :2], out[0, :2]) and torch.equal(ref[1], out[1]) and p.status() == 0


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("D,group", FORMATS)
def test_attention_over_scales_of_many_magnitudes(D, group, order):
    """bf16: values whose scales run from 2^-90 to 2^90 down or up the list, group by group in other steps, and queries from
    2^-60 to 2^60 against keys that make up for it: every dimension is held to the largest value that its group has."""
    n, T = 96, 2
    p = _pages(1, D, group, 32, 4, 1, 3)
    k, v = _rand(1, n, 1, D, seed=36), _rand(1, n, 1, D, seed=37)
    row = torch.arange(n, device=DEV).view(1, n, 1, 1) if order > 0 else torch.arange(n - 1, -1, -1, device=DEV).view(1, n, 1, 1)
    step = torch.arange(D // group, device=DEV).repeat_interleave(group).view(1, 1, 1, D) + 1
    v = (v * torch.exp2(((row // 16) * 12 - 36) * step.float() * (2.5 / (D // group)))).to(BF)
    k = (k * 2.0 ** -20).to(BF)
    p.reserve(_ids(0), n)
    p.write(k, v)
    q = (_rand(1, T, 8, D, seed=38) * 2.0 ** 20).to(BF)
    out, lse = p.attn(q, lse=True)
    assert p.status() == 0
    K, V = _list_values(p, 0)
    want, wl = op.attention(_wide(q[0]), K, V, D ** -0.5)
    # P in f16 relative to the group's largest scale met: 2^-11 of a term, or 2^-25 of the largest; output 2^-9
    big = np.abs(V).reshape(n, 1, D // group, group).max((0, 1, 3)).repeat(group)
    err = np.abs(_wide(out[0]) - want)
    assert (err <= (2.0 ** -9 + 1e-4) * np.abs(want) + 2.0 ** -10 * big).all()
    assert np.abs(lse[0].cpu().double().numpy() - wl).max() <= 2e-4


def test_attention_over_many_rows_a_warp():
    """64 lists of 16384 rows (the same pages, queries of their own): each warp sums over thousands of rows of one head, whose
    codes all have the same sign."""
    n, rows, hkv, D = 64, 16384, 4, 128
    p = _pages(hkv, D, 64, 256, 64, n, 64)
    k, v = _rand(1, rows, hkv, D, seed=44, dtype=BF, scale=0.2), _rand(1, rows, hkv, D, seed=45, dtype=BF)
    p.reserve(_ids(0), rows)
    p.write(k, v, _ids(0))
    p.table.copy_(p.table[:1].expand(n, -1).clone())
    p.lens.fill_(rows)
    q = _rand(n, 1, hkv, D, seed=46, dtype=BF)
    out, lse = p.attn(q, lse=True)
    assert p.status() == 0
    kd = torch.from_numpy(_quantised(k[0], 64)).to(DEV)
    vd = torch.from_numpy(_quantised(v[0], 64)).to(DEV)
    z = torch.einsum("nhd,rhd->nhr", q[:, 0].double(), kd) * D ** -0.5
    want = torch.einsum("nhr,rhd->nhd", torch.softmax(z, -1), vd)
    err = (out[:, 0].double() - want).abs()
    # P in f16 (2^-12 of a term, sums of 16384 of them about 2^-12 15 step / 128), the output's rounding, the sums' truncation
    # (64 steps of 2^-24 relative to 15 steps of the scale)
    step = (vd.max() - vd.min()) / 15
    assert bool((err <= 2.0 ** -9 * want.abs() + 15 * step * (2.0 ** -12 / 128 * 8 + 64 * 2.0 ** -24)).all())
    assert float((lse[:, :, 0].double() - torch.logsumexp(z, -1)).abs().max()) <= 1e-5


def test_attention_with_queries_and_values_near_the_ends_of_their_range():
    """Queries of 2^100 against keys of 2^-100, and the other way round; values of 2^120 and 2^-90."""
    p = _pages(1, 128, 32, 16, 8, 4, 2)
    k, v = _rand(4, 30, 1, 128, seed=47), _rand(4, 30, 1, 128, seed=48)
    e = torch.tensor([-100.0, 90.0, 0.0, 0.0], device=DEV).view(4, 1, 1, 1)
    w = torch.tensor([0.0, 0.0, 120.0, -90.0], device=DEV).view(4, 1, 1, 1)
    k, v = (k * torch.exp2(e)).to(BF), (v * torch.exp2(w)).to(BF)
    p.reserve(_ids(0, 1, 2, 3), 30)
    p.write(k, v)
    q = (_rand(4, 1, 3, 128, seed=49) * torch.exp2(-e)).to(BF)
    out, lse = p.attn(q, lse=True)
    assert p.status() == 0
    for i in range(4):
        K, V = _list_values(p, i)
        want, wl = op.attention(_wide(q[i]), K, V, 128 ** -0.5)
        tol = 2.0 ** -9 * np.abs(want) + 2.0 ** -10 * np.abs(V).max()
        assert (np.abs(_wide(out[i]) - want) <= tol).all(), i
        assert np.abs(lse[i].cpu().double().numpy() - wl).max() <= 1e-4, i


def test_attention_far_into_a_pool_beyond_four_gigabytes():
    """Pages whose byte offsets pass 2^32, written, attended, moved and read back."""
    hkv, D, pr = 32, 128, 64
    page = hkv * 4 * op.tile_bytes(D, 64)
    n_pages = (5 << 30) // page
    p = _pages(hkv, D, 64, pr, n_pages, 2, 2, poison=False)
    p.pool[-6:].fill_(0xFF)
    p.refs[:n_pages - 4] = 1
    p.reserve(_ids(0, 1), 70)
    assert p.table.tolist() == [[n_pages - 4, n_pages - 3], [n_pages - 2, n_pages - 1]]
    k, v = _rand(2, 70, hkv, D, seed=40, dtype=BF), _rand(2, 70, hkv, D, seed=41, dtype=BF)
    p.write(k[:1], v[:1], _ids(0))
    p.compact(_ids(0), _ids(1), n_rows=70)
    ko, vo = torch.zeros_like(k[:1]), torch.zeros_like(v[:1])
    p.read(ko, vo, _ids(1))
    assert p.status() == 0
    np.testing.assert_array_equal(_wide(ko), _as(_quantised(k[:1], 64), BF))
    np.testing.assert_array_equal(_wide(vo), _as(_quantised(v[:1], 64), BF))
    q = _rand(1, 1, hkv, D, seed=42, dtype=BF)
    out, lse = p.attn(q, _ids(1), lse=True)
    kd, vd = _quantised(k[0], 64), _quantised(v[0], 64)
    want, wl = op.attention(_wide(q[0]), kd, vd, D ** -0.5)
    assert np.abs(_wide(out[0]) - want).max() <= 2.0 ** -8 * 8 * 0.5 + 2.0 ** -8 * np.abs(want).max()
    assert np.abs(lse[0].cpu().double().numpy() - wl).max() <= 1e-4


# ------------------------------------------------------------------ pages

def test_reserve_fork_trim_against_the_book():
    """A few hundred random calls, valid ones and refused ones, against plain bookkeeping; copied pages carry the filled rows and
    leave the rest."""
    rng = np.random.default_rng(5)
    n_pages, n_lists, slots, pr, hkv, D = 60, 14, 6, 32, 2, 64
    p = _pages(hkv, D, 32, pr, n_pages, n_lists, slots)
    b = _book(p)
    stamp = 0
    for step in range(250):
        n = int(rng.integers(1, 6))
        what = rng.integers(0, 4)
        if what == 0:
            lists = rng.choice(n_lists, n, replace=bool(rng.random() < 0.2)).tolist()
            rows = rng.integers(0, 90, n).tolist()
            before = _state(p)
            want = b.reserve(lists, rows)
            p.reserve(_ids(*lists), _ids(*rows))
            if want is None:
                assert p.status() in (pb.PYR_ERR_INVALID, pb.PYR_ERR_CAPACITY)
                assert _unchanged(p, before)
            else:
                _same(p, b)
                pool = before[0].clone()
                tb = op.tile_bytes(D, 32)
                for old, new, filled in want:
                    a = pool.view(n_pages, hkv, pr // 16, tb)
                    whole, left = divmod(filled, 16)
                    a[new, :, :whole] = a[old, :, :whole]
                    for off, unit in ((0, 32), (512, 32), (1024, 8), (1152, 8)):
                        if left:
                            a[new, :, whole, off:off + left * unit] = a[old, :, whole, off:off + left * unit]
                assert torch.equal(p.pool, pool)
                # fill what was reserved with a stamp of its own and let the lists grow
                for l, r in zip(lists, rows):
                    if r:
                        stamp += 1
                        b.lens[l] += r
                        x = torch.full((1, r, hkv, D), float(stamp), device=DEV)
                        p.write(x, x, _ids(l))
        elif what == 1:
            src = rng.integers(0, n_lists, n).tolist()
            dst = rng.integers(0, n_lists, n).tolist()
            done = b.fork(src, dst)
            p.fork(_ids(*src), _ids(*dst))
            if not all(done):
                assert p.status() == pb.PYR_ERR_INVALID
        else:
            lists = rng.integers(0, n_lists, n).tolist()
            rows = rng.integers(0, 120, n).tolist() if what == 2 else [0] * n
            b.trim(lists, rows)
            p.trim(_ids(*lists), _ids(*rows) if what == 2 else None)
        _same(p, b)
    held = torch.zeros_like(p.refs)
    t = p.table[p.table >= 0].long()
    held.index_add_(0, t, torch.ones_like(t, dtype=torch.int32))
    assert torch.equal(held, p.refs)


def test_reserve_over_many_slices_and_lists():
    """A pool of several scan slices (some full, some empty) and more lists than a block has threads: the lowest free pages, in
    order."""
    n_pages, n_lists, slots = 20000, 2500, 4
    p = _pages(1, 64, 64, 16, n_pages, n_lists, slots, poison=False)
    rng = np.random.default_rng(6)
    taken = rng.random(n_pages) < 0.6
    taken[4096:8192], taken[8192:12288] = True, False
    p.refs.copy_(torch.from_numpy(taken.astype(np.int32)))
    b = _book(p)
    b.refs[:] = taken
    lists = rng.permutation(n_lists)
    rows = rng.integers(0, 50, n_lists)
    assert b.reserve(lists.tolist(), rows.tolist()) == []
    p.reserve(_ids(*lists), _ids(*rows))
    _same(p, b)
    state = _state(p)
    p.reserve(_ids(*lists), 64 - 50 + 40)              # some list would outgrow its table
    assert p.status() == pb.PYR_ERR_CAPACITY and _unchanged(p, state)


def test_a_fork_diverges_when_it_is_extended():
    """Forks share every page until one of them is extended; then the part-filled last page is copied, the full ones stay
    shared, and neither sees the other's rows."""
    hkv, D, pr = 2, 128, 32
    p = _pages(hkv, D, 64, pr, 12, 4, 4)
    k, v = _rand(1, 70, hkv, D, seed=50, dtype=BF), _rand(1, 70, hkv, D, seed=51, dtype=BF)
    p.reserve(_ids(0), 70)
    p.write(k, v, _ids(0))
    p.fork(_ids(0, 0), _ids(1, 3))
    assert p.refs.tolist()[:3] == [3, 3, 3]
    x = _rand(3, 1, hkv, D, seed=52, dtype=BF)
    state = _state(p)
    p.write(x, x, _ids(0, 1, 3))                      # shared pages must not be written
    assert p.status() == pb.PYR_ERR_INVALID and _unchanged(p, state)
    p.reserve(_ids(0, 1, 3), 1)
    p.write(x, x, _ids(0, 1, 3))
    assert p.status() == 0
    assert p.table[[0, 1, 3], :3].tolist() == [[0, 1, 3], [0, 1, 4], [0, 1, 5]] and p.refs.tolist()[:6] == [3, 3, 0, 1, 1, 1]
    kq, vq, xq = _quantised(k, 64)[0], _quantised(v, 64)[0], _quantised(x, 64)
    for i, l in enumerate((0, 1, 3)):
        K, V = _list_values(p, l)
        np.testing.assert_array_equal(K, np.concatenate([kq, xq[i]]))
        np.testing.assert_array_equal(V, np.concatenate([vq, xq[i]]))


@pytest.mark.parametrize("D,group", FORMATS)
@pytest.mark.parametrize("groups", [1, 3])
def test_compact_in_place_and_into_another_list(D, group, groups):
    hkv, pr, n, rows = 3, 32, 3, 150
    p = _pages(hkv, D, group, pr, 40, 2 * n, 5)
    b = _book(p)
    src, dst = _ids(*range(n)), _ids(*range(n, 2 * n))
    p.reserve(src, rows)
    k, v = _rand(n, rows, hkv, D, seed=60), _rand(n, rows, hkv, D, seed=61)
    p.write(k, v, src)
    kq, vq = _quantised(k, group), _quantised(v, group)
    counts = [71, 0, 33]
    g = torch.Generator().manual_seed(62)
    keep = torch.stack([torch.stack([torch.sort(torch.randperm(rows, generator=g)[:71]).values for _ in range(groups)]) for _ in range(n)])
    anyorder = torch.randint(0, rows, (n, groups, 71), generator=g).to(torch.int32)
    p.reserve(dst, 100)
    pool = p.pool.clone()
    p.compact(src, dst, idx=anyorder.to(DEV), counts=_ids(*counts))
    assert p.status() == 0 and p.lens.tolist() == [rows] * 3 + counts

    def check(l, i, sel):
        K, V = _list_values(p, l)
        for h in range(hkv):
            s = sel[i, h if groups == hkv else 0, :counts[i]].numpy()
            np.testing.assert_array_equal(K[:, h], kq[i, s, h])
            np.testing.assert_array_equal(V[:, h], vq[i, s, h])

    for i in range(n):
        check(n + i, i, anyorder)
        # rows behind the moved ones keep their bytes, the source is as it was
        tail = slice((counts[i] + pr - 1) // pr, None)
        for page in p.table[n + i][tail].tolist() + p.table[i].tolist():
            if page >= 0:
                assert torch.equal(p.pool[page], pool[page])
    p.compact(src, src, idx=keep.to(torch.int32).to(DEV), counts=_ids(*counts))
    assert p.status() == 0 and p.lens.tolist() == counts + counts
    for i in range(n):
        check(i, i, keep)
    want = [-(-c // pr) for c in counts]
    assert (p.table[:n] >= 0).sum(1).tolist() == want
    held = torch.zeros_like(p.refs)
    t = p.table[p.table >= 0].long()
    held.index_add_(0, t, torch.ones_like(t, dtype=torch.int32))
    assert torch.equal(held, p.refs)
    del b


def test_compact_in_place_keeps_a_shared_prefix_shared():
    """Rows that stay where they are do not need pages of their own; rows that move do."""
    p = _pages(1, 64, 64, 16, 12, 3, 5)
    k, v = _rand(1, 64, 1, 64, seed=70), _rand(1, 64, 1, 64, seed=71)
    p.reserve(_ids(0), 64)
    p.write(k, v, _ids(0))
    p.fork(_ids(0), _ids(1))
    p.trim(_ids(1), _ids(32))
    prefix = list(range(32)) + [40, 41, 63]
    state = _state(p)
    bad = list(range(20)) + [30, 40, 63]               # moves a row inside a shared page
    p.compact(_ids(0), _ids(0), idx=_ids(*bad).view(1, 1, -1))
    assert p.status() == pb.PYR_ERR_INVALID and _unchanged(p, state)
    p.compact(_ids(0), _ids(0), idx=_ids(*prefix).view(1, 1, -1))
    assert p.status() == 0 and p.lens.tolist() == [35, 32, 0]
    kq, vq = _quantised(k, 64)[0], _quantised(v, 64)[0]
    K, V = _list_values(p, 0)
    np.testing.assert_array_equal(K, kq[prefix])
    np.testing.assert_array_equal(V, vq[prefix])
    K, V = _list_values(p, 1)
    np.testing.assert_array_equal(K, kq[:32])
    assert p.refs.tolist()[:4] == [2, 2, 1, 0]


def test_compact_of_nothing_and_of_many_entries_at_once():
    """No rows, a copy of a list to itself, and calls whose entries are partly in place, partly not, partly refused: every entry
    is finished by itself, and the counters are left as the next call needs them."""
    n, hkv, D, pr = 6, 3, 64, 16
    p = _pages(hkv, D, 32, pr, 80, 2 * n, 8)
    k, v = _rand(n, 100, hkv, D, seed=75), _rand(n, 100, hkv, D, seed=76)
    src = _ids(*range(n))
    p.reserve(src, 100)
    p.write(k, v, src)
    p.reserve(_ids(6, 7, 8), 40)
    kq = _quantised(k, 32)
    idx = torch.stack([torch.arange(i, 100, 2 + i % 2)[:30] for i in range(n)]).to(torch.int32).view(n, 1, 30).to(DEV)
    for _ in range(2):
        dst = _ids(6, 1, 7, 3, 9, 8)                   # 1 and 3 in place; 9 has no pages
        if _ == 0:
            p.compact(src, dst, idx=idx)
            assert p.status() == pb.PYR_ERR_INVALID
            assert p.lens.tolist() == [100, 30, 100, 30, 100, 100, 30, 30, 30, 0, 0, 0]
        else:                                          # again: the refused entry given pages, the others as they are by now
            p.reserve(_ids(9), 30)
            p.compact(_ids(0, 2, 4, 5), _ids(6, 7, 9, 8), idx=idx[[0, 2, 4, 5]].contiguous())
            assert p.status() == 0 and p.lens.tolist() == [100, 30, 100, 30, 100, 100, 30, 30, 30, 30, 0, 0]
        for i, l in enumerate(dst.tolist()):
            if _ == 0 and l == 9:
                continue
            np.testing.assert_array_equal(_list_values(p, l)[0], kq[i, idx[i, 0].cpu().numpy()])
    p.compact(_ids(0), _ids(0), n_rows=50)             # a list's own first rows: only the length and the pages change
    assert p.status() == 0 and int(p.lens[0]) == 50 and int((p.table[0] >= 0).sum()) == 4
    two = _ids(2, 4)
    p.compact(two, two, n_rows=17)
    p.compact(_ids(5), _ids(6), n_rows=0)
    assert p.status() == 0 and p.lens[[2, 4, 6]].tolist() == [17, 17, 0]
    np.testing.assert_array_equal(_list_values(p, 2)[0], kq[2, :17])
    held = torch.zeros_like(p.refs)
    t = p.table[p.table >= 0].long()
    held.index_add_(0, t, torch.ones_like(t, dtype=torch.int32))
    assert torch.equal(held, p.refs)


# ------------------------------------------------------------------ refusals

def test_refused_entries_change_nothing_and_are_reported():
    hkv, D, pr = 2, 64, 16
    p = _pages(hkv, D, 32, pr, 20, 5, 4)
    x = _rand(2, 20, hkv, D, seed=80)
    p.reserve(_ids(0, 1), 20)
    p.write(x, x, _ids(0, 1))
    p.fork(_ids(1), _ids(3))
    p.reserve(_ids(4), 40)
    assert p.status() == 0
    state = _state(p)
    y = _rand(2, 3, hkv, D, seed=81)
    out = torch.full((2, 1, hkv, D), -9.0, device=DEV)
    calls = [
        lambda: p.write(y, y, _ids(7, -1)),                                        # list ids out of range
        lambda: p.write(y, y, _ids(0, 0)),                                         # one list twice
        lambda: p.write(y, y, _ids(2, 1)),                                         # no page / a shared page
        lambda: p.write(y, y, _ids(0, 4), first=_ids(21, -1)),                     # behind the end / negative
        lambda: p.write(y, y, _ids(0, 4), counts=_ids(4, -1)),                     # more than there are / negative
        lambda: p.write(torch.cat([x, x, x], 1)[:1], torch.cat([x, x, x], 1)[:1], _ids(0)),      # beyond the table
        lambda: p.read(out, out, _ids(5, -3)),
        lambda: p.read(out, out, _ids(0, 1), first=_ids(-1, -2)),
        lambda: p.read(out, out, _ids(0, 1), counts=_ids(2, -2)),
        lambda: p.attn(torch.zeros(2, 1, hkv, D, device=DEV), _ids(9, -2), out=out),
        lambda: p.fork(_ids(0), _ids(0)),
        lambda: p.fork(_ids(0, 0), _ids(2, 2)),                                    # one destination twice
        lambda: p.fork(_ids(0, 2), _ids(2, 4)),                                    # a destination that is a source; one with pages
        lambda: p.fork(_ids(9, 0), _ids(2, 9)),
        lambda: p.trim(_ids(0, 5), _ids(-1, 3)),
        lambda: p.compact(_ids(0), _ids(2), n_rows=10),                            # no pages
        lambda: p.compact(_ids(0), _ids(3), n_rows=10),                            # shared pages
        lambda: p.compact(_ids(0, 1), _ids(4, 4), n_rows=10),                      # one destination twice
        lambda: p.compact(_ids(0), _ids(4), n_rows=21),                            # more rows than the source has
        lambda: p.compact(_ids(0), _ids(4), idx=_ids(3, 20).view(1, 1, 2)),        # a row that is not there
        lambda: p.compact(_ids(0), _ids(4), idx=_ids(3, -1).view(1, 1, 2)),
        lambda: p.compact(_ids(0), _ids(0), idx=_ids(3, 3).view(1, 1, 2)),         # in place: not ascending
        lambda: p.compact(_ids(0), _ids(4), idx=_ids(3, 4).view(1, 1, 2), counts=_ids(3)),
        lambda: p.compact(_ids(8), _ids(4), n_rows=1),
        lambda: p.reserve(_ids(0, 0), 1),
        lambda: p.reserve(_ids(0, 12), 1),
        lambda: p.reserve(_ids(0, 4), _ids(1, -1)),
    ]
    for i, call in enumerate(calls):
        call()
        assert p.status() == pb.PYR_ERR_INVALID, i
        assert p.status() == 0, i
        assert _unchanged(p, state), i
        assert bool((out == -9).all()), i
    p.reserve(_ids(0, 2), 60)
    assert p.status() == pb.PYR_ERR_CAPACITY and _unchanged(p, state)
    # one bad entry does not keep the others from being served
    p.write(y, y, _ids(9, 0))
    assert p.status() == pb.PYR_ERR_INVALID and p.lens.tolist() == [23, 20, 0, 20, 0]


def test_kept_rows_out_of_range_are_stored_as_nan():
    p = _pages(1, 64, 64, 16, 2, 1, 1)
    x = _rand(1, 5, 1, 64, seed=85)
    p.reserve(_ids(0), 3)
    p.write(x, x, idx=_ids(2, 5, -1).view(1, 1, 3))
    assert p.status() == pb.PYR_ERR_INVALID and p.lens.tolist() == [3]
    ko, vo = torch.zeros(1, 3, 1, 64, device=DEV), torch.zeros(1, 3, 1, 64, device=DEV)
    p.read(ko, vo)
    assert torch.isnan(ko).any(-1).flatten().tolist() == [False, True, True] and torch.isnan(vo[0, 1:]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_out_of_range_in_a_table_are_not_followed(dtype):
    """Rows in pages that the table does not name properly take no part in attention, are not read, and are reported."""
    p = _pages(2, 128, 64, 16, 6, 1, 4)
    k, v = _rand(1, 50, 2, 128, seed=86, dtype=dtype), _rand(1, 50, 2, 128, seed=87, dtype=dtype)
    p.reserve(_ids(0), 50)
    p.write(k, v)
    K, V = _list_values(p, 0)
    p.table[0, 1] = 6
    p.table[0, 2] = -5
    q = _rand(1, 1, 2, 128, seed=88, dtype=dtype)
    out = p.attn(q)
    assert p.status() == pb.PYR_ERR_INVALID
    rows = list(range(16)) + [48, 49]
    want, _ = op.attention(_wide(q[0]), K[rows], V[rows], 128 ** -0.5)
    assert np.abs(_wide(out[0]) - want).max() <= 2.0 ** -8 * (np.abs(V).max() + 4 * (V.max() - V.min()) / 15)
    ko, vo = torch.full_like(k, -9.0), torch.full_like(v, -9.0)
    p.read(ko, vo)
    assert p.status() == pb.PYR_ERR_INVALID
    assert bool((ko[0, 16:48] == -9).all()) and bool((ko[0, 48:] != -9).any())


def test_binding_refuses_what_it_can_see():
    p = _pages(2, 64, 32, 16, 4, 2, 2)
    x = torch.zeros(1, 2, 2, 64, device=DEV)
    for call in (lambda: p.write(x, x.bfloat16()), lambda: p.write(x[..., :32], x[..., :32]), lambda: p.write(x.cpu(), x.cpu()),
                 lambda: p.write(x, x, _ids(0).long()), lambda: p.write(x, x, _ids(0, 1)), lambda: p.attn(x[..., :32]),
                 lambda: p.attn(x, out=x.bfloat16()), lambda: p.write(x.half(), x.half()), lambda: p.trim(_ids(0).cpu()),
                 lambda: p.write(x, x, idx=_ids(0, 1).view(1, 2)), lambda: p.fork(_ids(0), _ids(0, 1)),
                 lambda: p.write(x, x.transpose(0, 1).contiguous().transpose(0, 1)[:, :, :1])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(pb.PyrError):
        p.attn(torch.zeros(1, 1, 3, 64, device=DEV))               # query heads not a multiple of the KV heads
    with pytest.raises(pb.PyrError):
        p.write(torch.zeros(1, 2, 2, 66, device=DEV)[..., 1:65], torch.zeros(1, 2, 2, 66, device=DEV)[..., 1:65])     # alignment
    assert p.status() == 0


# ------------------------------------------------------------------ together

def test_calls_with_nothing_to_do():
    p = _pages(2, 64, 32, 32, 4, 3, 2)
    _fill(p, [5, 0, 40], seed=40)
    state = _state(p)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    kv = torch.zeros(0, 4, 2, 64, dtype=BF, device=DEV)
    p.reserve(none, 3)
    p.write(kv, kv, none)
    p.read(kv, kv, none)
    out, lse = p.attn(torch.zeros(0, 1, 4, 64, dtype=BF, device=DEV), none, lse=True)
    assert out.shape == (0, 1, 4, 64) and lse.shape == (0, 4, 1)
    p.fork(none, none)
    p.trim(none)
    p.compact(none, none, n_rows=4)
    empty = torch.zeros(3, 0, 2, 64, dtype=BF, device=DEV)
    p.write(empty, empty)
    p.read(empty, empty)
    assert p.status() == 0 and _unchanged(p, state)
    p.compact(_ids(0), _ids(0), idx=torch.zeros(1, 1, 0, dtype=torch.int32, device=DEV))
    assert p.status() == 0 and p.lens.tolist() == [0, 0, 40] and int(p.table[0].max()) == -1


def test_calls_run_on_the_stream_they_are_given():
    p = _pages(2, 128, 64, 16, 20, 2, 8)
    s = torch.cuda.Stream()
    k, v = _rand(2, 90, 2, 128, seed=90, dtype=BF), _rand(2, 90, 2, 128, seed=91, dtype=BF)
    q = _rand(2, 1, 4, 128, seed=92, dtype=BF)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    p.reserve(_ids(0, 1), 90, stream=s)
    p.write(k, v, stream=s)
    out, lse = p.attn(q, lse=True, stream=s)
    assert p.status(stream=s) == 0
    s.synchronize()
    _check_attn(p, q, range(2), out, lse, 128 ** -0.5)


def test_a_captured_decode_step_grows_its_lists_with_every_replay():
    """reserve + write + attention captured once: lengths live on the device, so each replay appends one row more."""
    n, hkv, hq, D = 3, 2, 8, 128
    p = _pages(hkv, D, 64, 16, 40, n, 8)
    lists = _ids(0, 1, 2)
    lens = [15, 40, 0]
    k0, v0 = _rand(n, 40, hkv, D, seed=100, dtype=BF), _rand(n, 40, hkv, D, seed=101, dtype=BF)
    p.reserve(lists, _ids(*lens))
    p.write(k0, v0, lists, counts=_ids(*lens))
    q, k, v = (torch.zeros(n, 1, h, D, dtype=BF, device=DEV) for h in (hq, hkv, hkv))
    out = torch.zeros_like(q)
    saved = _state(p)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                     # first launches happen outside the capture
        p.reserve(lists, 1); p.write(k, v, lists); p.attn(q, lists, out=out)
    torch.cuda.synchronize()
    for t, s in zip((p.pool, p.table, p.lens, p.refs), saved):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.reserve(lists, 1); p.write(k, v, lists); p.attn(q, lists, out=out)
    for t, s in zip((p.pool, p.table, p.lens, p.refs), saved):
        t.copy_(s)
    rows = [[], []]
    for step in range(20):
        q.copy_(_rand(n, 1, hq, D, seed=200 + step, dtype=BF))
        k.copy_(_rand(n, 1, hkv, D, seed=300 + step, dtype=BF))
        v.copy_(_rand(n, 1, hkv, D, seed=400 + step, dtype=BF))
        rows[0].append(_quantised(k, 64)); rows[1].append(_quantised(v, 64))
        graph.replay()
        assert p.status() == 0 and p.lens.tolist() == [x + step + 1 for x in lens]
        if step in (0, 1, 8, 19):
            for i in range(n):
                K = np.concatenate([_quantised(k0[i, :lens[i]], 64)] + [r[i] for r in rows[0]])
                V = np.concatenate([_quantised(v0[i, :lens[i]], 64)] + [r[i] for r in rows[1]])
                for a, w in zip(_list_values(p, i), (K, V)):
                    np.testing.assert_array_equal(a, w)
                want, _ = op.attention(_wide(q[i]), K, V, D ** -0.5)
                tol = 2.0 ** -9 * 8 * (V.max() - V.min()) / 15 * (1 + 2.0 ** -6) + 2.0 ** -8 * np.abs(want) + 1e-4
                assert (np.abs(_wide(out[i]) - want) <= tol).all()


def test_prompt_to_generation_on_pages():
    """As a serving engine would use it: prefill and selection by pyr_prefill_layer / pyr_select_compact, the kept rows straight
    into pages, a sequence forked into two samples, a few decode steps, one sample re-selected in place, one given up."""
    B, N, L, hq, hkv, D = 2, 256, 64, 8, 2, 128
    cache = pb.PyrCache(n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=D, sel_groups=hkv, dtype="bf16", batch=B, prompt_len=N,
                        recent_len=L, max_new_tokens=0, ratio=[0.5])
    Q, K, V = (_rand(B, N, h, D, seed=110 + i, dtype=BF) for i, h in enumerate((hq, hkv, hkv)))
    O = torch.empty_like(Q)
    cache.prefill_layer(0, Q, K, V, O)
    n_out = cache.select_compact(0, K, V)
    kept = cache.kept(0)[0]
    assert n_out == 96 + 64
    p = _pages(hkv, D, 64, 32, 30, 4, 8)
    p.reserve(_ids(0, 1), n_out)
    p.write(K, V, _ids(0, 1), idx=kept)
    Kc, Vc = cache.kv(0)
    for b in range(B):                               # what the layer's own cache holds, in 4 bits
        a, w = _list_values(p, b)
        np.testing.assert_array_equal(a, _quantised(Kc[b, :, :n_out].transpose(0, 1), 64))
        np.testing.assert_array_equal(w, _quantised(Vc[b, :, :n_out].transpose(0, 1), 64))
    p.fork(_ids(0), _ids(2))
    live = _ids(0, 1, 2)
    for step in range(5):
        q, k, v = (_rand(3, 1, h, D, seed=120 + 10 * step + i, dtype=BF) for i, h in enumerate((hq, hkv, hkv)))
        p.reserve(live, 1)
        p.write(k, v, live)
        out, lse = p.attn(q, live, lse=True)
        assert p.status() == 0
        _check_attn(p, q, live.tolist(), out, lse, D ** -0.5)
    assert p.lens.tolist() == [n_out + 5, n_out + 5, n_out + 5, 0]
    before = _list_values(p, 2)
    g = torch.Generator().manual_seed(130)
    sel = torch.stack([torch.sort(torch.randperm(n_out + 5, generator=g)[:90]).values for _ in range(hkv)])[None].to(torch.int32)
    p.compact(_ids(2), _ids(2), idx=sel.to(DEV))
    assert p.status() == pb.PYR_ERR_INVALID          # its full pages are shared with list 0: into a list of its own instead
    p.reserve(_ids(3), 90)
    p.compact(_ids(2), _ids(3), idx=sel.to(DEV))
    p.trim(_ids(2))
    assert p.status() == 0 and p.lens.tolist() == [n_out + 5, n_out + 5, 0, 90]
    for a, w in zip(_list_values(p, 3), before):
        for h in range(hkv):
            np.testing.assert_array_equal(a[:, h], w[sel[0, h].numpy(), h])
    q = _rand(1, 1, hq, D, seed=140, dtype=BF)
    out, lse = p.attn(q, _ids(3), lse=True)
    _check_attn(p, q, [3], out, lse, D ** -0.5)
    p.trim(_ids(0, 1, 3))
    assert p.status() == 0 and int(p.refs.sum()) == 0 and bool((p.table == -1).all())
