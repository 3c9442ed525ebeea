"""The paged 8-bit cache as programs use it, on paths that its kernels' rules keep apart: several heads a CTA with rows of each head's own,
chunks of a prompt attended as chunks, kept rows straight from the selection, captured chunks, and both formats on the same rows."""
import math

import numpy as np
import pytest
import torch

from oracle import pages8 as o8
from paper_2405_12532_b200 import binding as pb
from test_gpu_pages8 import BF, DEV, F32, _check, _compare, _dense, _filled, _ids, _np, _pages, _rand, _state

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ storing, several heads a CTA

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("pr,n,rows", [(16, 75, 60), (64, 24, 150), (128, 40, 200), (112, 34, 215), (16, 300, 33)])
def test_heads_of_a_cta_have_rows_and_positions_of_their_own(pr, n, rows, own, D, dtype):
    """13 KV heads and so many pages that a CTA takes 2 to 7 of them one after the other (the last fewer), for itself or behind a launch that
    decides; gathered rows and positions a head or a sequence, lists that begin inside pages, ragged counts, sources and positions
    out of range in some heads. fp32 with pages of 112 and 128 rows of 128 dimensions has one stage of copies, the rest two."""
    H, src, n_pos = 13, rows + 30, 700
    groups = H if own else 1
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert n * H * ((rows + pr - 2) // pr + 1) >= 2 * 4 * sms          # two heads a CTA at least
    g = torch.Generator().manual_seed(pr + n + D + own)
    begin = [(7 * i) % (pr + 5) for i in range(n)]
    counts = [rows - (i * 11) % 29 if i % 7 else rows for i in range(n)]
    counts[3] = 0
    slots = -(-(pr + 5 + rows) // pr)
    p = _pages(H, D, pr, n * slots + 5, n + 2, slots)
    lists = [n + 1 - i for i in range(n)]
    p.reserve(_ids(*lists), max(begin) + rows)
    k0, v0 = (_rand(n, max(begin), H, D, seed=s, dtype=dtype, scale=0.5) for s in (1, 2))
    p.write(k0, v0, _ids(*lists), counts=_ids(*begin))
    k, v = (_rand(n, H, src, D, seed=s, dtype=dtype, scale=2.0).transpose(1, 2) for s in (3, 4))
    idx = torch.randint(0, src, (n, groups, rows), generator=g).to(torch.int32)
    pos = torch.randint(0, n_pos, (n, groups, rows), generator=g).to(torch.int32)
    idx[5, groups - 1, 2], pos[6, groups // 2, 1], idx[7, 0, rows - 40 if rows > 40 else 0] = src, -1, -5
    rope = pb.glue_rope_table(n_pos, D)
    p.append(k, v, _ids(*lists), pos=pos.to(DEV), rope=rope, idx=idx.to(DEV), counts=_ids(*counts))
    assert p.status() == pb.PYR_ERR_INVALID and p.status() == 0          # the three rows
    table = _np(rope)
    for i in (0, 3, 5, 6, 7, n // 2, n - 1):
        want = o8.List8(H, D, pr, slots * pr)
        want.store(0, _np(k0[i, :begin[i]]), _np(v0[i, :begin[i]]))
        c = counts[i]
        ks, vs = np.zeros((c, H, D), np.float32), np.zeros((c, H, D), np.float32)
        for h in range(H):
            at, angle = idx[i, h % groups, :c].numpy(), pos[i, h % groups, :c].numpy()
            good = (at >= 0) & (at < src) & (angle >= 0) & (angle < n_pos)
            at, angle = np.where(good, at, 0), np.where(good, angle, 0)
            ks[:, h] = np.where(good[:, None], o8.rotate(_np(k[i])[at, h], table[angle]), np.nan)
            vs[:, h] = np.where(good[:, None], _np(v[i])[at, h], np.nan)
        if c:
            want.store(begin[i], ks, vs)
        _check(p, lists[i], want)


# ------------------------------------------------------------------ chunks

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,pr,H,rep,T", [(128, 64, 2, 4, 40), (64, 48, 3, 1, 41), (128, 128, 1, 3, 500), (64, 16, 1, 1, 333)])
def test_a_chunk_of_queries_attends_to_itself_and_what_came_before(D, pr, H, rep, T, dtype):
    """Many column groups, most of whose columns are different tokens; lists as long as the chunk, longer, shorter (the first tokens see no row)
    and empty."""
    lens = [T, 0, T + 1, T - 1, 3, 900, T + 16]
    p, want = _filled(H, D, pr, lens, seed=5, dtype=dtype)
    q = _rand(len(lens), T, H * rep, D, seed=6, dtype=dtype, scale=1.5)
    out, lse = p.attn(q, lse=True)
    again, lse2 = p.attn(q, lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2) and p.status() == 0
    for i, n in enumerate(lens):
        K, V = want[i].values()
        _compare(dtype, _np(out[i]), _np(lse[i]), o8.attention(_np(q[i]).astype(np.float64), K, V, _dense(n, T, H), 1 / math.sqrt(D)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_chunk_over_chosen_pages(dtype):
    """Forty tokens, each with pages of its own."""
    H, D, pr, rep, T, n_slots = 2, 128, 16, 4, 40, 5
    lens = [300, 40, 17]
    p, want = _filled(H, D, pr, lens, seed=7, dtype=dtype)
    q = _rand(3, T, H * rep, D, seed=8, dtype=dtype)
    slots = p.select(q, n_slots, keep_last=1)
    out, lse = p.attn_blocks(q, slots, lse=True)
    assert p.status() == 0
    got = slots.cpu().numpy()
    for i, n in enumerate(lens):
        w = want[i]
        np.testing.assert_array_equal(got[i], np.stack([o8.select(_np(q[i, t]), w.mn, w.mx, w.scale[0], n - (T - 1 - t), pr, n_slots, 0, 1) for t in range(T)]))
        K, V = w.values()
        _compare(dtype, _np(out[i]), _np(lse[i]), o8.attention(_np(q[i]).astype(np.float64), K, V, _dense(n, T, H, pr, got[i]), 1 / math.sqrt(D)))


@pytest.mark.parametrize("n,lists", [(3, [2, 0, 1]), (300, None)])
def test_chunks_are_captured_and_replayed(n, lists):
    """Room, rows stored with their queries turned, attention of the chunk: one graph for every chunk gives what eager calls on another handle
    give, where CTAs decide for themselves and behind a launch that decides."""
    H, rep, D, pr, rows = 2, 3, 64, 16, 6
    cap = 5 + 6 * rows
    handles = [_filled(H, D, pr, [i % 6 for i in range(n)], seed=9, spare=6 * rows)[0] for _ in range(2)]
    rope = pb.glue_rope_table(200, D)
    ids = _ids(*(lists or range(n)))
    k, v = torch.zeros(n, rows, H, D, dtype=BF, device=DEV), torch.zeros(n, rows, H, D, dtype=BF, device=DEV)
    q = torch.zeros(n, rows, H * rep, D, dtype=BF, device=DEV)
    counts, pos = torch.full((n,), rows, dtype=torch.int32, device=DEV), torch.zeros(n, 1, rows, dtype=torch.int32, device=DEV)
    outs = [torch.zeros_like(q), torch.zeros_like(q)]

    def step(p, k, v, q, pos, counts, outs):
        p.append(k, v, ids, pos=pos, rope=rope, q=q, q_out=outs[0], counts=counts)
        p.attn(outs[0], ids, out=outs[1])

    graphed, eager = handles
    state = _state(graphed)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(graphed, k, v, q, pos, counts, outs)                # (a first call outside the capture)
    torch.cuda.current_stream().wait_stream(side)
    for t, o in zip((graphed.pool, graphed.table, graphed.lens, graphed.refs), state):
        t.copy_(o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed, k, v, q, pos, counts, outs)
    for chunk in range(6):
        for x, seed in ((k, 1), (v, 2), (q, 3)):
            x.copy_(_rand(*x.shape, seed=100 * chunk + seed, dtype=BF, scale=1 + chunk % 3))
        pos.copy_((torch.arange(n * rows, dtype=torch.int32) % 31 + chunk).view(n, 1, rows))
        counts.copy_(torch.tensor([(i + chunk) % (rows + 1) for i in range(n)], dtype=torch.int32))
        graph.replay()
        mine = [torch.zeros_like(x) for x in outs]
        step(eager, k.clone(), v.clone(), q.clone(), pos.clone(), counts.clone(), mine)
        assert all(torch.equal(a, b) for a, b in zip(outs, mine))
    assert eager.status() == 0 and graphed.status() == 0 and int(graphed.lens.max()) <= cap
    assert all(torch.equal(a, b) for a, b in zip(_state(graphed)[1:], _state(eager)[1:]))


@pytest.mark.parametrize("groups", [1, 2])
def test_prompt_to_generation_with_kept_rows_at_their_positions(groups):
    """Prefill and selection by pyr_prefill_layer / pyr_select_compact; both pointers of pyr_cache_kept, the kept rows and their original
    positions, go straight into append; then decode steps over all rows and over chosen pages."""
    B, N, L, hq, hkv, D, pr = 2, 256, 64, 8, 2, 128, 32
    cache = pb.PyrCache(n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=D, sel_groups=groups, dtype="bf16", batch=B, prompt_len=N,
                        recent_len=L, max_new_tokens=0, ratio=[0.5])
    Q, K, V = (_rand(B, N, h, D, seed=110 + i, dtype=BF) for i, h in enumerate((hq, hkv, hkv)))
    cache.prefill_layer(0, Q, K, V, torch.empty_like(Q))
    n_out = cache.select_compact(0, K, V)
    kept, at = cache.kept(0)
    assert kept.shape == (B, groups, n_out) and torch.equal(kept, at)          # (the first layer: rows are positions)
    p = _pages(hkv, D, pr, 20, B, 8)
    rope = pb.glue_rope_table(N + 10, D)
    p.reserve(_ids(0, 1), n_out + 5)
    p.append(K, V, _ids(0, 1), pos=at, rope=rope, idx=kept)
    want = []
    for b in range(B):
        w = o8.List8(hkv, D, pr, 8 * pr)
        rows = kept[b].cpu().numpy()
        ks = np.stack([o8.rotate(_np(K[b])[rows[h % groups], h], _np(rope)[rows[h % groups]]) for h in range(hkv)], 1)
        vs = np.stack([_np(V[b])[rows[h % groups], h] for h in range(hkv)], 1)
        w.store(0, ks, vs)
        _check(p, b, w)
        want.append(w)
    for step in range(5):
        q, k, v = (_rand(B, 1, h, D, seed=120 + 10 * step + i, dtype=BF) for i, h in enumerate((hq, hkv, hkv)))
        qr = p.append(k, v, pos=torch.full((B, 1, 1), N + step, dtype=torch.int32, device=DEV), rope=rope, q=q)
        slots = p.select(qr, 3, keep_last=1)
        out, lse = p.attn(qr, lse=True)
        some, some_lse = p.attn_blocks(qr, slots, lse=True)
        for b in range(B):
            want[b].store(n_out + step, o8.rotate(_np(k[b]), _np(rope)[N + step]), _np(v[b]))
            _check(p, b, want[b])
            Kb, Vb = want[b].values()
            for o, s, chosen in ((out, lse, None), (some, some_lse, slots[b].cpu().numpy())):
                _compare(BF, _np(o[b]), _np(s[b]), o8.attention(_np(qr[b]).astype(np.float64), Kb, Vb, _dense(n_out + step + 1, 1, hkv, pr, chosen), 1 / math.sqrt(D)))
    assert p.status() == 0


# ------------------------------------------------------------------ both formats

@pytest.mark.parametrize("pr", [64, 128])
def test_errors_of_both_formats_on_the_same_rows(pr):
    """Gaussian rows. 4 bits: 64 of them span 4.7 deviations on average, a step of 0.31, its error 0.31 / sqrt(12). 8 bits: the largest magnitude
    of pr * 128 is about 4, a step of 0.032: a tenth. Row by row an old code is rounded anew each time that its page's scale grows, some five
    times at errors that shrink with the steps before: below half as much again. In every case a value is within s / 2 of its
    number, and as much for each time that s grew. One large dimension (20 times the rest, its largest of 64 or 128 rows about 2.5 deviations: s of 0.4,
    an error of 0.11) sets the scale of all dimensions in 8 bits, and of its group alone in 4: the other group is looked at."""
    H, D, n = 4, 128, pr
    x = _rand(1, n, H, D, seed=3)
    big = x.clone()
    big[..., 7] *= 20.0
    rms = {}
    for name, rows in (("gaussian", x), ("one large dimension", big)):
        for bits, kw in ((4, dict(group=64)), (8, {})):
            for once in (True, False):
                p = pb.PyrPages(bits=bits, n_kv_heads=H, head_dim=D, page_rows=pr, n_pages=2, n_lists=1, max_pages=1, **kw)
                p.reserve(_ids(0), n)
                if once:
                    p.write(rows, rows)
                else:
                    for r in range(n):
                        p.write(rows[:, r:r + 1], rows[:, r:r + 1])
                k, v = torch.zeros_like(rows), torch.zeros_like(rows)
                p.read(k, v)
                assert p.status() == 0
                err = (k - rows).double()
                assert torch.equal(k, v)
                rms[name, bits, once] = float(err[..., 64:].square().mean().sqrt())
                if bits == 8 and once:
                    s = rows.abs().amax((0, 1, 3)) / 127
                    assert bool((err.abs().amax((0, 1, 3)) <= s.double() * (0.5 + 2.0 ** -16)).all())
    assert rms["gaussian", 4, True] == rms["gaussian", 4, False]
    assert rms["gaussian", 8, True] * 8 <= rms["gaussian", 4, True] and rms["gaussian", 8, False] <= 1.5 * rms["gaussian", 8, True]
    assert rms["one large dimension", 8, True] >= rms["one large dimension", 4, True]
