"""Attention over the paged 4-bit cache where numbers are large, small or far apart, against fp64 (oracle/pages.py): query rows
over the whole range of their type."""
import numpy as np
import pytest
import torch

from oracle import pages as op
from paper_2405_12532_b200 import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def _ids(*x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def _wide(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _parts(p, l):
    """K values, then V's codes, scales and zeros per dimension, of a list's rows, all [rows, Hkv, D] in fp64."""
    c = p.cfg
    D, g, pr = c.head_dim, c.group, c.page_rows
    pool = p.pool.cpu().numpy().reshape(c.n_pages, c.n_kv_heads, pr // 16, -1)
    table, n = p.table[l].cpu().numpy(), int(p.lens[l])
    out = [np.zeros((n, c.n_kv_heads, D)) for _ in range(4)]
    for r0 in range(0, n, 16):
        m = min(16, n - r0)
        for h in range(c.n_kv_heads):
            kc, ks, kz, vc, vs, vz = op.unpack(pool[table[r0 // pr], h, r0 % pr // 16], D, g)
            for o, x in zip(out, (op.values(kc, ks, kz), vc, np.repeat(vs, g, -1), np.repeat(vz, g, -1))):
                o[r0:r0 + m, h] = x[:m]
    return out


def _score_error(q, K, scale):
    """Of one query row's scores: a code times a query value, summed in fp32 and multiplied by the row's (scale, zero), is off by
    at most (D + 8) 2^-23 of scale sum |q| (15 s + |zero|), and 15 s + |zero| is at most 3 times the row's largest |K| (a group
    that straddles zero has 15 s up to twice that, |zero| up to it) and the two roundings of the format."""
    return (K.shape[1] + 8) * 2.0 ** -23 * scale * np.abs(q).sum() * 3.1 * np.abs(K).max()


# ------------------------------------------------------------------ queries over the range of their type

# every binade where a factor of the kernels could leave fp32 or f16, both ends of bf16 (2^-133 is its smallest number) among them
EXPONENTS = [-133, -130, -127, -126, -125, -115, -114, -113, -112, -111, -100, -60, 0, 60, 96, 99, 100, 101, 113, 117, 118, 119, 121,
             122, 124, 126, 127]


@pytest.mark.parametrize("softmax_scale", [0.0, 1.0, 2.0 ** -30])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,group", [(64, 32), (128, 32), (128, 64), (128, 128)])
def test_query_rows_over_the_whole_range_of_bf16(D, group, dtype, softmax_scale):
    """List i's keys are of about 2^-e / softmax_scale (as far as numbers go), so that query rows of 2^e give scores of about 1;
    the first two KV rows are zeros. Every query head has a power of two of its own, e, e - 1, e - 40 and so on (columns of one
    matrix with factors of their own), some elements are zeros, one row is all zeros, and the largest element is the largest of
    its binade: at 127 that of bf16."""
    rows, T, hq = 45, 2, 6
    n = len(EXPONENTS)
    p = pb.PyrPages(n_kv_heads=1, head_dim=D, group=group, page_rows=32, n_pages=2 * n, n_lists=n, max_pages=2)
    g = torch.Generator().manual_seed(D + group)
    scale = softmax_scale or D ** -0.5
    e = torch.tensor(EXPONENTS, dtype=torch.float64).view(n, 1, 1, 1)
    k = torch.randn(n, rows, 1, D, generator=g, dtype=torch.float64).clamp(-1.9, 1.9)
    # the largest key is below 2^126: neither it nor its group's 15 steps leave the range
    k = (k * torch.exp2((-e + (30 if softmax_scale == 2.0 ** -30 else 0)).clamp(-140, 125))).float()
    k[:, :2] = 0
    v = torch.randn(n, rows, 1, D, generator=g)
    base = torch.randn(n, T, hq, D, generator=g, dtype=torch.float64).clamp(-1.9, 1.9)
    base[..., 3::7] = 0
    base[..., 5] = 1.9921875
    base[..., 9] = -1.9921875
    less = torch.tensor([0, 1, 40, 0, 7, 0], dtype=torch.float64).view(1, 1, hq, 1)
    q = (base * torch.exp2(e - less)).float().to(BF)           # (on the CPU: small numbers stay)
    q[:, 1, 3] = 0
    q = q.to(dtype)
    assert bool(torch.isfinite(q).all()) and float(q[-1].abs().max()) == float(torch.finfo(BF).max)
    p.reserve(_ids(*range(n)), rows)
    p.write(k.to(DEV), v.to(DEV))
    out, lse = p.attn(q.to(DEV), lse=True, softmax_scale=softmax_scale)
    assert p.status() == 0
    for i in range(n):
        K, vc, vs, vz = (x[:, 0] for x in _parts(p, i))
        V = vc * vs + vz
        for t in range(T):
            see = rows - (T - 1 - t)
            for h in range(hq):
                x = _wide(q[i, t, h])
                z = K[:see] @ x * scale
                want_lse = z.max() + np.log(np.exp(z - z.max()).sum())
                w = np.exp(z - want_lse)
                want = w @ V[:see]
                # fp32: the scores' error moves a weight by that factor; exponential and sums 2^-20. bf16 besides: weights
                # times a scale in f16 before they meet the codes, 2^-11 and what f16 cannot hold of a small one, 2^-25 a row (the
                # zeros' part stays in fp32), the output 2^-8
                ds = _score_error(x, K, scale) + 2.0 ** -22 * np.abs(z).max()
                rel = 2 * ds + 2.0 ** -20
                tol = rel * (w @ np.abs(V[:see]) + np.abs(want)) + 2.0 ** -24 * np.abs(want)
                if dtype == BF:
                    tol = tol + 2.0 ** -11 * (w @ (vc * vs)[:see]) + 2.0 ** -8 * np.abs(want) + 2.0 ** -25 * rows * 15 * vs.max()
                if rel > 0.5:                                  # scores so large that fp32 cannot tell the rows apart
                    assert bool(torch.isfinite(out[i, t, h]).all()), (EXPONENTS[i], t, h)
                    continue
                err = np.abs(_wide(out[i, t, h]) - want)
                assert (err <= tol).all(), (EXPONENTS[i], t, h, float(err.max()), float(tol.flat[err.argmax()]))
                lerr = abs(float(lse[i, h, t]) - want_lse)
                assert lerr <= ds + 2.0 ** -20 * (1 + abs(want_lse)), (EXPONENTS[i], t, h, lerr)


# ------------------------------------------------------------------ weights and scales far apart

def _attn_bound(z, w, c, s, zero, ds, small):
    """Of one bf16 output row: softmax weights w [rows], V's codes, scales, zeros [rows, D]. Weights off by 2 ds + 2^-20 and by
    their sums (each of a lane's adds 2^-24 over an eighth of the rows, each matrix instruction's 2^-23 over a sixteenth), the
    weights that meet the codes rounded to f16 (2^-11), `small` for what f16 cannot hold of them, the output's rounding."""
    v = c * s + zero
    rel = 2 * ds + 2.0 ** -20 + w.shape[0] * 2.0 ** -26
    want = w @ v
    return want, rel * (w @ v.abs() + want.abs()) + 2.0 ** -11 * (w @ (c * s)) + small + 2.0 ** -8 * want.abs()


@pytest.mark.parametrize("rows,outlier", [(16384, 50.0), (16384, 1.0), (65536, 8.0), (4096, 700.0)])
@pytest.mark.parametrize("D,group", [(64, 32), (128, 32), (128, 64), (128, 128)])
def test_many_small_weights_behind_a_large_one(D, group, rows, outlier):
    """Row 0 takes most of the weight, thousands of rows behind it 2^-16 to 2^-20.5 of its weight each (all alike: whatever
    is lost of one is lost of all), and one of the first 32 rows has values far above the others'. 407 entries of 4 heads are a
    (entry, head) a warp on 148 SMs, so that a warp meets all of it in order. f16 holds a weight times its normalised scale to
    2^-25, and that scale is at least 2^4 for the largest of any 32 rows read together: small = 2^-29 times code and that scale."""
    hkv, n = 4, 407
    p = pb.PyrPages(n_kv_heads=hkv, head_dim=D, group=group, page_rows=256, n_pages=rows // 256, n_lists=1, max_pages=rows // 256)
    g = torch.Generator().manual_seed(rows + D + group)
    k = torch.zeros(1, rows, hkv, D)
    k[0, 0] = (torch.tensor([16.0, 17.5, 19.5, 20.5]) * np.log(2.0) * D ** -0.5).view(hkv, 1)
    v = 1.2 * torch.randn(1, rows, hkv, D, generator=g)
    v[0, 5] *= outlier
    k, v = k.to(BF), v.to(BF)
    p.reserve(_ids(0), rows)
    p.write(k.to(DEV), v.to(DEV))
    q = torch.ones(n, 1, hkv, D, dtype=BF, device=DEV)
    out, lse = p.attn(q, _ids(*[0] * n), lse=True)
    assert p.status() == 0
    code, scale, zero = (torch.from_numpy(x).to(DEV) for x in op.quantise(v[0].float().numpy(), group))
    for h in range(hkv):
        c, s, z0 = code[:, h].double(), scale[:, h].double(), zero[:, h].double()
        near = torch.nn.functional.max_pool1d(s.T.unsqueeze(0), 63, 1, 31)[0].T
        small = 2.0 ** -29 * (c * near.repeat_interleave(group, 1)).sum(0)
        s, z0 = s.repeat_interleave(group, 1), z0.repeat_interleave(group, 1)
        z = k[0, :, h].double().sum(1).to(DEV) * D ** -0.5
        ds = (D + 8) * 2.0 ** -23 * float(z.max())
        want, tol = _attn_bound(z, torch.softmax(z, 0), c, s, z0, ds, small)
        err = (out[:, 0, h].double() - want).abs()
        assert bool((err <= tol).all()), (h, float(err.max()), float(tol.min()), float((err / tol).max()))
        assert float((lse[:, h, 0].double() - torch.logsumexp(z, 0)).abs().max()) <= ds + 2.0 ** -20 * 16 + rows * 2.0 ** -27


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_columns_with_magnitudes_of_their_own_over_scales_of_many(D, group, order):
    """The eight query heads of one column group are of 2^-60 to 2^60, the keys of three lists 2^-60, 1 and 2^60, and the scales of
    V run from 2^-90 to 2^90 up or down each list: held to the largest scale of the group (small = 2^-25 a row of it)."""
    n, rows, hq = 3, 96, 8
    p = pb.PyrPages(n_kv_heads=1, head_dim=D, group=group, page_rows=32, n_pages=9, n_lists=n, max_pages=3)
    g = torch.Generator().manual_seed(D + group + order)
    e = torch.tensor([-60.0, 0.0, 60.0]).view(n, 1, 1, 1)
    k = (torch.randn(n, rows, 1, D, generator=g) * torch.exp2(e)).to(BF)
    block = torch.arange(rows).view(1, rows, 1, 1) // 16
    v = (torch.randn(n, rows, 1, D, generator=g) * torch.exp2(order * (block * 36.0 - 90.0))).to(BF)
    q = (torch.randn(n, 1, hq, D, generator=g) * torch.exp2(torch.linspace(-60, 60, hq).round()).view(1, 1, hq, 1)).to(BF)
    p.reserve(_ids(0, 1, 2), rows)
    p.write(k.to(DEV), v.to(DEV))
    out, lse = p.attn(q.to(DEV), lse=True)
    assert p.status() == 0
    told = 0
    for i in range(n):
        K, c, s, z0 = (torch.from_numpy(x[:, 0]) for x in _parts(p, i))
        for h in range(hq):
            x = q[i, 0, h].double()
            z = K @ x * D ** -0.5
            ds = _score_error(x.numpy(), K.numpy(), D ** -0.5)
            assert bool(torch.isfinite(out[i, 0, h]).all())
            if ds > 0.1:
                continue
            told += 1
            w = torch.softmax(z, 0)
            want, tol = _attn_bound(z, w, c, s, z0, ds, 2.0 ** -25 * rows * 15 * s.max(0).values)
            err = (out[i, 0, h].double().cpu() - want).abs()
            assert bool((err <= tol).all()), (i, h, float((err / tol).max()))
            assert abs(float(lse[i, h, 0]) - float(torch.logsumexp(z, 0))) <= ds + 2.0 ** -20 * (1 + float(z.abs().max()))
    assert told >= 12


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("step", [3.9, 4.1, 5.0, 7.9])
def test_scores_a_step_of_fp32_apart(step, dtype):
    """Scores of about 2^26 of which two neighbouring numbers of fp32 are `step` powers of two of weight apart: 32 rows of the
    lower one, then eight of the upper one. fp32 says no more of the weights than that the upper ones are at least as large; whatever they
    are, an output lies among the values. (2000 entries: most are one warp's alone, which reads 32 rows, then eight.)"""
    D, rows, n = 128, 40, 2000
    p = pb.PyrPages(n_kv_heads=1, head_dim=D, group=32, page_rows=64, n_pages=1, n_lists=1, max_pages=1)
    g = torch.Generator().manual_seed(5)
    k = torch.zeros(1, rows, 1, D)
    k[..., :32] = 1.0                            # 32 of 1 and, in the last rows, 32 of 2^-23: a sum of 32, or of the next number
    k[:, 32:, :, 32:64] = 2.0 ** -23
    v = torch.randn(1, rows, 1, D, generator=g)
    v[..., ::32], v[..., 1::32] = 29.5, -29.5    # every group's scale just below 4
    p.reserve(_ids(0), rows)
    p.write(k.to(dtype).to(DEV), v.to(dtype).to(DEV))
    scale = step * float(np.log(2.0)) * 2.0 ** 18
    out, lse = p.attn(torch.ones(n, 1, 1, D, dtype=dtype, device=DEV), _ids(*[0] * n), lse=True, softmax_scale=scale)
    assert p.status() == 0
    K, c, s, z0 = (torch.from_numpy(x[:, 0]) for x in _parts(p, 0))
    assert set(K.sum(1).tolist()) == {32.0, 32.0 + 2.0 ** -18}
    V, got = c * s + z0, out[:, 0, 0].double().cpu()
    tol = 2.0 ** -8 * V.abs().max(0).values + 2.0 ** -11 * (c * s).max(0).values
    assert bool((got >= V.min(0).values - tol).all()) and bool((got <= V.max(0).values + tol).all())
    assert float((lse.double().cpu() / (float(K.sum(1).max()) * scale) - 1).abs().max()) <= 2.0 ** -21


def test_tokens_that_see_no_row_get_zeros_whatever_the_values():
    """48 tokens over 40 rows: the first eight, a column group of their own, see nothing, while the scales of V fall from 2^113 to
    2^-22 between two reads of 32 rows (a ratio beyond fp32)."""
    D, rows, T, n = 64, 40, 48, 300
    p = pb.PyrPages(n_kv_heads=1, head_dim=D, group=64, page_rows=64, n_pages=1, n_lists=1, max_pages=1)
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(1, rows, 1, D, generator=g), torch.randn(1, rows, 1, D, generator=g)
    v[:, :32] *= 2.0 ** 115
    v[:, 32:] *= 2.0 ** -20
    p.reserve(_ids(0), rows)
    p.write(k.to(BF).to(DEV), v.to(BF).to(DEV))
    q = torch.randn(1, T, 1, D, generator=g).to(BF).expand(n, -1, -1, -1).contiguous()
    out, lse = p.attn(q.to(DEV), _ids(*[0] * n), lse=True)
    assert p.status() == 0
    assert not bool(out[:, :8].any()) and bool(torch.isneginf(lse[:, :, :8]).all())
    K, c, s, z0 = (torch.from_numpy(x[:, 0]) for x in _parts(p, 0))
    for t in range(8, T):
        see = t - 7
        x = q[0, t, 0].double()
        z = K[:see] @ x * D ** -0.5
        want, tol = _attn_bound(z, torch.softmax(z, 0), c[:see], s[:see], z0[:see], _score_error(x.numpy(), K.numpy(), D ** -0.5),
                                2.0 ** -25 * rows * 15 * s.max(0).values)
        assert bool(((out[:, t, 0].double().cpu() - want).abs() <= tol).all()), t


# ------------------------------------------------------------------ tables with room to grow

@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_a_list_could_hold_does_not_refuse_a_call(dtype):
    """Tables for 2^31 rows, lists of 100: the same outputs, bit for bit, as with tables of one page."""
    hkv, hq, D, T, lens = 8, 64, 64, 80, [100, 90]
    res = []
    for slots in (1, 2097150):
        p = pb.PyrPages(n_kv_heads=hkv, head_dim=D, group=64, page_rows=1024, n_pages=2, n_lists=2, max_pages=slots)
        g = torch.Generator().manual_seed(4)
        k, v, q = (torch.randn(2, r, h, D, generator=g).to(dtype).to(DEV) for r, h in ((100, hkv), (100, hkv), (T, hq)))
        p.reserve(_ids(0, 1), 100)
        p.write(k, v, counts=_ids(*lens))
        out, lse = p.attn(q, lse=True)
        assert p.status() == 0 and p.lens.tolist() == lens
        res.append((out, lse))
        del p
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1]) and bool(torch.isfinite(res[0][0]).all())


# ------------------------------------------------------------------ long lists

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_means_of_thousands_of_rows(D, group, T, dtype):
    """Small queries: softmax is almost flat, an output is the mean of thousands of values of about 1, itself about 0.01, and the
    scores' own errors are far below that. The f16 roundings of the weights (bf16) are of either sign, at most 2^-11, spread
    evenly: eight standard deviations of their sum; the rest as for a row of many weights. Half an output lost would be 50 times
    the bound."""
    lens, hkv, hq = [5000, 4099, 70], 2, 8
    p = pb.PyrPages(n_kv_heads=hkv, head_dim=D, group=group, page_rows=64, n_pages=200, n_lists=3, max_pages=80)
    g = torch.Generator().manual_seed(D + group + T)
    k, v = (torch.randn(3, max(lens), hkv, D, generator=g).to(dtype) for _ in range(2))
    q = (torch.randn(3, T, hq, D, generator=g) * 2.0 ** -6).to(dtype)
    p.reserve(_ids(0, 1, 2), _ids(*lens))
    p.write(k.to(DEV), v.to(DEV), counts=_ids(*lens))
    out, lse = p.attn(q.to(DEV), lse=True)
    assert p.status() == 0
    for i, n in enumerate(lens):
        parts = [torch.from_numpy(x) for x in _parts(p, i)]
        for h in range(hq):
            K, c, s, z0 = (x[:, h // (hq // hkv)] for x in parts)
            for t in range(T):
                see = n - (T - 1 - t)
                x = q[i, t, h].double()
                z = K[:see] @ x * D ** -0.5
                w = torch.softmax(z, 0)
                cs = (c * s)[:see]
                values = cs + z0[:see]
                want = w @ values
                rel = 2 * _score_error(x.numpy(), K.numpy(), D ** -0.5) + 2.0 ** -20 + see * 2.0 ** -26
                tol = rel * (w @ values.abs() + want.abs()) + 2.0 ** -24 * want.abs()
                if dtype == BF:
                    tol = tol + 8 * 2.0 ** -11 / 3 ** 0.5 * torch.sqrt(w.square() @ cs.square()) + 2.0 ** -8 * want.abs()
                err = (out[i, t, h].double().cpu() - want).abs()
                assert bool((err <= tol).all()), (i, h, t, float((err / tol).max()))
                assert abs(float(lse[i, h, t]) - float(torch.logsumexp(z, 0))) <= rel + 2.0 ** -20 * 16
