"""Attention over the paged 8-bit cache where queries, keys and the softmax scale lie anywhere in the range of their types, against fp64
over what the codes stand for."""
import numpy as np
import pytest
import torch

from oracle import pages8 as o8
from paper_2405_12532_b200 import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
# both ends of bf16 (2^-133 is its smallest number), and where a query row's power of two or a product with it could leave fp32 or f16
EXPONENTS = [-133, -130, -127, -126, -125, -115, -114, -113, -112, -111, -100, -60, -20, 0, 20, 60, 96, 100, 112, 113, 114, 121, 124, 126, 127]


@pytest.mark.parametrize("softmax_scale", [0.0, 1.0, 2.0 ** -30, 2.0 ** 60, 2.0 ** 126, 2.0 ** -100, 2.0 ** -126, 1.5 * 2.0 ** -148])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_query_rows_over_the_whole_range_of_bf16(D, dtype, softmax_scale):
    """List i's keys are of about 2^-e / softmax_scale (as far as they can be stored), so that query rows of 2^e give scores of about 1. Every
    query head has a power of two of its own, some elements are zeros, one row is all zeros, and the largest element is
    the largest of its binade: at 127 that of bf16. Keys whose page has a scale of 0 are zeros: their scores are."""
    rows, T, hq = 45, 2, 6
    n = len(EXPONENTS)
    p = pb.PyrPages(bits=8, n_kv_heads=1, head_dim=D, page_rows=64, n_pages=n, n_lists=n, max_pages=1)
    g = torch.Generator().manual_seed(D)
    scale = softmax_scale or D ** -0.5
    e = torch.tensor(EXPONENTS, dtype=torch.float64).view(n, 1, 1, 1)
    k = torch.randn(n, rows, 1, D, generator=g, dtype=torch.float64).clamp(-1.9, 1.9)
    k = (k * torch.exp2((-e - round(np.log2(scale) if softmax_scale else 0)).clamp(-140, 125))).float()
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
    p.reserve(torch.arange(n, dtype=torch.int32, device=DEV), rows)
    p.write(k.to(DEV), v.to(DEV))
    out, lse = p.attn(q.to(DEV), lse=True, softmax_scale=softmax_scale)
    assert p.status() == 0
    pool, told = p.pool.cpu().numpy(), 0
    for i in range(n):
        kc, vc, ks, vs, *_ = o8.unpack(pool, p.table[i].cpu().numpy(), rows, 1, D, 64)
        K, V = (c[:, 0] * s.astype(np.float64) for c, s in ((kc, ks), (vc, vs)))
        for t in range(T):
            see = rows - (T - 1 - t)
            for h in range(hq):
                x = q[i, t, h].double().numpy()
                z = K[:see] @ x * scale
                want_lse = z.max() + np.log(np.exp(z - z.max()).sum())
                w = np.exp(z - want_lse)
                want = w @ V[:see]
                # a score: the instruction's 8 sums of 16 products lose 2^-22 of their size each, fp32 queries are two f16 (2^-22), five
                # products are rounded: 2^-19 (fp32: 2^-18) of sum |q| |k|, and elements below 2^-31 of a row's largest, here zeros. A weight: that
                # error twice (numerator and denominator), f16 2^-11 (fp32: two, 2^-22) or 2^-35 of the largest, exponential and sums 2^-19
                ds = (np.abs(K[:see]) @ np.abs(x)).max() * scale * 2.0 ** (-19 if dtype == BF else -18)
                rel = 2 * ds + 2.0 ** -19 + (2.0 ** -11 if dtype == BF else 0)
                tol = rel * (w @ np.abs(V[:see])) + 2.0 ** (-8 if dtype == BF else -22) * np.abs(want) + 2.0 ** -35 * rows * np.abs(V).max()
                assert bool(torch.isfinite(out[i, t, h]).all()), (EXPONENTS[i], t, h)
                if rel > 0.5:                                  # scores so large that fp32 cannot tell the rows apart
                    continue
                told += 1
                err = np.abs(out[i, t, h].double().cpu().numpy() - want)
                assert (err <= tol).all(), (EXPONENTS[i], t, h, float((err / tol).max()))
                lerr = abs(float(lse[i, h, t]) - want_lse)
                assert lerr <= ds + 2.0 ** -20 * (1 + abs(want_lse)), (EXPONENTS[i], t, h, lerr)
    assert told > n * T * hq * 3 // 4


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_whose_codes_a_query_does_not_meet_score_zero(dtype):
    """A query of 2^126 in one dimension, keys of 2^60 in another: every factor of a score leaves fp32, every score is 0."""
    D, rows = 128, 40
    p = pb.PyrPages(bits=8, n_kv_heads=1, head_dim=D, page_rows=64, n_pages=1, n_lists=1, max_pages=1)
    k, q = torch.zeros(1, rows, 1, D, device=DEV), torch.zeros(1, 1, 1, D, dtype=dtype, device=DEV)
    k[..., 3], q[..., 90] = 2.0 ** 60, 2.0 ** 126
    v = torch.randn(1, rows, 1, D, generator=torch.Generator().manual_seed(1)).to(DEV)
    p.reserve(torch.zeros(1, dtype=torch.int32, device=DEV), rows)
    p.write(k, v)
    out, lse = p.attn(q, lse=True)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    p.read(ko, vo)
    assert p.status() == 0 and abs(float(lse) - np.log(rows)) <= 2.0 ** -20
    want = vo.double().mean(1)
    # all weights are alike and f16 numbers: the sums' 2^-20 of the mean magnitude and the output's rounding
    tol = 2.0 ** -20 * vo.double().abs().mean(1) + (2.0 ** -8 if dtype == BF else 2.0 ** -22) * want.abs() + 2.0 ** -11 * vo.double().abs().mean(1) * (dtype == BF)
    assert bool(((out[:, 0].double() - want).abs() <= tol).all())
