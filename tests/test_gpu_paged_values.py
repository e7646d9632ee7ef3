"""Attention over pages with values at the ends of their type: NaN and Inf in queries and keys that a row sees, values far above
1 behind scores that climb.  Outputs are checked as in test_gpu_paged_attention."""
import numpy as np
import pytest
import torch

from oracle import paged as o_paged
from test_gpu_paged_attention import check
from test_gpu_paged_step import steep
from test_gpu_qk_rows import BF16, F16, make_cache, np64, randn

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
# (tokens held, new ones), query heads on 2 KV heads: the kernel's blocks of 16, 32, 128 and 256 rows, whole and split
SHAPES = {"16 rows": ([(60, 1), (90, 2)], 8), "16 rows, split": ([(2000, 1), (90, 2)], 8), "32 rows": ([(60, 7), (90, 5)], 8),
          "32 rows, split": ([(2000, 7), (90, 5)], 8), "128 rows": ([(60, 20), (90, 31)], 8),
          "128 rows, split": ([(2000, 20), (90, 31)], 8), "256 rows": ([(60, 130), (30, 70)], 8), "256 rows, split": ([(1500, 130), (30, 70)], 8)}


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F16, 64)])
@pytest.mark.parametrize("lens,Hq", SHAPES.values(), ids=SHAPES.keys())
def test_nan_in_what_a_row_sees_makes_it_nan_and_no_other(lens, Hq, dtype, D):
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(61)
    cache, table, off, N = make_cache(gen, lens, 16, 2, D, dtype)
    q = randn(gen, N, Hq, D, dtype=dtype)
    good = dsbd.dsbd_paged_attention(cache, q)
    for bad in (NAN, INF, -INF):                             # in one query: its scores are NaN or Inf, and no other row's
        x = q.clone()
        x[N - 1, 5, 3] = bad
        out, lse, fault = dsbd.dsbd_paged_attention(cache, x)
        assert int(fault) == 0 and bool(out[N - 1, 5].isnan().all()) and bool(lse[N - 1, 5].isnan())
        keep = torch.ones((N, Hq), dtype=torch.bool, device="cuda")
        keep[N - 1, 5] = False
        assert torch.equal(out[keep], good[0][keep]) and torch.equal(lse[keep], good[1][keep])
    s, t = 1, lens[1][0] - 3                                 # in a key of the second sequence, in front of its new tokens
    p, slot = o_paged.place(table, 16, s, t)
    cache.k_pages[p, slot, 1, 3] = NAN
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    hit = torch.zeros((N, Hq), dtype=torch.bool, device="cuda")
    hit[off[1]:, Hq // 2:] = True
    assert int(fault) == 0 and bool(out[hit].isnan().all()) and bool(lse[hit].isnan().all())
    assert torch.equal(out[~hit], good[0][~hit]) and torch.equal(lse[~hit], good[1][~hit])


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F16, 64)])
@pytest.mark.parametrize("lens,Hq", SHAPES.values(), ids=SHAPES.keys())
def test_a_score_of_minus_infinity_counts_as_not_there(lens, Hq, dtype, D):
    """A key with an infinite channel: rows whose query has the other sign there give it no weight, the others are NaN."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(62)
    cache, table, off, N = make_cache(gen, lens, 16, 2, D, dtype)
    q = randn(gen, N, Hq, D, dtype=dtype)
    q[:, :, 3] = torch.where(torch.arange(Hq, device="cuda") % 2 == 0, 1.0, -1.0).to(dtype)
    at = [c - 2 for c, _ in lens]
    for s, t in enumerate(at):
        p, slot = o_paged.place(table, 16, s, t)
        cache.k_pages[p, slot, :, 3] = INF
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == 0 and bool(out[:, ::2].isnan().all()) and bool(lse[:, ::2].isnan().all())
    kp, vp = np64(cache.k_pages), np64(cache.v_pages)
    eps = torch.finfo(dtype).eps
    for s, (c, n) in enumerate(lens):
        k, there = o_paged.gather(kp, table, 16, s, c + n)
        v, _ = o_paged.gather(vp, table, 16, s, c + n)
        k[at[s]], there[at[s]] = 0, False
        for i in sorted({0, n - 1}):
            r = int(off[s]) + i
            w, wl, size = o_paged.attend(np64(q[r:r + 1]), k[:c + i + 1], v[:c + i + 1], there[:c + i + 1], c + i, D ** -0.5)
            tol = eps / 2 * (np.abs(w) + size) + 2e-4 * size + (c + n) * 2.0 ** -33 * size.max() + torch.finfo(dtype).smallest_normal
            assert (np.abs(np64(out[r]) - w[0]) <= tol[0])[1::2].all() and (np.abs(np64(lse[r]) - wl[0]) <= 2e-4)[1::2].all(), (s, i)


def large_values(lens, Hq, Hk, far, rows):
    """bf16 values about 2^100: the weighted sum stays in fp32's range, 2^128, while the reference trails the maximum.  Products and
    sums of the scores are exact, as in test_gpu_paged_step."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(63)
    cache, table, off, N = make_cache(gen, lens, 16, Hk, 128, BF16)
    cache.k_pages.copy_(steep(gen, cache.k_pages.shape, BF16))
    cache.v_pages.mul_(2.0 ** 100)
    for s, (c, n) in enumerate(lens):
        t = torch.arange(c + n)
        up = ((t >= c - 9).float() if far else t.float() / (c + n)).mul(48).round().div(8).to(BF16).cuda()       # up to 6, times 4: 2^34.6
        cache.k_pages[torch.from_numpy(table)[s, t // 16].long().cuda(), (t % 16).cuda(), :, 0] = up[:, None]
    q = steep(gen, (N, Hq, 128), BF16).mul(1.0 / 64)
    q[:, :, 0] = 4
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q, scale=1.0)
    assert int(fault) == 0 and bool(out.isfinite().all())
    check(cache, table, off, lens, q, out, lse, scale=1.0, rows=rows)


@pytest.mark.parametrize("lens,Hq", SHAPES.values(), ids=SHAPES.keys())
@pytest.mark.parametrize("far", [False, True], ids=["all along", "at the end"])
def test_large_values_behind_climbing_scores(lens, Hq, far):
    large_values(lens, Hq, 2, far, 10)


@pytest.mark.parametrize("n", [1, 6])
def test_large_values_where_a_wave_takes_step_after_step(n):
    """Enough sequences to fill the device: none is split, and a wave sees the far ones in its third step."""
    large_values([(380, n)] * 520, 8, 2, True, 2)
