"""Attention of chunks of new tokens over a paged cache, against the softmax in 64 bits.

What an output may be off by: its own rounding, eps/2 of it; the numerators' rounding to the type in front of the product
with V, eps/2 of every term, so eps/2 of the weighted sum of |v|; the scores' sums in fp32, D products of up to 50 added up in
their turn: below 1e-4 in the exponent, so 2e-4 of the same sum; f16 numerators below 2^-14 lose 2^-25 of 2^8 each."""
import numpy as np
import pytest
import torch

from oracle import paged as o_paged
from test_gpu_qk_rows import BF16, F16, logical, make_cache, np64, randn

pytestmark = pytest.mark.gpu


def trees(gen, lens):
    out = []
    for _, n in lens:
        m = []
        for i in range(n):
            m.append((m[int(torch.randint(0, i, (1,), generator=gen))] if i else 0) | 1 << i)
        out += m
    return np.array(out, dtype=np.uint64)


def check(cache, table, off, lens, q, out, lse, scale=None, anc=None, rows=None, front=None):
    page = cache.k_pages.shape[2 if cache.head_major else 1]
    kp, vp = np64(logical(cache.k_pages, cache.head_major)), np64(logical(cache.v_pages, cache.head_major))
    eps, D = torch.finfo(out.dtype).eps, q.shape[2]
    o, l, q = np64(out), np64(lse), np64(q)
    for s, (c, n) in enumerate(lens):
        if n == 0:
            continue
        k, there = o_paged.gather(kp, table, page, s, c + n)
        v, _ = o_paged.gather(vp, table, page, s, c + n)
        a, b = int(off[s]), int(off[s + 1])
        pick = np.arange(n) if rows is None or n <= rows else np.unique(np.concatenate([[0, 1, n - 1], np.linspace(0, n - 1, rows).astype(int)]))
        for i in pick if front is None else range(front):      # row by row: what it sees of the chunk ends with itself, or is its mask's
            m = n if anc is not None else i + 1
            w, wl, size = o_paged.attend(q[a + i:a + i + 1], k[:c + m], v[:c + m], there[:c + m], c if anc is not None else c + i,
                                         D ** -0.5 if scale is None else scale, None if anc is None else anc[a + i:a + i + 1])
            tol = eps / 2 * (np.abs(w) + size) + 2e-4 * size + (c + m) * 2.0 ** -33 * size.max() + torch.finfo(out.dtype).smallest_normal
            err = np.abs(o[a + i] - w[0])
            assert (err <= tol[0]).all(), (s, i, float((err / tol[0]).max()))
            empty = np.isinf(wl[0])
            assert (l[a + i][empty] == -np.inf).all() and (np.abs(l[a + i][~empty] - wl[0][~empty]) <= 2e-4).all(), (s, i)
            assert (o[a + i][empty] == 0).all()


SHAPES = {
    "one token": [(0, 1)],
    "short": [(31, 1), (32, 1)],
    "tokens": [(0, 1), (1, 1), (63, 1), (700, 1), (33, 1), (1500, 1)],
    "empty ones": [(5, 0), (40, 3), (0, 0), (0, 2), (9, 0)],
    "chunks": [(0, 70), (3, 33), (129, 5), (64, 1), (200, 150)],
    "long": [(4001, 2)],
    "prompt": [(0, 515)],
}


@pytest.mark.parametrize("lens", SHAPES.values(), ids=SHAPES.keys())
@pytest.mark.parametrize("dtype,D,Hq,Hk,page,head_major", [
    (BF16, 128, 8, 2, 16, False), (F16, 128, 4, 4, 64, True), (BF16, 64, 6, 2, 3, False), (F16, 64, 7, 1, 1, True),
    (BF16, 128, 5, 5, 256, True), (F16, 128, 12, 2, 24, False)])
def test_causal_chunks(lens, dtype, D, Hq, Hk, page, head_major):
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(len(lens) * 100 + page)
    cache, table, off, N = make_cache(gen, lens, page, Hk, D, dtype, head_major)
    q = randn(gen, N, Hq, D, dtype=dtype, scale=1.5)
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse, rows=24)


@pytest.mark.parametrize("lens", [[(40, 7), (0, 31), (333, 64), (32, 1)], [(2000, 31)]], ids=["ragged", "long"])
@pytest.mark.parametrize("dtype,D,Hq,Hk,page", [(BF16, 128, 8, 2, 16), (F16, 64, 4, 4, 32)])
def test_trees(lens, dtype, D, Hq, Hk, page):
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(11)
    cache, table, off, N = make_cache(gen, lens, page, Hk, D, dtype)
    q = randn(gen, N, Hq, D, dtype=dtype)
    anc = trees(gen, lens)
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q, anc_mask=torch.from_numpy(anc.view(np.int64)).cuda(), scale=0.2)
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse, scale=float(np.float32(0.2)), anc=anc, rows=12)


def test_rows_that_see_nothing_and_padding():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(12)
    lens = [(0, 5), (7, 3)]
    cache, table, off, N = make_cache(gen, lens, 16, 2, 64, BF16, front=1, behind=4)
    q = randn(gen, N, 4, 64)
    anc = np.zeros(N, dtype=np.uint64)
    anc[1 + 1] = 0b11                       # of the first tree only the second node sees anything
    out, lse = torch.full((N, 4, 64), 3.0, dtype=BF16, device="cuda"), torch.full((N, 4), 3.0, device="cuda")
    dsbd.dsbd_paged_attention(cache, q, anc_mask=torch.from_numpy(anc.view(np.int64)).cuda(), out=out, lse=lse)
    check(cache, table, off, lens, q, out, lse, anc=anc)
    for t in (out, lse):
        assert bool((t[:1] == 3).all()) and bool((t[9:] == 3).all())
    assert bool((out[1] == 0).all()) and bool((lse[3] == -float("inf")).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("D,Hk,dtype", [(128, 2, BF16), (64, 1, F16)])
def test_what_a_row_does_not_see_does_not_reach_it(bad, D, Hk, dtype):
    """Slots behind the last token, other pages, and the chunk's later tokens hold NaN or Inf."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(13)
    for lens, spoilt in ([(20, 9)], 4), ([(130, 200)], 150), ([(5, 1)], 1), ([(0, 40)], 33):
        cache, table, off, N = make_cache(gen, lens, 16, Hk, D, dtype)
        q = randn(gen, N, 4, D, dtype=dtype)
        ctx, n = lens[0]
        used = torch.zeros(cache.k_pages.shape[:2], dtype=torch.bool)
        for t in range(ctx + n):
            used[o_paged.place(table, 16, 0, t)] = True
        for pages in (cache.k_pages, cache.v_pages):
            pages[~used.cuda()] = bad
        out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
        assert int(fault) == 0
        clean = out.clone(), lse.clone()
        check(cache, table, off, lens, q, out, lse, rows=10)
        if spoilt < n:                      # a token of the chunk: rows in front of it stay as they were, it and those behind see it
            p, slot = o_paged.place(table, 16, 0, ctx + spoilt)
            cache.v_pages[p, slot, :, 3] = bad
            out, lse, _ = dsbd.dsbd_paged_attention(cache, q)
            check(cache, table, off, lens, q, out, lse, front=spoilt)
            assert torch.equal(lse, clean[1])
            assert not bool(out[spoilt:, :, 3].isfinite().any()) and bool(out[spoilt:, :, 4:].isfinite().all())
            cache.k_pages[p, slot] = bad
            out, lse, _ = dsbd.dsbd_paged_attention(cache, q)
            check(cache, table, off, lens, q, out, lse, front=spoilt)
            assert torch.equal(lse[:spoilt], clean[1][:spoilt])


def test_lost_pages_and_bad_lengths_are_reported():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(14)
    lens = [(70, 3), (10, 2), (33, 4)]
    cache, table, off, N = make_cache(gen, lens, 16, 2, 64, BF16)
    q = randn(gen, N, 4, 64)
    good = dsbd.dsbd_paged_attention(cache, q)
    cache.page_table[0, 2], table = cache.k_pages.shape[0] + 5, cache.page_table.cpu().numpy().copy()
    table[0, 2] = cache.k_pages.shape[0] + 5
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == dsbd.DSBD_FAULT_BOUNDS
    check(cache, table, off, lens, q, out, lse)                      # the other pages' tokens count
    assert torch.equal(out[off[1]:], good[0][off[1]:])
    cache.page_table[0, 2] = 0
    for name, value in (("ctx_len", -1), ("ctx_len", 1 << 30), ("ctx_len", (1 << 31) - 1)):
        keep = cache.ctx_len.clone()
        cache.ctx_len[1] = value
        out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
        assert int(fault) == dsbd.DSBD_FAULT_BOUNDS
        a, b = int(off[1]), int(off[2])
        assert bool((out[a:b] == 0).all()) and bool((lse[a:b] == -float("inf")).all())
        assert torch.equal(out[b:], good[0][b:])
        cache.ctx_len.copy_(keep)


def test_many_sequences_and_loose_bounds():
    """More sequences than lanes, lengths that differ a hundredfold, bounds far above the lengths."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(15)
    lens = [(int(3000 * float(torch.rand(1, generator=gen)) ** 6), 1 + i % 2) for i in range(150)]
    cache, table, off, N = make_cache(gen, lens, 16, 1, 64, BF16)
    q = randn(gen, N, 2, 64)
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse)
    cache.max_new, cache.max_len = 4000, 1 << 30
    o2, l2, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == 0
    check(cache, table, off, lens, q, o2, l2)


def test_strides_streams_and_workspace():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(16)
    lens = [(900, 2), (17, 30)]
    cache, table, off, N = make_cache(gen, lens, 32, 2, 128, BF16)
    base = randn(gen, 8, N, 128)
    q = base.transpose(0, 1)                                             # head-major queries
    out = torch.zeros((N, 10, 128), dtype=BF16, device="cuda")[:, 1:9]   # a slice of wider rows
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.full((dsbd.dsbd_paged_attention_workspace_bytes(cache, N, 8),), 255, dtype=torch.uint8, device="cuda")
    _, lse, fault = dsbd.dsbd_paged_attention(cache, q, out=out, workspace=ws, stream=side)
    side.synchronize()
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse)
    again = dsbd.dsbd_paged_attention(cache, q.contiguous(), want_lse=False)
    assert again[1] is None and torch.equal(again[0], out)
    with pytest.raises(dsbd.DsbdError) as e:
        dsbd.dsbd_paged_attention(cache, q, workspace=ws[:-256])
    assert e.value.code == -3


def test_captured_calls_follow_their_inputs():
    """Append and attention in a graph, replayed with other lengths, tables and rows between eager calls."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(17)
    lens = [(47, 1), (703, 1), (47, 1)]
    cache, table, off, N = make_cache(gen, lens, 16, 2, 128, BF16)
    q, k, v = randn(gen, N, 8, 128), randn(gen, N, 2, 128), randn(gen, N, 2, 128)
    f, s = dsbd.rope_inv_freq(128)
    prep = dsbd.QKPrep(inv_freq=f, rot_scale=s)

    def step():
        qo, _ = dsbd.dsbd_paged_append(cache, k, v, q=q, prep=prep)
        return dsbd.dsbd_paged_attention(cache, qo)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse, fault = step()
    for i in range(4):
        for t in (q, k, v):
            t.copy_(randn(gen, *t.shape))
        cache.ctx_len.copy_(torch.tensor([[40, 700, 5], [41, 701, 6], [2, 30, 47], [47, 350, 0]][i], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = step()
        assert int(fault) == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
