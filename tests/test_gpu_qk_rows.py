"""Norm and rotation of the rows of q and k, and their way into the pages of a cache, against the formulas in 64 bits.

A result is off by the rounding to its type, half a step (eps / 2 of it), and by what fp32 makes of the formula: the
sum of D <= 256 squares and the root 256 * 2^-24, sines and products a few 2^-24, all of the pair's length: 2.1e-5 of it."""
import numpy as np
import pytest
import torch

from oracle import paged as o_paged
from oracle import qk_rows as o_rows

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def np64(t):
    return t.detach().double().cpu().numpy()


def close(got, want, size):
    eps = torch.finfo(got.dtype).eps
    off = np.abs(np64(got) - want)
    tol = eps / 2 * np.abs(want) + 2.1e-5 * size + torch.finfo(got.dtype).smallest_normal * eps
    assert (off <= tol).all(), (float((off / tol).max()), np.argwhere(off > tol)[:4].tolist())


def randn(gen, *shape, dtype=BF16, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float32) * scale).to(dtype).cuda()


def prep_for(gen, D, rot, norm, interleaved, Hq, Hk, dtype, scaling=None):
    import paper_2409_16560_amd as dsbd
    f, s = dsbd.rope_inv_freq(rot, 10000.0, scaling, 4.0 if scaling else 1.0, orig_len=512) if rot else (None, 1.0)
    qw = kw = None
    if norm in ("shared", "heads"):
        qw = randn(gen, *((Hq, D) if norm == "heads" else (D,)), dtype=dtype)
        kw = randn(gen, *((Hk, D) if norm == "heads" else (D,)), dtype=dtype)
    return dsbd.QKPrep(norm=norm != "none", q_weight=qw, k_weight=kw, eps=1e-5, inv_freq=f, rot_scale=s, interleaved=interleaved)


def want_rows(x, pos, prep, w):
    return o_rows.qk_rows(np64(x), pos, None if prep.inv_freq is None else np64(prep.inv_freq), prep.rot_scale, prep.interleaved,
                          prep.norm, None if w is None else np64(w), prep.eps)


@pytest.mark.parametrize("D,rot", [(16, 16), (64, 64), (64, 32), (80, 80), (96, 48), (112, 0), (128, 128), (128, 64), (256, 256), (208, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm,N,Hq,Hk,dtype", [("none", 1, 4, 4, BF16), ("shared", 67, 6, 2, F16), ("heads", 5, 40, 3, BF16), ("plain", 9, 1, 1, F16)])
def test_rows_against_the_formula(D, rot, interleaved, norm, N, Hq, Hk, dtype):
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(D * 7 + rot)
    x = randn(gen, N, Hq + 2 * Hk, D, dtype=dtype)           # one projection: the rows are its slices
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    prep = prep_for(gen, D, rot, norm, interleaved, Hq, Hk, dtype)
    pos = torch.randint(0, 9000, (N,), generator=gen, dtype=torch.int32)
    before = x.clone()
    qo, ko, vo = dsbd.dsbd_qk_norm_rope(q, k, pos.cuda(), prep, v=v)
    assert torch.equal(x, before) and torch.equal(vo, v) and qo.is_contiguous() and ko.is_contiguous()
    close(qo, *want_rows(q, pos.numpy(), prep, prep.q_weight))
    close(ko, *want_rows(k, pos.numpy(), prep, prep.k_weight))


def test_far_and_negative_positions_and_scaled_tables():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(1)
    pos = torch.tensor([0, 1, -1, -5000, 131071, 1 << 20, (1 << 31) - 1, -(1 << 31)], dtype=torch.int64).to(torch.int32)
    for scaling in (None, "linear", "base", "by_parts", "by_turns"):
        q, k = randn(gen, 8, 3, 128), randn(gen, 8, 1, 128)
        prep = prep_for(gen, 128, 128, "shared", False, 3, 1, BF16, scaling)
        qo, ko, _ = dsbd.dsbd_qk_norm_rope(q, k, pos.cuda(), prep)
        close(qo, *want_rows(q, pos.numpy(), prep, prep.q_weight))
        close(ko, *want_rows(k, pos.numpy(), prep, prep.k_weight))


def test_in_place_head_major_single_inputs_and_other_streams():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(2)
    N, Hq, Hk, D = 33, 4, 2, 64
    prep = prep_for(gen, D, 64, "shared", True, Hq, Hk, F16)
    pos = torch.arange(N, dtype=torch.int32)
    qh, kh = randn(gen, Hq, N, D, dtype=F16), randn(gen, Hk, N, D, dtype=F16)      # head-major tensors
    q, k = qh.transpose(0, 1), kh.transpose(0, 1)
    wq, wk = want_rows(q, pos.numpy(), prep, prep.q_weight), want_rows(k, pos.numpy(), prep, prep.k_weight)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    alone = dsbd.dsbd_qk_norm_rope(q, None, pos.cuda(), prep, stream=side)
    side.synchronize()
    assert alone[1] is None and alone[2] is None
    close(alone[0], *wq)
    out = dsbd.dsbd_qk_norm_rope(q, k, pos.cuda(), prep, q_out=q, k_out=k)
    assert out[0].data_ptr() == qh.data_ptr()
    close(qh.transpose(0, 1), *wq)
    close(kh.transpose(0, 1), *wk)
    e = torch.empty((0, Hq, D), dtype=F16, device="cuda")
    assert dsbd.dsbd_qk_norm_rope(e, None, torch.empty(0, dtype=torch.int32, device="cuda"), prep)[0].shape == (0, Hq, D)


def test_a_broadcast_row_and_extreme_values():
    """One row for all tokens (stride 0); rows of zeros, of large values and of NaN: every row by itself."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(3)
    one = randn(gen, 1, 2, 128).expand(50, 2, 128)
    prep = prep_for(gen, 128, 128, "shared", False, 2, 2, BF16)
    pos = torch.arange(50, dtype=torch.int32)
    close(dsbd.dsbd_qk_norm_rope(one, None, pos.cuda(), prep)[0], *want_rows(one, pos.numpy(), prep, prep.q_weight))
    x = randn(gen, 4, 2, 128)
    x[0] = 0
    x[1] = 1e15
    x[2, 0, 5] = float("nan")
    out = dsbd.dsbd_qk_norm_rope(x, None, pos[:4].cuda(), prep)[0]
    assert bool((out[0] == 0).all()) and bool(out[2, 0].isnan().all())
    keep = [0, 1, 3]
    close(out[keep], *want_rows(x[keep], pos.numpy()[keep], prep, prep.q_weight))
    close(out[2:3, 1:], *want_rows(x[2:3, 1:], pos.numpy()[2:3], prep, prep.q_weight))


# ------------------------------------------------------------------------------------------------ into the pages

def make_cache(gen, lens, page, Hk, D, dtype, head_major=False, front=0, behind=0, extra=2):
    """Pages filled with random values, tables in random order; lens: (ctx, new) of every sequence."""
    import paper_2409_16560_amd as dsbd
    need = [max(1, -(-(c + n) // page)) for c, n in lens]
    total = sum(need) + extra
    ids = torch.randperm(total, generator=gen)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = ids[at:at + m].to(torch.int32)
        at += m
    shape = (total, Hk, page, D) if head_major else (total, page, Hk, D)
    kp, vp = randn(gen, *shape, dtype=dtype), randn(gen, *shape, dtype=dtype)
    off = np.concatenate([[0], np.cumsum([n for _, n in lens])]) + front
    cache = dsbd.PagedKV(kp, vp, table.cuda(), [c for c, _ in lens], off.tolist(), max_new=max(n for _, n in lens),
                         max_len=max(c + n for c, n in lens), head_major=head_major)
    return cache, table.numpy(), off, int(off[-1]) + behind


def logical(pages, head_major):
    return pages.transpose(1, 2) if head_major else pages


@pytest.mark.parametrize("page,head_major", [(1, False), (3, True), (16, False), (16, True), (64, True), (100, False)])
@pytest.mark.parametrize("lens", [[(0, 1)], [(15, 1), (16, 17), (7, 0), (0, 33)], [(i % 37, i % 3) for i in range(200)]], ids=["one", "ragged", "many"])
def test_append_writes_its_tokens_and_nothing_else(page, head_major, lens):
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(page)
    Hq, Hk, D = 6, 2, 64
    cache, table, off, N = make_cache(gen, lens, page, Hk, D, BF16, head_major, front=2, behind=3)
    prep = prep_for(gen, D, 32, "shared", False, Hq, Hk, BF16)
    x = randn(gen, N, Hq + 2 * Hk, D)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    q_out = torch.full((N, Hq, D), 7.0, dtype=BF16, device="cuda")
    want_k, want_v = logical(cache.k_pages, head_major).clone(), logical(cache.v_pages, head_major).clone()
    out, fault = dsbd.dsbd_paged_append(cache, k, v, q=q, prep=prep, q_out=q_out)
    assert int(fault) == 0 and out.data_ptr() == q_out.data_ptr()
    pos = np.zeros(N, dtype=np.int64)
    for s, (c, n) in enumerate(lens):
        pos[off[s]:off[s + 1]] = c + np.arange(n)
    wk, sk = want_rows(k, pos, prep, prep.k_weight)
    got_k, got_v = logical(cache.k_pages, head_major), logical(cache.v_pages, head_major)
    for s, (c, n) in enumerate(lens):
        for i in range(n):
            p, slot = o_paged.place(table, page, s, c + i)
            row = int(off[s]) + i
            close(got_k[p, slot], wk[row], sk[row])
            assert torch.equal(got_v[p, slot], v[row])
            want_k[p, slot], want_v[p, slot] = got_k[p, slot], got_v[p, slot]
    assert torch.equal(got_k, want_k) and torch.equal(got_v, want_v)          # every other slot as it was
    a, b = int(off[0]), int(off[-1])
    close(out[a:b], *[t[a:b] for t in want_rows(q, pos, prep, prep.q_weight)])
    assert bool((out[:a] == 7).all()) and bool((out[b:] == 7).all())          # padding as it was


def test_append_plain_copy_and_given_positions():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(4)
    cache, table, off, N = make_cache(gen, [(5, 4), (20, 7)], 16, 2, 128, F16)
    k, v = randn(gen, N, 2, 128, dtype=F16), randn(gen, N, 2, 128, dtype=F16)
    out, fault = dsbd.dsbd_paged_append(cache, k, v)
    assert out is None and int(fault) == 0
    for s, (c, n) in enumerate([(5, 4), (20, 7)]):
        for i in range(n):
            p, slot = o_paged.place(table, 16, s, c + i)
            assert torch.equal(cache.k_pages[p, slot], k[off[s] + i]) and torch.equal(cache.v_pages[p, slot], v[off[s] + i])
    prep = prep_for(gen, 128, 128, "none", True, 2, 2, F16)
    pos = torch.tensor([5, 6, 6, 7, 20, 21, 21, 21, 22, 22, 23], dtype=torch.int32)     # a tree's depths
    dsbd.dsbd_paged_append(cache, k, v, positions=pos.cuda(), prep=prep)
    wk, sk = want_rows(k, pos.numpy(), prep, None)
    for s, (c, n) in enumerate([(5, 4), (20, 7)]):
        for i in range(n):
            p, slot = o_paged.place(table, 16, s, c + i)
            close(cache.k_pages[p, slot], wk[off[s] + i], sk[off[s] + i])


def test_append_reports_bad_pages_and_lengths_and_stores_nothing_there():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(5)
    lens = [(14, 4), (3, 2), (0, 5), (31, 1)]
    for what in ("page", "negative", "table", "ctx", "max_new"):
        cache, table, off, N = make_cache(gen, lens, 16, 2, 64, BF16)
        k, v, q = randn(gen, N, 2, 64), randn(gen, N, 2, 64), randn(gen, N, 4, 64)
        kp = cache.k_pages.clone()
        lost = {0: (2, 3)}                              # sequence: its tokens that are not stored
        if what == "page":
            cache.page_table[0, 1] = cache.k_pages.shape[0]
        elif what == "negative":
            cache.page_table[0, 1] = -7
        elif what == "table":
            cache.ctx_len[0], cache.max_len, lost = 31, 64, {0: (1, 2, 3)}      # tokens 32 .. behind a table of two pages
            cache.page_table[0, 1] = cache.page_table[0, 0]
        elif what == "ctx":
            cache.ctx_len[0], lost = -3, {0: (0, 1, 2, 3)}
        else:
            cache.max_new, lost = 4, {2: (0, 1, 2, 3, 4)}
        out, fault = dsbd.dsbd_paged_append(cache, k, v, q=q)
        assert int(fault) == dsbd.DSBD_FAULT_BOUNDS, what
        assert torch.equal(out, q), what
        ctx, table = cache.ctx_len.tolist(), cache.page_table.cpu().numpy()
        for s, (_, n) in enumerate(lens):
            for i in range(n):
                if i not in lost.get(s, ()):
                    p, slot = o_paged.place(table, 16, s, ctx[s] + i)
                    assert torch.equal(cache.k_pages[p, slot], k[off[s] + i]), (what, s, i)
                    kp[p, slot] = k[off[s] + i]
        assert torch.equal(cache.k_pages, kp), what


def test_offsets_beyond_32_bits():
    """A pool of 5 GiB: element offsets of its last pages pass 2^31."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(6)
    n_pages = 21000
    kp = torch.empty((n_pages, 64, 16, 128), dtype=BF16, device="cuda")
    vp = torch.empty((n_pages, 64, 16, 128), dtype=BF16, device="cuda")
    assert kp.numel() > 1 << 31
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    cache = dsbd.PagedKV(kp, vp, table, [100], [0, 40], max_new=40, max_len=140)
    for p in table[0].tolist():
        kp[p].normal_()
        vp[p].normal_()
    k, v, q = randn(gen, 40, 16, 128), randn(gen, 40, 16, 128), randn(gen, 40, 16, 128)
    _, fault = dsbd.dsbd_paged_append(cache, k, v)
    assert int(fault) == 0
    assert torch.equal(kp[3, 36:], k[:28]) and torch.equal(kp[n_pages - 2, :12], k[28:]) and torch.equal(vp[n_pages - 2, :12], v[28:])
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    small = dsbd.PagedKV(kp[table[0].long()].clone(), vp[table[0].long()].clone(), [[0, 1, 2]], [100], [0, 40], max_new=40, max_len=140)
    o2, l2, _ = dsbd.dsbd_paged_attention(small, q)
    assert int(fault) == 0 and torch.equal(out, o2) and torch.equal(lse, l2)
