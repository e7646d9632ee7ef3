"""Rows of q, k and v where one of them has no heads."""
import pytest
import torch

from test_gpu_qk_rows import BF16, close, prep_for, randn, want_rows

pytestmark = pytest.mark.gpu


def test_rows_next_to_a_tensor_without_heads():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(71)
    prep = prep_for(gen, 64, 64, "shared", False, 1, 2, BF16)
    k, v, none = randn(gen, 9, 2, 64), randn(gen, 9, 2, 64), torch.empty((9, 0, 64), dtype=BF16, device="cuda")
    pos = torch.arange(9, dtype=torch.int32)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    q, _, _ = dsbd.dsbd_qk_norm_rope(none, k, pos.cuda(), prep, v=v, k_out=ko, v_out=vo)
    assert q.shape == (9, 0, 64) and torch.equal(vo, v)
    close(ko, *want_rows(k, pos.numpy(), prep, prep.k_weight))
    qo = torch.full_like(k, 7.0)
    out = dsbd.dsbd_qk_norm_rope(k, none, pos.cuda(), prep, v=none, q_out=qo)
    assert out[1].shape == out[2].shape == (9, 0, 64)
    close(qo, *want_rows(k, pos.numpy(), prep, prep.q_weight))
    assert [t.shape for t in dsbd.dsbd_qk_norm_rope(none, none, pos.cuda(), prep, v=none)] == [(9, 0, 64)] * 3


def test_a_cache_without_heads_is_refused():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(72)
    pages = torch.empty((4, 16, 0, 64), dtype=BF16, device="cuda")
    cache = dsbd.PagedKV(pages, pages, [[0, 1]], [3], [0, 2], max_new=2, max_len=32)
    none, q = torch.empty((2, 0, 64), dtype=BF16, device="cuda"), randn(gen, 2, 4, 64)
    with pytest.raises(dsbd.DsbdError):
        dsbd.dsbd_paged_append(cache, none, none, q=q)
    with pytest.raises(dsbd.DsbdError):
        dsbd.dsbd_paged_attention(cache, q)
