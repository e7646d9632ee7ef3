"""Handles that work their tensors out when they are asked for them: the call holds them until it returns."""
import torch

import pytest

from test_gpu_logits import setup
from test_gpu_qk_rows import BF16, make_cache, prep_for, randn

pytestmark = pytest.mark.gpu


def on_demand(handle, names):
    """The same handle, whose attributes of these names are new tensors every time."""
    kept = {n: getattr(handle, n) for n in names}

    class Made(type(handle)):
        def __init__(self):
            self.__dict__.update({k: v for k, v in handle.__dict__.items() if k not in names})

        def __getattribute__(self, n):
            if n in kept:
                torch.zeros(7)                       # (what was made before and not held is gone by now)
                return None if kept[n] is None else kept[n].view(kept[n].shape)
            return super().__getattribute__(n)
    return Made()


def test_cache_and_preparation():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(95)
    cache, table, off, N = make_cache(gen, [(40, 3), (7, 30)], 16, 2, 64, BF16)
    q, k, v = randn(gen, N, 4, 64), randn(gen, N, 2, 64), randn(gen, N, 2, 64)
    prep = prep_for(gen, 64, 64, "heads", False, 4, 2, BF16)
    late = on_demand(cache, ("k_pages", "v_pages", "page_table", "ctx_len", "q_off")), on_demand(prep, ("q_weight", "k_weight", "inv_freq"))
    want = dsbd.dsbd_paged_append(cache, k, v, q=q, prep=prep)[0]
    pages = cache.k_pages.clone()
    got = dsbd.dsbd_paged_append(late[0], k, v, q=q, prep=late[1])[0]
    assert torch.equal(got, want) and torch.equal(cache.k_pages, pages)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    for a, b in zip(dsbd.dsbd_qk_norm_rope(q, k, pos, late[1], v=v), dsbd.dsbd_qk_norm_rope(q, k, pos, prep, v=v)):
        assert torch.equal(a, b)
    assert dsbd.dsbd_paged_attention_workspace_bytes(late[0], N, 4) == dsbd.dsbd_paged_attention_workspace_bytes(cache, N, 4)
    for a, b in zip(dsbd.dsbd_paged_attention(late[0], got), dsbd.dsbd_paged_attention(cache, got)):
        assert torch.equal(a, b)


def test_forest_and_rules():
    import paper_2409_16560_amd as dsbd
    forest, z, rules, _, _ = setup(96, 3000, shared_mask=True)
    want, fault = dsbd.dsbd_process_logits(forest, z, rules)
    got, f2 = dsbd.dsbd_process_logits(on_demand(forest, ("tree_prompt", "tree_off", "parent", "token")), z, on_demand(rules, tuple(rules.__dict__)))
    assert int(fault) == int(f2) == 0 and torch.equal(got, want)
