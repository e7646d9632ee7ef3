"""Many trees and prompts under the rules on logits, many sequences in a paged cache: more than the lanes of a wave, and more than their
square.  Tolerances as in test_gpu_logits, test_gpu_qk_rows and test_gpu_paged_attention."""
import numpy as np
import pytest
import torch

from test_gpu_logits import close as logits_close, setup
from test_gpu_paged_attention import check
from test_gpu_qk_rows import BF16, F16, close, make_cache, prep_for, randn, want_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("trees,prompts", [(63, 63), (64, 3), (5, 64), (70, 70), (200, 9), (300, 100)])
@pytest.mark.parametrize("rows", [None, 50])
def test_rules_over_many_trees(trees, prompts, rows):
    import paper_2409_16560_amd as dsbd
    forest, z, rules, rn, want = setup(trees, 4500, trees=trees, max_nodes=5, prompts=prompts, rows=rows, shared_mask=True)
    out, fault = dsbd.dsbd_process_logits(forest, z, rules, row_node=rn)
    assert int(fault) == 0
    logits_close(out, z, want)


@pytest.mark.parametrize("trees", [7, 80])
def test_a_tree_above_the_bound(trees):
    """Rows behind max_tree_nodes stay as they were; the others do not notice."""
    import paper_2409_16560_amd as dsbd
    forest, z, rules, _, want = setup(91, 4500, trees=trees, max_nodes=9, masks=False)
    off = want["tree_off"]
    big = int(np.argmax(np.diff(off)))
    n = int(off[big + 1] - off[big])
    assert n >= 4
    others = np.diff(off).copy()
    others[big] = 0
    forest.max_tree_nodes = max(n - 2, int(others.max()))
    if forest.max_tree_nodes >= n:
        forest.max_tree_nodes = n - 2
    kept = np.concatenate([np.arange(off[t], min(off[t + 1], off[t] + forest.max_tree_nodes)) for t in range(trees)])
    out = torch.full(z.shape, 77.0, device="cuda")
    _, fault = dsbd.dsbd_process_logits(forest, z, rules, out=out)
    assert int(fault) == dsbd.DSBD_FAULT_BOUNDS
    rest = np.setdiff1d(np.arange(len(z)), kept)
    assert len(rest) and bool((out[rest] == 77).all())
    logits_close(out[kept], z[kept], dict(want, rows=kept))


def test_append_and_attention_of_many_sequences():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(92)
    lens = [(i % 19, 1 + i % 2 if i % 5 else 0) for i in range(4500)]
    cache, table, off, N = make_cache(gen, lens, 16, 1, 64, F16, front=1, behind=2)
    x = randn(gen, N, 4, 64, dtype=F16)
    q, k, v = x[:, :2], x[:, 2:3], x[:, 3:]
    prep = prep_for(gen, 64, 64, "none", False, 2, 1, F16)
    qo, fault = dsbd.dsbd_paged_append(cache, k, v, q=q, prep=prep)
    assert int(fault) == 0
    pos, seq = np.zeros(N, dtype=np.int64), np.full(N, -1)
    for s, (c, n) in enumerate(lens):
        pos[off[s]:off[s + 1]], seq[off[s]:off[s + 1]] = c + np.arange(n), s
    live = torch.from_numpy(seq >= 0).cuda()
    page = torch.from_numpy(table[np.maximum(seq, 0), pos // 16]).long().cuda()
    slot = torch.from_numpy(pos % 16).cuda()
    wk, sk = want_rows(k, pos, prep, None)
    wq, sq = want_rows(q, pos, prep, None)
    at = seq >= 0
    close(cache.k_pages[page[live], slot[live]], wk[at], sk[at])
    close(qo[live], wq[at], sq[at])
    assert torch.equal(cache.v_pages[page[live], slot[live]], v[live])
    out, lse, fault = dsbd.dsbd_paged_attention(cache, qo)
    assert int(fault) == 0
    check(cache, table, off, lens, qo, out, lse)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_trees_of_many_sequences(dtype):
    import paper_2409_16560_amd as dsbd
    from test_gpu_paged_attention import trees
    gen = torch.Generator().manual_seed(93)
    lens = [(int(400 * float(torch.rand(1, generator=gen)) ** 3), 9 + i % 11) for i in range(130)]
    cache, table, off, N = make_cache(gen, lens, 8, 2, 64, dtype)
    q, anc = randn(gen, N, 8, 64, dtype=dtype), trees(gen, lens)
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q, anc_mask=torch.from_numpy(anc.view(np.int64)).cuda())
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse, anc=anc, rows=3)
