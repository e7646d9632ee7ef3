"""How the attention of many rows over pages is cut up: parts against the places that the device has.

A workspace of the caller's begins with two numbers per (row, head), whose second one says in how many parts the row was taken.
Outputs are checked as in test_gpu_paged_attention, whose tolerances hold here too."""
import numpy as np
import pytest
import torch

from test_gpu_paged_attention import check, trees
from test_gpu_qk_rows import BF16, make_cache, randn

pytestmark = pytest.mark.gpu
PLACES = {128: 512, 256: 256}            # workgroups that the device holds, by the rows of a block


def shape_of(cache, N, Hq, Hk):
    """Rows of a block, units (block, KV head), and whether units may be split."""
    G, page = Hq // Hk, cache.k_pages.shape[1]
    most = min(cache.max_new, N) * G
    rows = 128 if most <= 128 else 256
    assert most > 32
    n = np.diff(cache.q_off.cpu().numpy())
    bound = (N * G // rows + len(n)) * Hk
    return rows, int((-(-n * G // rows)).sum()) * Hk, bound < 2 * PLACES[rows] and cache.max_len > 256


def run(cache, q, anc=None, want=1000.0):
    """Outputs, filled with `want` before, and the parts of every (row, head)."""
    import paper_2409_16560_amd as dsbd
    N, Hq, D = q.shape
    ws = torch.zeros(dsbd.dsbd_paged_attention_workspace_bytes(cache, N, Hq), dtype=torch.uint8, device="cuda")
    out, lse = torch.full((N, Hq, D), want, dtype=q.dtype, device="cuda"), torch.full((N, Hq), want, device="cuda")
    a = None if anc is None else torch.from_numpy(anc.view(np.int64)).cuda()
    _, _, fault = dsbd.dsbd_paged_attention(cache, q, anc_mask=a, out=out, lse=lse, workspace=ws)
    parts = ws[:8 * N * Hq].view(torch.int32).view(N, Hq, 2)[..., 1].cpu().numpy() if 8 * N * Hq <= ws.numel() else None
    return out, lse, int(fault), parts


def parts_of_units(cache, parts, Hq, Hk, rows):
    """Parts of every (sequence, block, KV head)."""
    G, off = Hq // Hk, cache.q_off.cpu().numpy()
    return [[int(parts[off[s] + r // G, g * G + r % G]) for r in range(0, (off[s + 1] - off[s]) * G, rows) for g in range(Hk)]
            for s in range(len(off) - 1)]


@pytest.mark.parametrize("lens,Hq,Hk,rows,tree", [([(2000, 31)] * 40, 32, 8, 128, True), ([(2000, 1536)], 32, 8, 256, False),
                                                  ([(1900, 400), (2100, 500), (2000, 600)], 32, 8, 256, False),
                                                  ([(1200, 31)] * 70, 16, 4, 128, True)],
                         ids=["trees", "a chunk", "chunks", "more trees than lanes"])
def test_units_that_fill_more_than_half_of_the_device_are_not_cut_for_a_second_round(lens, Hq, Hk, rows, tree):
    gen = torch.Generator().manual_seed(51)
    cache, table, off, N = make_cache(gen, lens, 16, Hk, 64, BF16)
    block, units, splits = shape_of(cache, N, Hq, Hk)
    assert block == rows and splits and PLACES[rows] < 2 * units <= 2 * PLACES[rows]
    q, anc = randn(gen, N, Hq, 64), trees(gen, lens) if tree else None
    out, lse, fault, parts = run(cache, q, anc)
    assert fault == 0
    check(cache, table, off, lens, q, out, lse, anc=anc, rows=2)
    of = parts_of_units(cache, parts, Hq, Hk, rows)
    assert units <= sum(map(sum, of)) <= PLACES[rows]


def test_a_long_sequence_among_many_short_ones_is_cut():
    gen = torch.Generator().manual_seed(52)
    lens = [(100, 5)] * 150 + [(30000, 5)] + [(100, 5)] * 150
    cache, table, off, N = make_cache(gen, lens, 16, 1, 64, BF16)
    block, units, splits = shape_of(cache, N, 8, 1)
    assert block == 128 and splits and units == 301
    q = randn(gen, N, 8, 64)
    out, lse, fault, parts = run(cache, q)
    assert fault == 0
    check(cache, table, off, lens, q, out, lse, rows=2)
    of = parts_of_units(cache, parts, 8, 1, 128)
    assert sum(map(sum, of)) <= 512 and of[150][0] >= 64      # (470 tiles; 301 of 512 places are the units' own)
