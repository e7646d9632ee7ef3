"""How the attention of many rows over pages is cut up: parts against the places that the device has, blocks of rows handed out
longest first, and faults in what the lengths and offsets say.

A workspace of the caller's begins with two numbers per (row, head), whose second one says in how many parts the row was taken.
Outputs are checked as in test_gpu_paged_attention, whose tolerances hold here too."""
import numpy as np
import pytest
import torch

from test_gpu_paged_attention import check, trees
from test_gpu_qk_rows import BF16, F16, make_cache, randn

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


def chunks(seed, count, lo, hi, far, longest=None):
    rng = np.random.default_rng(seed)
    lens = [(int(rng.integers(0, far)), int(rng.integers(lo, hi + 1))) for _ in range(count)]
    lens[0] = (lens[0][0], hi)
    if longest:
        lens[count // 2] = (longest, lens[count // 2][1])
    lens[3] = (lens[3][0], 0)                                 # one without new tokens
    return lens


# lens, query and KV heads, rows of a block, a tree's mask, whether units may be split
FIRST = {
    "128 rows, trees, cut": (chunks(1, 34, 17, 31, 700, 5000), 64, 16, 128, True, True),
    "128 rows, trees, whole": (chunks(2, 44, 17, 31, 700), 64, 16, 128, True, False),
    "128 rows, short, whole": (chunks(3, 34, 17, 31, 220), 64, 16, 128, False, False),
    "128 rows, chunks, cut": (chunks(4, 34, 17, 31, 700, 5000), 64, 16, 128, False, True),
    "256 rows, trees, cut": (chunks(5, 34, 33, 64, 900, 6000), 32, 8, 256, True, True),
    "256 rows, chunks": (chunks(6, 6, 300, 700, 900, 3000), 32, 8, 256, False, True),
    "256 rows, chunks, cut": (chunks(6, 8, 250, 600, 900, 9000), 32, 8, 256, False, True),
    "256 rows, chunks, whole": (chunks(7, 6, 300, 900, 300), 32, 32, 256, False, False),
}


def cut_a_quarter_above(lens, new, G, Hk, rows, tree):
    """Parts of every (sequence, block, KV head): a unit of more than 5/4 of an even share of all tiles is cut into shares of that
    size.  (A sequence of a bad length, given as (0, 0) with new rows all the same, has units of one tile.)"""
    tiles = []
    for (c, n), m in zip(lens, new):
        last = [(min(r + rows, m * G) - 1) // G for r in range(0, m * G, rows)]
        tiles.append([1 if n == 0 else -(-(c + (n if tree else t + 1)) // 64) for t in last])
    # (the share goes by the first block and the last: what lies between them counts as their mean)
    seen = sum(len(t) * (t[0] + t[-1]) / 2 for t in tiles if t) * Hk
    cut = max(int(np.ceil(1.25 * seen / PLACES[rows])), 4)
    return [[1 + (x - 1) // cut for x in t for _ in range(Hk)] for t in tiles]


@pytest.mark.parametrize("spoilt", [False, True], ids=["good", "one bad length"])
@pytest.mark.parametrize("lens,Hq,Hk,rows,tree,splits", FIRST.values(), ids=FIRST.keys())
def test_more_units_than_places_of_a_few_sequences(lens, Hq, Hk, rows, tree, splits, spoilt):
    """Units are handed out longest first, what is far longer than the others in parts."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(53)
    cache, table, off, N = make_cache(gen, lens, 16, Hk, 64, F16 if Hk == 32 else BF16, front=2, behind=3)
    block, units, may = shape_of(cache, N, Hq, Hk)
    assert block == rows and may == splits and units > PLACES[rows] and len(lens) <= 64
    q, anc = randn(gen, N, Hq, 64, dtype=cache.k_pages.dtype), None
    if tree:
        anc = np.concatenate([np.zeros(2, np.uint64), trees(gen, lens), np.zeros(3, np.uint64)])
    if spoilt:
        cache.ctx_len[1], lens = -5, lens[:1] + [(0, 0)] + lens[2:]
    out, lse, fault, parts = run(cache, q, anc)
    assert fault == (dsbd.DSBD_FAULT_BOUNDS if spoilt else 0)
    a, b = int(off[0]), int(off[-1])
    for t in (out, lse):                                      # every row is written, and nothing else
        assert bool((t[:a] == 1000).all()) and bool((t[b:] == 1000).all()) and not bool((t[a:b] == 1000).any())
    if spoilt:
        a, b = int(off[1]), int(off[2])
        assert b > a and bool((out[a:b] == 0).all()) and bool((lse[a:b] == -float("inf")).all())
    check(cache, table, off, lens, q, out, lse, anc=anc, rows=4 if tree or rows == 128 else 14)
    if splits:
        assert parts_of_units(cache, parts, Hq, Hk, rows) == cut_a_quarter_above(lens, np.diff(off), Hq // Hk, Hk, rows, tree)


FAULTY = {
    "128 rows, may be split": ([(50, 20), (20, 30), (300, 12)], 32, 25, 128),
    "128 rows, whole": ([(50, 20), (20, 30), (100, 12)], 32, 25, 128),
    "256 rows, may be split": ([(50, 70), (20, 100), (300, 66)], 110, 80, 256),
    "256 rows, whole": ([(50, 70), (20, 100), (100, 66)], 110, 80, 256),
}


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lens,loose,tight,rows", FAULTY.values(), ids=FAULTY.keys())
def test_bad_lengths_and_offsets_where_rows_share_tiles(lens, loose, tight, rows, dtype):
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(54)
    Hq, Hk = 8, 2
    cache, table, off, N = make_cache(gen, lens, 16, Hk, 64, dtype, front=1, behind=2)
    cache.max_new, splits = loose, cache.max_len > 256
    q = randn(gen, N, Hq, 64, dtype=dtype)
    others = [lens[0], (0, 0), lens[2]]
    a, b = int(off[1]), int(off[2])

    def zeros_in_the_middle(how):
        assert shape_of(cache, N, Hq, Hk)[::2] == (rows, splits), how
        out, lse, fault, _ = run(cache, q)
        assert fault == dsbd.DSBD_FAULT_BOUNDS, how
        check(cache, table, off, others, q, out, lse, rows=8)
        assert bool((out[a:b] == 0).all()) and bool((lse[a:b] == -float("inf")).all()), how
        for t in (out, lse):
            assert bool((t[:1] == 1000).all()) and bool((t[-2:] == 1000).all()), how

    out, lse, fault, _ = run(cache, q)
    assert fault == 0
    check(cache, table, off, lens, q, out, lse, rows=8)
    for bad in (-1, cache.max_len - (b - a) + 1, 1 << 30, (1 << 31) - 1, -(1 << 31)):
        cache.ctx_len[1] = bad
        zeros_in_the_middle(bad)
    cache.ctx_len[1] = lens[1][0]
    cache.max_new = tight                                     # the second has more
    zeros_in_the_middle("max_new")
    cache.max_new = loose
    # the second ends in front of its beginning, the third begins inside the first
    n = lens[0][1]
    cache.q_off[2] = 1 + n - 8
    assert int(cache.q_off[3]) - (1 + n - 8) > loose
    out, lse, fault, _ = run(cache, q)
    assert fault == dsbd.DSBD_FAULT_BOUNDS
    check(cache, table, off, lens[:1], q, out, lse, front=n - 8)
    for bad in (N + 1, (1 << 31) - 1, -1):                    # rows that the call does not have
        cache.q_off[2] = bad
        out, lse, fault, _ = run(cache, q)
        assert fault == dsbd.DSBD_FAULT_BOUNDS
        check(cache, table, off, lens[:1], q, out, lse, rows=8)
        for t in (out, lse):
            assert bool((t[:1] == 1000).all()) and bool((t[-2:] == 1000).all())
