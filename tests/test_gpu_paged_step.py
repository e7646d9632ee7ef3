"""A serving step on paged caches, call behind call: the prompts' chunk, single tokens of beams that share the prompt's pages, a
draft forest (through the pages and through the forest attention), rules on its logits and the verification; and calls at the
edges of what the attention takes.

Attention is checked as in test_gpu_paged_attention, whose tolerances hold here too; rules and verification by their oracles."""
import numpy as np
import pytest
import torch

from oracle import logit_rules as o_rules
from test_gpu_paged_attention import check
from test_gpu_qk_rows import BF16, F16, close, logical, make_cache, prep_for, randn, want_rows

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def tokens_of(pages, table, page, s, a, b):
    t = torch.arange(a, b)
    return pages[torch.from_numpy(table)[s, t // page].long().cuda(), (t % page).cuda()]


@pytest.mark.parametrize("D,Hq,Hk,page", [(128, 8, 2, 16), (64, 4, 4, 32)])
def test_prompts_tokens_forest_rules_verification(D, Hq, Hk, page):
    import gpu_util as gu
    import paper_2409_16560_amd as dsbd
    from dsbd_synth import make_workload
    from oracle import forest as o_forest
    gen = torch.Generator().manual_seed(31)
    w = make_workload("c4", n_prompts=2, V=257, L=(5, 9), Hq=Hq, Hkv=Hk)
    d = gu.DeviceWorkload(w)
    prompt_len, more = [3 * page + 5, 7], 4                          # tokens of the prompts, tokens that every beam adds
    T, P = w.n_trees, w.n_prompts
    prep = prep_for(gen, D, D, "heads", False, Hq, Hk, BF16)
    x = lambda n: (lambda r: (r[:, :Hq], r[:, Hq:Hq + Hk], r[:, Hq + Hk:]))(randn(gen, n, Hq + 2 * Hk, D))
    per = -(-(max(prompt_len) + more + w.max_tree_nodes) // page)
    pool = P * per + T * per
    kp, vp = (torch.full((pool, page, Hk, D), float("nan"), dtype=BF16, device="cuda") for _ in range(2))

    # the prompts, a chunk each
    table = np.arange(P * per, dtype=np.int32).reshape(P, per)
    off = np.concatenate([[0], np.cumsum(prompt_len)])
    cache = dsbd.PagedKV(kp, vp, i32(table), i32([0] * P), i32(off), max_new=max(prompt_len), max_len=max(prompt_len))
    q, k, v = x(off[-1])
    held_k, held_v = [k[off[p]:off[p + 1]] for p in range(P)], [v[off[p]:off[p + 1]] for p in range(P)]
    qo, fault = dsbd.dsbd_paged_append(cache, k, v, q=q, prep=prep)
    out, lse, f2 = dsbd.dsbd_paged_attention(cache, qo)
    assert int(fault) == int(f2) == 0
    check(cache, table, off, [(0, n) for n in prompt_len], qo, out, lse, rows=12)

    # beams: whole pages are shared, the last one is copied
    of = [int(p) for p in w.tree_prompt]
    beams = np.zeros((T, per), dtype=np.int32)
    for b in range(T):
        whole = prompt_len[of[b]] // page
        beams[b, :whole] = table[of[b], :whole]
        beams[b, whole:] = P * per + b * per + np.arange(per - whole)
        for pages in (kp, vp):
            pages[int(beams[b, whole])] = pages[int(table[of[b], whole])]
    keys, values = [[held_k[of[b]]] for b in range(T)], [[held_v[of[b]]] for b in range(T)]
    ctx = np.array([prompt_len[of[b]] for b in range(T)])
    cache = dsbd.PagedKV(kp, vp, i32(beams), i32(ctx), i32(np.arange(T + 1)), max_new=1, max_len=max(prompt_len) + more)
    for _ in range(more):
        q, k, v = x(T)
        qo, fault = dsbd.dsbd_paged_append(cache, k, v, q=q, prep=prep)
        out, lse, f2 = dsbd.dsbd_paged_attention(cache, qo)
        assert int(fault) == int(f2) == 0
        check(cache, beams, np.arange(T + 1), [(int(c), 1) for c in ctx], qo, out, lse)
        for b in range(T):
            keys[b].append(k[b:b + 1]); values[b].append(v[b:b + 1])
        cache.ctx_len += 1
        ctx += 1
    for b in range(T):                                               # what lies in the pages is what went in
        n = int(ctx[b])
        close(tokens_of(kp, beams, page, b, 0, n), *want_rows(torch.cat(keys[b]), np.arange(n), prep, prep.k_weight))
        assert torch.equal(tokens_of(vp, beams, page, b, 0, n), torch.cat(values[b]))

    # the forest's nodes: in front of the forest attention, and through the pages
    q, k, v = x(w.n_nodes)
    tree = o_forest.tree_of_node(w.tree_off, w.n_nodes)
    depth = np.zeros(w.n_nodes, dtype=np.int64)
    for i, a in enumerate(w.parent):
        depth[i] = 0 if a < 0 else depth[a] + 1
    pos = i32(ctx[tree] + depth)
    qo, ko, vo = dsbd.dsbd_qk_norm_rope(q, k, pos, prep, v=v)
    kv = dsbd.PrefixKV([tokens_of(kp, beams, page, b, 0, int(ctx[b])) for b in range(T)],
                       [tokens_of(vp, beams, page, b, 0, int(ctx[b])) for b in range(T)])
    anc = torch.zeros(w.n_nodes, dtype=torch.int64, device="cuda")
    one, one_lse, fault = dsbd.dsbd_forest_attention(d.forest, kv, qo, ko, vo, anc_mask_out=anc)
    assert int(fault) == 0
    cache = dsbd.PagedKV(kp, vp, i32(beams), i32(ctx), d.forest.tree_off, max_new=w.max_tree_nodes,
                         max_len=int(ctx.max()) + w.max_tree_nodes)
    q2, fault = dsbd.dsbd_paged_append(cache, k, v, q=q, positions=pos, prep=prep)
    assert torch.equal(q2, qo)
    for b in range(T):
        a, e = int(w.tree_off[b]), int(w.tree_off[b + 1])
        assert torch.equal(tokens_of(kp, beams, page, b, int(ctx[b]), int(ctx[b]) + e - a), ko[a:e])
    two, two_lse, f2 = dsbd.dsbd_paged_attention(cache, q2, anc_mask=anc)
    assert int(fault) == int(f2) == 0
    lens = [(int(ctx[b]), int(w.tree_off[b + 1] - w.tree_off[b])) for b in range(T)]
    check(cache, beams, np.asarray(w.tree_off), lens, qo, two, two_lse, anc=anc.cpu().numpy().view(np.uint64))
    assert float((one.float() - two.float()).abs().max()) <= gu.ATOL and float((one_lse - two_lse).abs().max()) <= gu.ATOL

    # rules on both models' logits, then the verification of what they leave
    rng = np.random.default_rng(32)
    mask = rng.random((w.n_nodes, 257)) < 0.8
    lens = rng.integers(1, 40, T)
    rule = dict(hist=rng.integers(0, 257, lens.sum()), hist_off=np.concatenate([[0], np.cumsum(lens)]), prompt_len=lens // 2,
                repetition=np.float32([1.3, 0.9]), frequency=np.float32([0.2, 0.0]), presence=np.float32([0.1, 0.4]),
                temperature=np.float32([0.8, 1.2]))
    f32 = lambda a: torch.from_numpy(a).cuda()

    def through_the_rules(z):
        bits = np.zeros((w.n_nodes, 9 * 32), dtype=bool)
        bits[:, :257] = mask
        rules = dsbd.LogitRules(i32(rule["hist"]), i32(rule["hist_off"]), i32(rule["prompt_len"]), f32(rule["repetition"]),
                                f32(rule["frequency"]), f32(rule["presence"]), f32(rule["temperature"]),
                                mask=torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).cuda())
        want, size = o_rules.process(z.double().cpu().numpy(), np.arange(w.n_nodes), w.tree_prompt, w.tree_off, w.parent, w.token, mask=mask, **rule)
        out, fault = dsbd.dsbd_process_logits(d.forest, z, rules)
        got = out.cpu().numpy()
        assert int(fault) == 0 and (np.isinf(got) == ~mask).all()
        assert (np.abs(got[mask] - want[mask]) <= 8 * 2.0 ** -24 * size[mask]).all()
        return out
    raw = d.logits_p, d.logits_q
    d.logits_p, d.logits_q = (through_the_rules(z) for z in raw)
    assert int(d.verify().fault) & dsbd.DSBD_FAULT_NONFINITE         # a grammar that excludes drafted tokens is a mistake
    for i, a in enumerate(w.parent):
        if a >= 0:
            mask[a, w.token[i]] = True
    d.logits_p, d.logits_q = (through_the_rules(z) for z in raw)
    w.logits_p, w.logits_q = d.logits_p.cpu().numpy(), d.logits_q.cpu().numpy()
    res = d.verify()
    torch.cuda.synchronize()
    gu.compare_verify(res, gu.oracle_verify(w), w)


def steep(gen, shape, dtype):
    """Multiples of 1/16 up to 4: 128 products of two of them add up exactly in fp32."""
    return (randn(gen, *shape, dtype=torch.float32) * 16).round().clamp(-64, 64).div(16).to(dtype)


RAMPS = {
    "up": lambda t, n: t / n,
    "down": lambda t, n: 1 - t / n,
    "one token far above": lambda t, n: (t == n * 5 // 7).float(),
    "first seen far above, last further": lambda t, n: 0.5 * (t == 1).float() + (t == n - 2).float(),
    "saw": lambda t, n: (t % 97) / 97 * (t / n),
}


@pytest.mark.parametrize("ramp", RAMPS.values(), ids=RAMPS.keys())
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lens,Hq,Hk,D", [([(1500, 1), (299, 1)], 4, 1, 128), ([(700, 5)], 8, 2, 64), ([(900, 30)], 4, 1, 128), ([(130, 300)], 2, 2, 128)],
                         ids=["16 rows", "32 rows", "128 rows", "more"])
def test_scores_that_climb(lens, Hq, Hk, D, dtype, ramp):
    """Scores hundreds apart: references are raised, steeply and late, and numerators vanish.  Products and sums are exact, so what a
    score of up to 4 * 31 + 40 (as a power of two 240) is off by is the rounding of its scaling, 240 * 3 * 2^-24: 5e-5."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(33)
    cache, table, off, N = make_cache(gen, lens, 16, Hk, D, dtype)
    cache.k_pages.copy_(steep(gen, cache.k_pages.shape, dtype))
    for s, (c, n) in enumerate(lens):
        t = torch.arange(c + n)
        up = (ramp(t.float(), c + n) * 248).round().div(8).to(dtype).cuda()       # multiples of 1/8 up to 31
        cache.k_pages[torch.from_numpy(table)[s, t // 16].long().cuda(), (t % 16).cuda(), :, 0] = up[:, None]
    q = steep(gen, (N, Hq, D), dtype)
    q[:, :, 0] = 4
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q, scale=1.0)
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse, scale=1.0, rows=16)


def test_offsets_that_do_not_ascend_and_chunks_above_the_bound():
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(34)
    for Hq, Hk, max_new in (8, 2, 4), (8, 2, 40):                    # either kernel
        lens = [(50, 3), (20, 4), (300, 2)]
        cache, table, off, N = make_cache(gen, lens, 16, Hk, 64, BF16)
        cache.max_new = max_new
        q = randn(gen, N, Hq, 64)
        good = dsbd.dsbd_paged_attention(cache, q)
        assert int(good[2]) == 0
        cache.q_off[1], cache.q_off[2] = 7, 3                        # 0 7 3 9: the second has none, the others more than they hold
        cache.max_new, out, lse = 8, torch.full_like(q, 5.0), torch.full((N, Hq), 5.0, device="cuda")
        _, _, fault = dsbd.dsbd_paged_attention(cache, q, out=out, lse=lse)
        assert int(fault) == dsbd.DSBD_FAULT_BOUNDS
        cache.q_off.copy_(i32([0, 3, 100, 9]))                       # rows that the call does not have
        _, _, fault = dsbd.dsbd_paged_attention(cache, q, out=out, lse=lse)
        assert int(fault) == dsbd.DSBD_FAULT_BOUNDS
        check(cache, table, [0, 3], lens[:1], q, out, lse)           # (another bound, another kernel: not the same roundings)
        cache.q_off.copy_(i32(off))
        cache.max_new = 3                                            # the second sequence has more: rows of 0, all of them
        out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
        assert int(fault) == dsbd.DSBD_FAULT_BOUNDS and bool((out[3:7] == 0).all()) and bool((lse[3:7] == -float("inf")).all())
    lens = [(300, 1), (10, 60), (40, 1)]                             # far more rows than the kernel's block has
    cache, table, off, N = make_cache(gen, lens, 16, 1, 64, BF16)
    q, cache.max_new = randn(gen, N, 4, 64), 2
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == dsbd.DSBD_FAULT_BOUNDS and bool((out[1:61] == 0).all()) and bool((lse[1:61] == -float("inf")).all())
    check(cache, table, off, [(300, 1), (0, 0), (40, 1)], q, out, lse)


@pytest.mark.parametrize("Hq,Hk,n", [(4, 2, 1), (8, 2, 6)])
def test_ranges_over_many_sequences(Hq, Hk, n):
    """Ranges of steps that take in many short sequences, begin and end inside long ones, with empty ones between; more than 64."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(35)
    lens = [(4000, n), (0, 0), (0, n)] + [(5 + i % 40, n if i % 7 else 0) for i in range(130)] + [(2500, n), (31, n), (33, 0)]
    cache, table, off, N = make_cache(gen, lens, 16, Hk, 64, F16)
    q = randn(gen, N, Hq, 64, dtype=F16)
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse)


def test_a_page_in_several_places():
    """Two sequences with one table, and a table that names one page again and again."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(36)
    lens = [(200, 1), (200, 1), (330, 1)]
    cache, table, off, N = make_cache(gen, lens, 16, 2, 128, BF16)
    table[1] = table[0]
    table[2, :15] = table[2, 0]
    cache.page_table.copy_(torch.from_numpy(table))
    q = randn(gen, N, 8, 128)
    q[1] = q[0]
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == 0 and torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])
    check(cache, table, off, lens, q, out, lse)


def test_two_streams_at_once_and_two_graphs_of_one_pool():
    """Calls on two streams with workspaces of their own; two graphs that share a memory pool, replayed in turn."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(37)
    sets = []
    for lens, Hq in ([(3000, 1), (700, 1)], 8), ([(2000, 31)], 16):
        cache, table, off, N = make_cache(gen, lens, 16, 2, 128, BF16)
        q = randn(gen, N, Hq, 128)
        sets.append((cache, q, dsbd.dsbd_paged_attention(cache, q)))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (cache, q, _) in enumerate(sets):
            got[i].append(dsbd.dsbd_paged_attention(cache, q, stream=streams[i]))
    torch.cuda.synchronize()
    for i, (_, _, want) in enumerate(sets):
        for g in got[i]:
            assert int(g[2]) == 0 and torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])
    graphs, outs, pool = [], [], None
    for cache, q, _ in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            outs.append(dsbd.dsbd_paged_attention(cache, q))
        pool = g.pool()
        graphs.append(g)
    for turn in range(3):
        for i, (cache, q, _) in enumerate(sets):
            q.mul_(-1 if turn else 1)
            graphs[i].replay()
            torch.cuda.synchronize()
            a, b = outs[i][0].clone(), outs[i][1].clone()
            want = dsbd.dsbd_paged_attention(cache, q)
            assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.parametrize("lens,Hq,Hk", [([(260 + 7 * (i % 11), 1) for i in range(150)], 16, 8), ([(400, 1), (90, 1)], 80, 40),
                                        ([(0, 0)] + [(300 + i, 9 + i % 5) for i in range(72)], 32, 8), ([(2, 140), (900, 130)], 24, 24)],
                         ids=["more sequences than are cut", "40 heads", "many trees", "many heads of a chunk"])
def test_many_units(lens, Hq, Hk):
    """Calls with enough (sequence, KV head) to fill the device, which split nothing, and head numbers that divide it unevenly."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(38)
    cache, table, off, N = make_cache(gen, lens, 16, Hk, 64, BF16)
    q = randn(gen, N, Hq, 64)
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == 0
    check(cache, table, off, lens, q, out, lse, rows=3)


@pytest.mark.parametrize("n", [1, 12, 90])
def test_tokens_behind_the_tables_end(n):
    """A table that ends inside a sequence: its further tokens count as not there, and are reported."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(39)
    lens = [(500, n), (100, n)]
    cache, table, off, N = make_cache(gen, lens, 16, 2, 128, F16)
    table = np.ascontiguousarray(table[:, :14])
    cache.page_table = torch.from_numpy(table).cuda()
    q = randn(gen, N, 4, 128, dtype=F16)
    out, lse, fault = dsbd.dsbd_paged_attention(cache, q)
    assert int(fault) == dsbd.DSBD_FAULT_BOUNDS
    check(cache, table, off, lens, q, out, lse, rows=8)
