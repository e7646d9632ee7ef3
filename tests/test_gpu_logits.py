"""Rules on logits against a row-by-row computation in 64 bits.

Every rule is one operation in fp32 (two for the penalties), each off by at most 2^-24 of its result: eight of them, of the sum of
what was added up."""
import numpy as np
import pytest
import torch

from oracle import logit_rules as o_rules

pytestmark = pytest.mark.gpu


def forest_of(rng, trees, max_nodes, prompts, V):
    off, parent = [0], []
    for _ in range(trees):
        n = int(rng.integers(1, max_nodes + 1))
        base = off[-1]
        parent += [-1] + [base + int(rng.integers(0, i)) for i in range(1, n)]
        off.append(base + n)
    token = rng.integers(0, min(V, 12), len(parent))                 # tokens that repeat along the paths
    return (np.sort(rng.integers(0, prompts, trees)), np.array(off), np.array(parent), token)


def setup(seed, V, trees=5, max_nodes=9, prompts=3, dtype=torch.float32, held=60, rows=None, masks=True, biases=True, shared_mask=False):
    import paper_2409_16560_amd as dsbd
    rng = np.random.default_rng(seed)
    tp, off, parent, token = forest_of(rng, trees, max_nodes, prompts, V)
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    f32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.float32, device="cuda")
    forest = dsbd.Forest(tp, off, parent, token, n_prompts=prompts, max_tree_nodes=max_nodes, max_depth=max_nodes,
                         max_prompt_trees=trees, device=torch.device("cuda", 0))
    lens = rng.integers(0, held + 1, trees)
    ho = np.concatenate([[0], np.cumsum(lens)])
    hist = rng.integers(0, V, ho[-1])
    hist[::3] = rng.integers(0, min(V, 12), len(hist[::3]))
    plen = rng.integers(0, held + 6, trees)
    p = {n: np.float32(rng.uniform(*r, prompts)) for n, r in (("repetition", (0.7, 1.5)), ("frequency", (-0.3, 0.6)),
                                                             ("presence", (-0.3, 0.6)), ("temperature", (0.5, 1.5)))}
    nodes = np.arange(len(parent)) if rows is None else rng.integers(0, len(parent), rows)
    bias, bo, bt, bv = None, None, None, None
    if biases:
        cnt = rng.integers(0, 40, prompts)
        bo = np.concatenate([[0], np.cumsum(cnt)])
        bt, bv = rng.integers(0, min(V, 50), bo[-1]), np.float32(rng.normal(0, 4, bo[-1]))     # tokens that come several times
        bias = [list(zip(bt[bo[i]:bo[i + 1]], bv[bo[i]:bo[i + 1]])) for i in range(prompts)]
    mask = mrow = words = None
    if masks:
        n = 3 if shared_mask else len(nodes)
        mask = rng.random((n, V)) < rng.choice([0.02, 0.5, 0.97], (n, 1))
        mask[0] = False
        W = (V + 31) // 32 + 1
        bits = np.zeros((n, W * 32), dtype=bool)
        bits[:, :V] = mask
        words = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
        mrow = rng.integers(-1, n, len(nodes)) if shared_mask else None
    z = torch.tensor(rng.normal(0, 3, (len(nodes), V)), dtype=torch.float32).to(dtype).cuda()
    rules = dsbd.LogitRules(i32(hist), i32(ho), i32(plen), f32(p["repetition"]), f32(p["frequency"]), f32(p["presence"]),
                            f32(p["temperature"]), None if bo is None else i32(bo), None if bo is None else i32(bt),
                            None if bo is None else f32(bv), None if words is None else torch.from_numpy(words.copy()).cuda(),
                            None if mrow is None else i32(mrow))
    want = dict(rows=nodes, tree_prompt=tp, tree_off=off, parent=parent, token=token, hist=hist, hist_off=ho, prompt_len=plen,
                bias=bias, mask=mask, mask_row=mrow, **p)
    return forest, z, rules, (None if rows is None else i32(nodes)), want


def close(out, z, want):
    w, size = o_rules.process(z.double().cpu().numpy(), **want)
    got = out.double().cpu().numpy()
    inf = np.isinf(w)
    assert (got[inf] == w[inf]).all()
    off = np.abs(got[~inf] - w[~inf])
    assert (off <= 8 * 2.0 ** -24 * size[~inf] + 1e-37).all(), float((off / (size[~inf] + 1e-30)).max())


@pytest.mark.parametrize("V", [1, 7, 256, 4096, 4097, 10001, 50273])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rows_of_a_forest(V, dtype):
    import paper_2409_16560_amd as dsbd
    forest, z, rules, rn, want = setup(V, V, dtype=dtype)
    before = z.clone()
    out, fault = dsbd.dsbd_process_logits(forest, z, rules)
    assert int(fault) == 0 and torch.equal(z, before)
    close(out, z, want)


@pytest.mark.parametrize("rows,shared", [(1, False), (40, True), (3, True)])
def test_rows_of_chosen_nodes(rows, shared):
    import paper_2409_16560_amd as dsbd
    for seed in range(3):
        forest, z, rules, rn, want = setup(seed, 9001, trees=7, rows=rows, shared_mask=shared, dtype=torch.bfloat16)
        out, fault = dsbd.dsbd_process_logits(forest, z, rules, row_node=rn)
        assert int(fault) == 0
        close(out, z, want)


def test_each_rule_alone_and_none():
    import paper_2409_16560_amd as dsbd
    forest, z, rules, _, want = setup(5, 5003)
    names = ("repetition", "frequency", "presence", "temperature", "bias", "mask", None)
    for name in names:
        r = dsbd.LogitRules(rules.hist, rules.hist_off, rules.prompt_len)
        w = {k: v for k, v in want.items() if k not in names or k == name}
        if name == "bias":
            r.bias_off, r.bias_token, r.bias_value = rules.bias_off, rules.bias_token, rules.bias_value
        elif name:
            setattr(r, name, getattr(rules, name))
        out, fault = dsbd.dsbd_process_logits(forest, z, r)
        assert int(fault) == 0
        close(out, z, w)
        if name is None:
            assert torch.equal(out, z)
    # no text in front of the roots, no prompt lengths: the paths alone
    r = dsbd.LogitRules(repetition=rules.repetition, frequency=rules.frequency)
    out, fault = dsbd.dsbd_process_logits(forest, z, r)
    assert int(fault) == 0
    close(out, z, {k: v for k, v in want.items() if k in ("rows", "tree_prompt", "tree_off", "parent", "token", "repetition", "frequency")})


def test_in_place_strided_rows_special_values_and_other_streams():
    import paper_2409_16560_amd as dsbd
    inf = float("inf")
    forest, z, rules, _, want = setup(6, 6007)
    z[0, 5], z[1, 6], z[2, 7], z[3] = -inf, inf, -inf, -inf
    wide = torch.full((z.shape[0], 6007 + 13), 9.0, device="cuda")
    wide[:, 3:3 + 6007] = z
    view = wide[:, 3:3 + 6007]                     # rows that no vector load is aligned to
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, fault = dsbd.dsbd_process_logits(forest, view, rules, out=view, stream=side)
    side.synchronize()
    assert out.data_ptr() == view.data_ptr() and int(fault) == 0
    assert bool((wide[:, :3] == 9).all()) and bool((wide[:, 6010:] == 9).all())
    with np.errstate(invalid="ignore"):
        close(out, z, want)
    # NaN behind a mask is -Inf, in front of none it stays
    z[0, :] = float("nan")
    out, _ = dsbd.dsbd_process_logits(forest, z, rules)
    assert bool((out[0] == -inf).all())
    rules.mask = None
    out, _ = dsbd.dsbd_process_logits(forest, z, rules)
    assert bool(out[0].isnan().all()) and not bool(out[1].isnan().any())


def test_faults_leave_their_rule_out():
    import paper_2409_16560_amd as dsbd
    base = dict(seed=7, V=5000)

    def run(change):
        forest, z, rules, rn, want = setup(rows=12, shared_mask=True, **base)
        change(forest, rules, rn, want)
        out, fault = dsbd.dsbd_process_logits(forest, z, rules, row_node=rn)
        return out, int(fault), z, want, rn

    def token(f, r, rn, w):
        r.hist[::2] = 5000
        w["hist"] = np.where(np.arange(len(w["hist"])) % 2 == 0, 4999, w["hist"])
    out, fault, z, want, _ = run(token)
    assert fault == dsbd.DSBD_FAULT_TOKEN
    keep = [v for v in range(4999)]                 # (the oracle counted them at 4999)
    w, size = o_rules.process(z.double().cpu().numpy(), **want)
    got = out.double().cpu().numpy()
    fin = np.isfinite(w[:, keep])
    assert (np.abs(got[:, keep][fin] - w[:, keep][fin]) <= 8 * 2.0 ** -24 * size[:, keep][fin]).all()

    def heat(f, r, rn, w):
        r.temperature[:] = 0
        r.repetition[:] = -1
        w["temperature"] = w["repetition"] = None
    out, fault, z, want, _ = run(heat)
    assert fault == dsbd.DSBD_FAULT_BOUNDS
    close(out, z, want)

    def mask(f, r, rn, w):
        r.mask_row[:] = 1 << 20
        w["mask"] = None
    out, fault, z, want, _ = run(mask)
    assert fault == dsbd.DSBD_FAULT_BOUNDS
    close(out, z, want)

    def offsets(f, r, rn, w):
        r.hist_off[-1] = 1 << 30
        r.bias_off[:] = torch.tensor([3, 2, 1, -9], dtype=torch.int32)
        w["bias"] = None
        w["hist_off"] = np.concatenate([w["hist_off"][:-1], w["hist_off"][-2:-1]])
    out, fault, z, want, _ = run(offsets)
    assert fault == dsbd.DSBD_FAULT_BOUNDS
    close(out, z, want)

    def node(f, r, rn, w):
        rn[0], rn[5] = -1, 1 << 20
        r.mask = r.mask_row = None
    out, fault, z, want, rn = run(node)
    assert fault == dsbd.DSBD_FAULT_TOPOLOGY
    assert torch.equal(out[0], z[0].float()) and torch.equal(out[5], z[5].float())


def test_captured_call_and_long_texts():
    import paper_2409_16560_amd as dsbd
    forest, z, rules, rn, want = setup(8, 20011, trees=3, held=9000, prompts=1, dtype=torch.bfloat16)
    first, fault = dsbd.dsbd_process_logits(forest, z, rules)
    close(first, z, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, fault = dsbd.dsbd_process_logits(forest, z, rules)
    for i in range(3):
        z.copy_(torch.randn(z.shape, device="cuda"))
        rules.hist.copy_(torch.randint(0, 20011, rules.hist.shape, device="cuda", dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        eager, f2 = dsbd.dsbd_process_logits(forest, z, rules)
        assert int(fault) == int(f2) == 0 and torch.equal(out, eager)
