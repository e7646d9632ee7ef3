"""Rules on logits, to the last bit: a quotient is off by half a step (2^-24 of it, 2^-150 below the normal numbers)."""
import numpy as np
import pytest
import torch

from oracle import logit_rules as o_rules
from test_gpu_logits import setup

pytestmark = pytest.mark.gpu


def half_a_step(got, want):
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -150).all(), float(np.abs(got / want - 1).max())


# (1e-40 and 2e-38 lie below and just above the smallest normal number; the reciprocals of the last two below it)
@pytest.mark.parametrize("by", [0.7, 1.3, 3.0, 1e-30, 2e-38, 1e-40, 1.7e38, 3.3e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [None, 9])
def test_quotients(by, dtype, rows):
    import paper_2409_16560_amd as dsbd
    forest, z, rules, rn, want = setup(21, 5003, dtype=dtype, rows=rows, masks=False, biases=False)
    if by < 1e-20:
        z.mul_(2.0 ** -10)                                    # (the quotients stay finite)
    by = float(np.float32(by))
    x = z.double().cpu().numpy()
    t = torch.full((3,), by, device="cuda")
    out, fault = dsbd.dsbd_process_logits(forest, z, dsbd.LogitRules(temperature=t), row_node=rn)
    assert int(fault) == 0
    half_a_step(out, x / by)
    r = dsbd.LogitRules(rules.hist, rules.hist_off, rules.prompt_len, repetition=t)
    out, fault = dsbd.dsbd_process_logits(forest, z, r, row_node=rn)
    assert int(fault) == 0
    keep = {k: v for k, v in want.items() if k in ("rows", "tree_prompt", "tree_off", "parent", "token", "hist", "hist_off", "prompt_len")}
    w, _ = o_rules.process(x, repetition=np.full(3, by), **keep)
    assert bool((out.double().cpu().numpy() != x).any())
    fits = np.abs(w) < 3e38
    half_a_step(torch.where(torch.from_numpy(fits).cuda(), out, 0), np.where(fits, w, 0) + 0.0)


def test_values_of_no_positive_number_are_left_out():
    import paper_2409_16560_amd as dsbd
    forest, z, _, _, _ = setup(22, 300, masks=False, biases=False)
    for bad in (0.0, -0.0, -1.0, -1e-40, float("nan"), -float("inf")):
        out, fault = dsbd.dsbd_process_logits(forest, z, dsbd.LogitRules(temperature=torch.full((3,), bad, device="cuda"),
                                                                        repetition=torch.full((3,), bad, device="cuda")))
        assert int(fault) == dsbd.DSBD_FAULT_BOUNDS and torch.equal(out, z)
