"""Rows of logits that belong to no node of the forest."""
import pytest
import torch

from test_gpu_logits import close, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_a_row_of_no_node_is_copied_whatever_its_mask(dtype, shared):
    import paper_2409_16560_amd as dsbd
    forest, z, rules, rn, want = setup(23, 5000, dtype=dtype, rows=12, shared_mask=shared)
    if shared:
        rules.mask_row[0] = rules.mask_row[5] = rules.mask_row[11] = 0       # (a mask that leaves nothing)
        want["mask_row"][[0, 5, 11]] = 0
    for i, bad in ((0, -1), (5, 1 << 20), (11, forest.n_nodes)):
        rn[i] = bad
    out, fault = dsbd.dsbd_process_logits(forest, z, rules, row_node=rn)
    assert int(fault) == dsbd.DSBD_FAULT_TOPOLOGY
    for i in (0, 5, 11):
        assert torch.equal(out[i], z[i].float())
    rest = [i for i in range(12) if i not in (0, 5, 11)]
    pick = dict(want, rows=want["rows"][rest], mask=want["mask"] if shared else want["mask"][rest],
                mask_row=want["mask_row"][rest] if shared else None)
    close(out[rest], z[rest], pick)
