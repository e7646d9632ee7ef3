"""Norm and rotation of bf16 rows whose squares leave fp32's range.  Tolerances as in test_gpu_qk_rows."""
import numpy as np
import pytest
import torch

from test_gpu_qk_rows import BF16, close, prep_for, randn, want_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,rot", [(128, 128), (64, 0), (80, 32), (256, 256)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_far_from_one(D, rot, eps):
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(81)
    powers = [-120, -110, -90, -64, -62, -45, -40, -39, 0, 50, 55, 56, 57, 60, 63, 64, 90, 120, 124]
    x = randn(gen, len(powers), 5, D).clamp_(-4, 4)
    for i, p in enumerate(powers):                     # every power in a token of its own, next to heads of ordinary size
        x[i, ::2] = torch.ldexp(x[i, ::2].float(), torch.tensor(p, device="cuda")).to(BF16)
    prep = prep_for(gen, D, rot, "shared", False, 5, 5, BF16)
    prep.eps = eps
    pos = torch.arange(len(powers), dtype=torch.int32)
    out, _, _ = dsbd.dsbd_qk_norm_rope(x, None, pos.cuda(), prep)
    assert bool(out.isfinite().all())
    close(out, *want_rows(x, pos.numpy(), prep, prep.q_weight))


def test_rows_without_a_size():
    """Zeros stay zeros with eps and are 0/0 without, NaN and Inf make their own row NaN."""
    import paper_2409_16560_amd as dsbd
    gen = torch.Generator().manual_seed(82)
    x = randn(gen, 4, 2, 128)
    x[0], x[1, 0, 3], x[2, 1, 100] = 0, float("inf"), float("nan")
    pos = torch.arange(4, dtype=torch.int32)
    prep = prep_for(gen, 128, 128, "shared", False, 2, 2, BF16)
    for eps in (1e-6, 0.0):
        prep.eps = eps
        out, _, _ = dsbd.dsbd_qk_norm_rope(x, None, pos.cuda(), prep)
        assert bool((out[0] == 0).all() if eps else out[0].isnan().all())
        assert bool(out[1, 0].isnan().any()) and bool(out[2, 1].isnan().all())
        keep = np.array([[False, False], [False, True], [True, False], [True, True]])
        with np.errstate(invalid="ignore"):
            w, size = want_rows(x, pos.numpy(), prep, prep.q_weight)
        close(out[torch.from_numpy(keep).cuda()], w[keep], size[keep])
