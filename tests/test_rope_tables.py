"""Frequency tables whose trained length is short against the wanted numbers of turns."""
import math

import pytest
import torch

import paper_2409_16560_amd as dsbd


@pytest.mark.parametrize("rot,orig,low,high", [(64, 4, 1.0, 32.0), (128, 6, 1.0, 32.0), (64, 4096, 1000.0, 5000.0), (64, 100, 1.0, 32.0),
                                               (64, 4096, 1.0, 32.0), (32, 1 << 20, 2.0, 3.0)])
@pytest.mark.parametrize("kind", ["by_parts", "by_turns"])
def test_pairs_of_few_turns_are_divided_and_those_of_many_left(kind, rot, orig, low, high):
    plain = dsbd.rope_inv_freq(rot, 10000.0, device="cpu")[0]
    f, _ = dsbd.rope_inv_freq(rot, 10000.0, kind, 8.0, orig_len=orig, low=low, high=high, device="cpu")
    turns = orig * plain / (2 * math.pi)
    assert torch.allclose(f[turns <= low], plain[turns <= low] / 8, rtol=1e-14)
    assert torch.allclose(f[turns >= high], plain[turns >= high], rtol=1e-14)
    assert bool((f <= plain * (1 + 1e-14)).all()) and bool((f >= plain / 8 * (1 - 1e-14)).all())
