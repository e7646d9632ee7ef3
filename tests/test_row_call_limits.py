"""Numbers behind which 32-bit indices of the calls on rows, pages and logits would run over: refused, on the host."""
import pytest

import paper_2409_16560_amd.binding as b
from test_row_call_refusals import P, cache, forest, prep, rows, rules

FAR = (1 << 30) + 1


@pytest.mark.parametrize("kw", [dict(n_seqs=FAR), dict(max_len=FAR), dict(page_size=FAR), dict(n_seqs=(1 << 31) - 1)])
def test_caches(kw):
    lib = b.load_library()
    assert lib.dsbd_paged_append(cache(**kw), 2, 8, 2, 128, 0, rows(), rows(), rows(), None, prep(), rows(), P, None) == -2
    assert lib.dsbd_paged_attention(cache(**kw), 2, 8, 2, 128, 0, rows(), 0.0, None, rows(), None, P, 1 << 62, P, None) == -2


@pytest.mark.parametrize("f,r", [({}, dict(hist=P, hist_off=P, n_hist=FAR)), ({}, dict(hist=P, hist_off=P, n_hist=(1 << 31) - 1)),
                                 ({}, dict(bias_off=P, bias_token=P, bias_value=P, n_bias=FAR)), (dict(n_trees=FAR), {})])
def test_logits(f, r):
    assert b.load_library().dsbd_process_logits(forest(**f), None, 3, 100, 2, P, 100, rules(**r), P + 65536, 100, P, None) == -2
