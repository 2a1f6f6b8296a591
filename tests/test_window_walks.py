"""Windowed attention: what the profile counts of it."""
import numpy as np
import pytest
import torch

import paper_2407_20761_amd as ob
from test_window_attention import _call
from window_ref import allowed

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("lens,window,sinks", [([100], 1, 64), ([1000], 16, 64), ([300, 5, 64, 65], 64, 64), ([70, 200], 30, 4), ([40], 100, 7),
                                               ([90, 3], 12, 0), ([50], 20, 50)])
def test_the_profile_counts_the_pairs_that_see_each_other(lens, window, sinks):
    """the work of a class is 4 nq d flops to a (row, key it sees) forward, half of that for dQ and one and a half for dK / dV"""
    c = _call(lens, 2, 1, 64, window, sinks)
    pairs = sum(int(allowed(n, window, sinks).sum()) for n in lens)
    ob.ob_prof_begin(64)
    c.run()
    torch.cuda.synchronize()
    work = {name: v[2] for name, v in ob.ob_prof_end().items()}
    flops = 4.0 * 2 * 64 * pairs
    assert work == {"attn_fwd": flops, "attn_bwd_dq": 0.5 * flops, "attn_bwd_dkv": 1.5 * flops}
