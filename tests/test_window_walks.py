"""Windowed attention: what the profile counts of it, launches that are refused."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2407_20761_amd as ob
import synth_inputs as si
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


# ---- launches that there are no threads for: no GPU --------------------------------------------------

def _ones(n):
    seg = ob.Segments(np.arange(n + 1, dtype=np.int32), device=None)
    seg.c.cu_dev = 0x1000
    return seg


@pytest.mark.parametrize("nq,nkv,d,n,fits", [(3, 1, 64, 1 << 22, True), (4, 1, 64, 1 << 22, False), (2, 2, 128, (1 << 22) - 1, True), (4, 4, 128, 1 << 21, False), (2, 2, 128, 1 << 22, False),
                                             (64, 8, 128, 1 << 18, False), (64, 8, 128, 1 << 17, True)])
def test_launches_of_too_many_workgroups_are_refused(nq, nkv, d, n, fits):
    """256 threads to a tile and head; the runtime would run a part of 2^32 threads and more"""
    seg, p, sizes = _ones(n), C.c_void_p(0x1000), (nq * d, nkv * d, nq * d)
    assert (ob.ob_varlen_attn_window_bwd_workspace_bytes(seg, nq, nkv, d, 8, 1) > 0) == fits
    assert ob.ob_varlen_attn_window_bwd_workspace_bytes(seg, nq, nkv, d, 8, 1, ob.OB_FP32) > 0
    desc = ob.make_desc(si.small_shape(hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, mlp_dim=64, mask=si.MASK_CAUSAL))
    attn = ob.BlockAttn(8, 1)
    assert (ob.ob_block_attn_workspace_bytes(desc, attn, seg) > 0) == fits
    if fits:
        return
    w, g, big = ob.ob_block_weights(*[0x1000] * 12), ob.ob_block_grads(*[0x1000] * 12), 1 << 60
    calls = [lambda: ob.lib.ob_varlen_attn_window_fwd(p, p, p, p, p, *sizes, C.byref(seg.c), nq, nkv, d, 0.125, 8, 1, 0, None),
             lambda: ob.lib.ob_varlen_attn_window_bwd(*[p] * 9, *sizes, C.byref(seg.c), nq, nkv, d, 0.125, 8, 1, 0, p, big, None),
             lambda: ob.lib.ob_varlen_attn_fwd(p, p, p, p, p, *sizes, C.byref(seg.c), nq, nkv, d, 0.125, 1, 0, None),
             lambda: ob.lib.ob_block_attn_fwd(C.byref(desc), C.byref(attn.c), C.byref(w), p, p, p, big, C.byref(seg.c), p, big, None),
             lambda: ob.lib.ob_block_attn_bwd(C.byref(desc), C.byref(attn.c), C.byref(w), C.byref(g), 0, p, p, p, p, big, C.byref(seg.c), p, big, None)]
    for call in calls:
        assert call() == ob.OB_EUNSUPPORTED and "too many tiles" in ob.ob_last_error()
