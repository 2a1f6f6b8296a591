"""Windowed attention: the walks that long rows, many segments and large scores take, the roundings of its gradients, what the profile counts,
launches that are refused."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2407_20761_amd as ob
import synth_inputs as si
from test_window_attention import DEV, Call, _call, _host_segments, _split
from window_ref import U, allowed

gpu = pytest.mark.gpu


# ---- sinks in chunks -----------------------------------------------------------------------------------

# more segments with chunks than a wave looks at, behind more segments than a round of the search does; chunks of 128 and of 256 rows in one batch
CHUNKED = [([20] * 150 + [200, 20] * 70 + [129, 257, 1, 64, 109], 16, 1, 64, 8, 3, 146), ([20] * 150 + [200, 20] * 70 + [129, 257, 1, 64, 109], 16, 1, 128, 8, 40, 146),
           ([5000, 30, 2500, 4097, 4096], 4, 1, 64, 100, 5, 20 + 20 + 17 + 32), ([30, 2500, 4200], 4, 2, 128, 70, 33, 20 + 17)]


@pytest.mark.parametrize("lens,nq,nkv,d,window,sinks,chunks", CHUNKED)
def test_chunks_of_the_sinks(lens, nq, nkv, d, window, sinks, chunks):
    assert ob.ob_varlen_attn_window_bwd_plan(_host_segments(lens), nq, nkv, d, window, sinks)[2] == chunks


@gpu
@pytest.mark.parametrize("lens,nq,nkv,d,window,sinks", [c[:6] for c in CHUNKED])
def test_sinks_of_many_segments_and_of_mixed_chunks(lens, nq, nkv, d, window, sinks):
    _call(lens, nq, nkv, d, window, sinks, seed=2).run().check()


# ---- long rows -----------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ldq,ldkv,ldo", [(524296, 600008, 540680), (1 << 24, 1 << 24, 1 << 24)])
@pytest.mark.parametrize("lens,nq,nkv,window,sinks", [([7, 130, 1], 2, 1, 40, 3), ([138], 16, 1, 20, 9)])
def test_rows_far_apart(lens, nq, nkv, window, sinks, ldq, ldkv, ldo, d):
    """More than a megabyte from row to row a descriptor serves one tile alone; at the largest stride the offsets in a tile take 32 bits.  The same values in
    compact rows give the same bits"""
    c = _call(lens, nq, nkv, d, window, sinks).run()
    T, wide, narrow = sum(lens), nq * d, nkv * d

    def far(ld, width, values=None):      # (nothing but the rows' own columns is touched)
        t = torch.empty((T - 1) * ld + width, dtype=torch.bfloat16, device=DEV).as_strided((T, width), (ld, 1))
        return t.fill_(float("nan")) if values is None else t.copy_(values)
    q, k, v = (far(ld, w, t) for ld, w, t in zip((ldq, ldkv, ldkv), (wide, narrow, narrow), _split(c.qkv, nq, nkv, d)))
    dq, dk, dv, o, d_o = far(ldq, wide), far(ldkv, narrow), far(ldkv, narrow), far(ldo, wide), far(ldo, wide, c.d_o)
    lse, ws = torch.full_like(c.lse, float("nan")), torch.full_like(c.ws, 255)
    ob.ob_varlen_attn_window_fwd(q, k, v, o, lse, ldq, ldkv, ldo, c.seg, nq, nkv, d, c.scale, window, sinks)
    ob.ob_varlen_attn_window_bwd(d_o, q, k, v, o, lse, dq, dk, dv, ldq, ldkv, ldo, c.seg, nq, nkv, d, c.scale, window, sinks, ws)
    assert torch.equal(o, c.o) and torch.equal(lse, c.lse)
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), _split(c.dqkv, nq, nkv, d)))


# ---- roundings -----------------------------------------------------------------------------------------

def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a)).bfloat16().double().numpy()


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(16, 2), (64, 0), (193, 4), (300, 4), (1000, 0)])
def test_gradients_carry_the_roundings_that_are_said_and_no_more(window, sinks, d):
    """dQ and dK: dS once to bf16, the result once; dV: P once, the result once.  What those leave in norm is worked out here from the same inputs.  P's
    11 bits on its way to dK's dS (1 / 64 of a bf16 rounding's square), Delta from the rounded o behind the short walks (a 100th of dS's at 100 keys) and fp32
    add 2 % at most; one more rounding to bf16 would add 22 %"""
    lens, nq, nkv = [1100, 130], 2, 1
    c = _call(lens, nq, nkv, d, window, sinks).run()
    got, want = c.results(), c.expected()
    T = sum(lens)
    np64 = lambda t: t.double().cpu().numpy().reshape(T, -1, d)
    q, k, v = (np64(t) for t in _split(c.qkv, nq, nkv, d))
    g, err = np64(c.d_o), {n: np.zeros_like(want[n][0]) for n in ("dq", "dk", "dv")}
    for a, b in zip(c.cu[:-1], c.cu[1:]):
        for h in range(nq):
            Q, K, V, G = q[a:b, h], k[a:b, 0], v[a:b, 0], g[a:b, h]
            S = np.where(allowed(b - a, window, sinks), c.scale * (Q @ K.T), -np.inf)
            P = np.exp(S - S.max(1, keepdims=True))
            P /= P.sum(1, keepdims=True)
            dS = P * (G @ V.T - (G * (P @ V)).sum(1, keepdims=True))
            e = _bf16(dS) - dS
            err["dq"][a:b, h] = c.scale * e @ K
            err["dk"][a:b, 0] += c.scale * e.T @ Q
            err["dv"][a:b, 0] += (_bf16(P) - P).T @ G
    for n, e in err.items():
        ref = want[n][0]
        assert np.linalg.norm(got[n] - ref) <= 1.04 * np.hypot(np.linalg.norm(_bf16(ref) - ref), np.linalg.norm(e)), n


# ---- large scores --------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_large_scores(d):
    """scores of +-1000: most probabilities are 0 or 1, which P on its way to dS holds as 2^15"""
    c = _call([300, 5], 2, 1, d, 40, 4)
    c.scale = 20.0 * (128 / d) ** 0.5
    c.run()
    got, want, T = c.results(), c.expected(), 305
    np64 = lambda t: t.double().cpu().numpy().reshape(T, -1, d)
    q, k, v = (np64(t) for t in _split(c.qkv, 2, 1, d))
    g = np64(c.d_o)
    bound = {n: u * np.abs(want[n][0]) + 1e-6 for n, u in (("dq", U), ("dk", U), ("dv", U))}
    for a, b in zip(c.cu[:-1], c.cu[1:]):
        for h in range(2):
            Q, K, V, G = q[a:b, h], k[a:b, 0], v[a:b, 0], g[a:b, h]
            see, S = allowed(b - a, 40, 4), c.scale * (Q @ K.T)
            # a score, d / 16 sums one after the other, is off by d / 16 times 2^-24 of its terms' sum, in the log-sum-exp and in the probability, which are
            # rounded themselves
            eps = c.scale * (np.abs(Q) @ np.abs(K).T) * (d / 16) * 2.0 ** -24
            eps = np.where(see, eps + np.where(see, eps, 0).max(1, keepdims=True) + 4 * 2.0 ** -24 * np.where(see, np.abs(S), 0).max(1, keepdims=True), 0)
            S = np.where(see, S, -np.inf)
            P = np.exp(S - S.max(1, keepdims=True))
            P /= P.sum(1, keepdims=True)
            P_err = P * np.expm1(eps) + 2.0 ** -24
            dP, dP_mag, o_mag = G @ V.T, np.abs(G) @ np.abs(V).T, (np.abs(G) * (P @ np.abs(V))).sum(1, keepdims=True)
            delta = (G * (P @ V)).sum(1, keepdims=True)
            # Delta from o: the errors of P, its rounding, o's own
            delta_err = (np.abs(G) * (P_err @ np.abs(V))).sum(1, keepdims=True) + 2 * U * o_mag
            dS = P * (dP - delta)
            dS_err = P_err * (np.abs(dP - delta) + delta_err) + P * (delta_err + 2e-4 * (dP_mag + o_mag)) + (U + 2.0 ** -11) * np.abs(dS)
            bound["dq"][a:b, h] += c.scale * dS_err @ np.abs(K) * (1 + U)
            bound["dk"][a:b, 0] += c.scale * dS_err.T @ np.abs(Q) * (1 + U)
            bound["dv"][a:b, 0] += (P_err + (U + 2.0 ** -11) * P).T @ np.abs(G) * (1 + U)
    for n, e in bound.items():
        assert float((np.abs(got[n] - want[n][0]) / e).max()) <= 1, n


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_scores_at_the_limit(d):
    """Whole numbers times 1024, up to 2^20 and exact: every row takes the largest alone, or those that share it.

    The log-sum-exp is ((m s) + log2 l) ln 2, s the scale times log2 e: the floats of log2 e and ln 2 are off by -1.34e-8 and 2.7e-9 of their values, the scale
    is a power of two, the sum and the product are rounded, 2^-24 each.  Together 2 x 2^-24 + 1.1e-8 = 1.31e-7 of it.
    The backward takes exp2(score s - lse log2 e), whose second product is rounded once more: 3 x 2^-24 + 1.1e-8 of 2^20 log2 e = 1.513e6 makes 0.287, a
    factor of up to 1.22"""
    lens, nq, nkv, window, sinks = [300, 5], 2, 1, 50, 3
    c = _call(lens, nq, nkv, d, window, sinks)
    q, k, _ = _split(c.qkv, nq, nkv, d)
    gen = torch.Generator().manual_seed(d)
    T, hot = sum(lens), torch.zeros((sum(lens), nkv, d))
    q.copy_(torch.nn.functional.one_hot(torch.randint(0, 4, (T, nq), generator=gen), d).reshape(T, -1).to(DEV) * 8)
    hot[:, :, :4] = torch.randint(-127, 128, (T, nkv, 4), generator=gen)
    k.copy_(hot.reshape(T, -1).to(DEV))
    c.scale = 1024.0
    c.run()
    got, want = c.results(), c.expected()
    assert np.abs(want["lse"][0]).max() > 0.9 * (1 << 20)
    assert (np.abs(got["lse"] - want["lse"][0]) <= 1.31e-7 * np.abs(want["lse"][0]) + 1e-5).all()
    v = _split(c.qkv, nq, nkv, d)[2].double().cpu().numpy()
    assert np.abs(got["o"] - want["o"][0]).max() <= 2.5 * U * np.abs(v).max()
    assert (np.abs(got["dv"] - want["dv"][0]) <= _spread(c, window, sinks)).all()
    assert all(np.isfinite(t).all() for t in got.values())


def _spread(c, window, sinks):
    """0.22, and three roundings, of the terms of dV"""
    nq, nkv, d = c.dims[:3]
    T = c.qkv.shape[0]
    np64 = lambda t: t.double().cpu().numpy().reshape(T, -1, d)
    q, k, v = (np64(t) for t in _split(c.qkv, nq, nkv, d))
    g, out = np.abs(np64(c.d_o)), np.zeros((T, nkv, d))
    for a, b in zip(c.cu[:-1], c.cu[1:]):
        for h in range(nq):
            S = np.where(allowed(b - a, window, sinks), c.scale * (q[a:b, h] @ k[a:b, 0].T), -np.inf)
            P = np.exp(S - S.max(1, keepdims=True))
            out[a:b, 0] += (P / P.sum(1, keepdims=True)).T @ g[a:b, h]
    return 0.24 * out + 1e-6


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [1e-20, 1e6])
def test_scales_at_their_limits(scale, d):
    """the smallest makes every score 0, against which a masked one has to be far below; at the largest a masked one has to be finite"""
    c = _call([300, 5, 64], 2, 1, d, 40, 4)
    if scale > 1:
        _split(c.qkv, 2, 1, d)[0].mul_(1e-6 * d ** -0.5)
    c.scale = scale
    c.run().check()


# ---- the profile ---------------------------------------------------------------------------------------


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
