"""Varlen attention with a sliding window and sinks: against its definition in 64 bits, and what it refuses."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2407_20761_amd as ob
import synth_inputs as si
from window_ref import F32, U, allowed, window_attention

gpu = pytest.mark.gpu
DEV = "cuda"


def _tensors(T, nq, nkv, d, seed, dtype):
    """rows of one [T, (nq + 2 nkv) d] buffer with columns to spare, and the gradient of o"""
    rng = np.random.default_rng(seed)
    qkv = si.round_to_bf16(rng.standard_normal((T, (nq + 2 * nkv) * d + 16)).astype(np.float32))
    d_o = si.round_to_bf16(rng.standard_normal((T, nq * d)).astype(np.float32))
    return torch.from_numpy(qkv).to(DEV).to(dtype), torch.from_numpy(d_o).to(DEV).to(dtype)


def _split(t, nq, nkv, d):
    return t[:, :nq * d], t[:, nq * d:(nq + nkv) * d], t[:, (nq + nkv) * d:(nq + 2 * nkv) * d]


class Call:
    """One forward and backward, its buffers poisoned beforehand."""

    def __init__(self, qkv, d_o, cu, nq, nkv, d, window, sinks, scale=None):
        self.cu, self.dims = np.asarray(cu, dtype=np.int32), (nq, nkv, d, window, sinks)
        self.qkv, self.d_o, self.scale = qkv, d_o, d ** -0.5 if scale is None else scale
        self.code = ob.OB_BF16 if qkv.dtype == torch.bfloat16 else ob.OB_FP32
        self.seg = ob.Segments(self.cu)
        T = qkv.shape[0]
        nan = lambda *s, dt=qkv.dtype: torch.full(s, float("nan"), dtype=dt, device=DEV)
        self.o, self.lse, self.dqkv = nan(T, nq * d), nan(nq, T, dt=torch.float32), nan(*qkv.shape)
        n = ob.ob_varlen_attn_window_bwd_workspace_bytes(self.seg, nq, nkv, d, window, sinks, self.code)
        assert n > 0
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)

    def fwd(self, stream=None):
        nq, nkv, d, window, sinks = self.dims
        q, k, v = _split(self.qkv, nq, nkv, d)
        ld = self.qkv.stride(0)
        ob.ob_varlen_attn_window_fwd(q, k, v, self.o, self.lse, ld, ld, nq * d, self.seg, nq, nkv, d, self.scale, window, sinks, self.code, stream)

    def bwd(self, stream=None):
        nq, nkv, d, window, sinks = self.dims
        q, k, v = _split(self.qkv, nq, nkv, d)
        ld = self.qkv.stride(0)
        ob.ob_varlen_attn_window_bwd(self.d_o, q, k, v, self.o, self.lse, *_split(self.dqkv, nq, nkv, d), ld, ld, nq * d, self.seg, nq, nkv, d,
                                     self.scale, window, sinks, self.ws, self.code, stream)

    def run(self):
        self.fwd()
        self.bwd()
        return self

    def results(self):
        nq, nkv, d = self.dims[:3]
        T = self.qkv.shape[0]
        np64 = lambda t: t.float().cpu().numpy().astype(np.float64)
        dq, dk, dv = (np64(t).reshape(T, -1, d) for t in _split(self.dqkv, nq, nkv, d))
        return {"o": np64(self.o).reshape(T, nq, d), "lse": np64(self.lse), "dq": dq, "dk": dk, "dv": dv}

    def expected(self):
        nq, nkv, d, window, sinks = self.dims
        T = self.qkv.shape[0]
        np64 = lambda t: t.float().cpu().numpy().astype(np.float64)
        q, k, v = (np64(t).reshape(T, -1, d) for t in _split(self.qkv, nq, nkv, d))
        return window_attention(q, k, v, self.cu, window, sinks, self.scale, np64(self.d_o).reshape(T, nq, d),
                                U if self.code == ob.OB_BF16 else 0.0)

    def check(self):
        got, want = self.results(), self.expected()
        for n, (value, bound) in want.items():
            worst = float((np.abs(got[n] - value) / bound).max())
            assert worst <= 1, n          # (not so for a NaN either)
        assert torch.isnan(self.dqkv[:, -16:].float()).all()        # columns that are not the call's


def _call(lens, nq, nkv, d, window, sinks, seed=0, dtype=torch.bfloat16):
    print(f"window attention: lens={lens} nq={nq} nkv={nkv} d={d} window={window} sinks={sinks} {dtype}", flush=True)
    cu = np.concatenate([[0], np.cumsum(lens)])
    return Call(*_tensors(int(cu[-1]), nq, nkv, d, seed, dtype), cu, nq, nkv, d, window, sinks)


RAGGED = [1, 2, 63, 64, 65, 128, 129, 192, 300, 31]
CASES = [
    # lengths of a tile of keys, of queries, beside them; windows of one row, around a tile, of everything
    (RAGGED, 2, 1, 64, 1, 0), (RAGGED, 2, 1, 64, 1, 1), (RAGGED, 2, 2, 64, 33, 4), (RAGGED, 3, 1, 64, 64, 64), (RAGGED, 2, 1, 64, 65, 63),
    (RAGGED, 2, 1, 64, 128, 0), (RAGGED, 2, 1, 64, 2 ** 31 - 1, 5), (RAGGED, 2, 1, 128, 1, 0), (RAGGED, 2, 1, 128, 7, 64),
    (RAGGED, 4, 2, 128, 64, 1), (RAGGED, 2, 1, 128, 127, 33), (RAGGED, 2, 1, 128, 129, 4), (RAGGED, 2, 2, 128, 300, 16),
    ([1], 1, 1, 64, 1, 0), ([1], 8, 1, 128, 5, 64), ([5], 2, 1, 64, 2, 64), ([2], 2, 1, 128, 1, 1),
    # several chunks of a segment's queries, tiles of the band without a mask, an odd and an even number of masked ones in front
    ([1100], 2, 1, 64, 200, 3), ([1100], 2, 1, 128, 200, 3), ([1500, 257], 4, 1, 64, 513, 16), ([1500, 257], 4, 1, 128, 512, 16),
    ([4200, 150], 1, 1, 64, 70, 9), ([4200, 300], 1, 1, 128, 130, 64),
    ([900], 6, 1, 64, 90, 40), ([900], 6, 1, 128, 447, 64), ([2101], 1, 1, 128, 700, 8), ([2101], 1, 1, 64, 1030, 0),
]


@gpu
@pytest.mark.parametrize("lens,nq,nkv,d,window,sinks", CASES)
def test_forward_and_backward(lens, nq, nkv, d, window, sinks):
    _call(lens, nq, nkv, d, window, sinks, seed=len(lens) + window % 97).run().check()


@gpu
@pytest.mark.parametrize("lens,nq,nkv,d,window,sinks", [([1, 2, 65, 200], 4, 2, 64, 33, 4), ([129, 70], 2, 1, 128, 1, 64), ([300], 2, 2, 64, 400, 0),
                                                        ([77], 3, 1, 128, 20, 1)])
def test_fp32(lens, nq, nkv, d, window, sinks):
    _call(lens, nq, nkv, d, window, sinks, dtype=torch.float32).run().check()


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(2, 0), (3, 1), (12, 0)])
def test_rows_of_few_keys(d, window, sinks):
    """A rounding's error is at most U of the value, spread evenly: U / sqrt(3) in the mean square.  Of dS and of the result that is
    sqrt(2 / 3) U in norm; a Delta from the rounded o alone would be off by more than that at two keys to a row"""
    c = _call([500, 1, 130], 4, 2, d, window, sinks).run()
    got, want = c.results(), c.expected()
    for n in ("dq", "dk", "dv"):
        assert np.linalg.norm(got[n] - want[n][0]) <= (2 / 3) ** 0.5 * U * np.linalg.norm(want[n][0]), n


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_many_segments(d):
    """more segments than the search for a tile looks at in a round, and more tiles than the table of the order of work holds"""
    rng = np.random.default_rng(5)
    _call(rng.integers(1, 40, 700).tolist(), 1, 1, d, 9, 3).run().check()
    _call([130] * 950, 1, 1, d, 100, 2).run().check()


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_a_window_of_the_whole_segment_is_causal_attention(d):
    lens, nq, nkv = [700, 130], 4, 2
    c = _call(lens, nq, nkv, d, 700, 4).run()
    q, k, v = _split(c.qkv, nq, nkv, d)
    ld, T = c.qkv.stride(0), sum(lens)
    o, lse, dqkv = torch.empty_like(c.o), torch.empty_like(c.lse), torch.full_like(c.dqkv, float("nan"))
    ob.ob_varlen_attn_fwd(q, k, v, o, lse, ld, ld, nq * d, c.seg, nq, nkv, d, c.scale, ob.OB_MASK_SEG_CAUSAL)
    ws = torch.empty(ob.ob_varlen_attn_bwd_workspace_bytes(T, nq, nkv, d), dtype=torch.uint8, device=DEV)
    ob.ob_varlen_attn_bwd(c.d_o, q, k, v, o, lse, *_split(dqkv, nq, nkv, d), ld, ld, nq * d, c.seg, nq, nkv, d, c.scale, ob.OB_MASK_SEG_CAUSAL, ws)
    assert torch.equal(c.o, o) and torch.equal(c.lse, lse)
    # (two results within the bound of the same value)
    want = c.expected()
    got, ref = c.results(), [t.float().cpu().numpy().astype(np.float64).reshape(T, -1, d) for t in _split(dqkv, nq, nkv, d)]
    for n, r in zip(("dq", "dk", "dv"), ref):
        assert float((np.abs(got[n] - r) / want[n][1]).max()) <= 2, n


@gpu
@pytest.mark.parametrize("d,window,sinks", [(64, 100, 20), (128, 100, 20), (128, 1000, 0)])
def test_packed_segments_give_what_they_give_alone(d, window, sinks):
    lens, nq, nkv = [257, 1, 700, 64, 333], 4, 2
    c = _call(lens, nq, nkv, d, window, sinks).run()
    for a, n in zip(np.concatenate([[0], np.cumsum(lens)]), lens):
        one = Call(c.qkv[a:a + n].clone(), c.d_o[a:a + n].clone(), [0, n], nq, nkv, d, window, sinks).run()
        assert torch.equal(one.o, c.o[a:a + n]) and torch.equal(one.lse, c.lse[:, a:a + n])
        assert torch.equal(one.dqkv[:, :-16], c.dqkv[a:a + n, :-16])


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nothing_of_another_segment_reaches_a_row(d, bad):
    lens, nq, nkv, at = [150, 40, 333], 2, 1, 150
    c = _call(lens, nq, nkv, d, 50, 4).run()
    keep = [t.clone() for t in (c.o, c.lse, c.dqkv)]
    c.qkv[at:at + 40] = bad
    c.d_o[at:at + 40] = bad
    c.run()
    rows = [r for r in range(sum(lens)) if not at <= r < at + 40]
    for t, k in ((c.o, keep[0]), (c.lse.t(), keep[1].t()), (c.dqkv[:, :-16], keep[2][:, :-16])):
        assert torch.equal(t[rows], k[rows])


@gpu
def test_large_scores():
    """scores of +-1000: the sum of a row is that of its maximum alone"""
    c = _call([300, 5], 2, 1, 128, 40, 4)
    c.scale = 20.0
    c.run()
    got, want = c.results(), c.expected()
    # a score is off by 2^-24 of its terms' sum: up to 20 x 128 x 4 x 4 x 2^-24 = 2.4e-3, which the exponential turns into a factor
    assert np.abs(got["o"] - want["o"][0]).max() <= 2.5 * (U + 3e-3) * 4.5
    assert all(np.isfinite(t).all() for t in got.values())


@gpu
def test_side_stream_and_captured_calls():
    """on a stream of its own, and captured: replayed among eager calls on the same buffers"""
    c = _call([700, 129, 400], 4, 2, 128, 150, 8).run()
    want = [t.clone() for t in (c.o, c.lse, c.dqkv[:, :-16])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (c.o, c.lse, c.dqkv):
        t.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    c.fwd(side)
    c.bwd(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((c.o, c.lse, c.dqkv[:, :-16]), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for turn in range(3):
        for t in (c.o, c.lse, c.dqkv):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((c.o, c.lse, c.dqkv[:, :-16]), want)), turn
        c.run()


@gpu
def test_differences_along_a_direction():
    """fp32: the gradients against the change of <o, d_o> along a direction, h^2 = 1e-6 of curvature and 6e-8 / h of rounding apart"""
    lens, nq, nkv, d, window, sinks = [90, 41], 2, 1, 64, 17, 3
    c = _call(lens, nq, nkv, d, window, sinks, dtype=torch.float32).run()
    way = torch.randn(c.qkv.shape, generator=torch.Generator().manual_seed(1)).to(DEV)
    way[:, -16:] = 0
    h, ends = 1e-3, []
    for sign in (1, -1):
        e = Call(c.qkv + sign * h * way, c.d_o, c.cu, nq, nkv, d, window, sinks)
        e.fwd()
        ends.append((e.o.double() * c.d_o.double()).sum())
    slope = float((ends[0] - ends[1]) / (2 * h))
    grad = c.dqkv.clone()
    grad[:, -16:] = 0
    exact = float((grad.double() * way.double()).sum())
    size = float((grad.double() * way.double()).abs().sum())
    assert abs(slope - exact) <= 2e-4 * size


# ---- the definition, and refusals: no GPU ------------------------------------------------------------

def test_allowed():
    m = allowed(6, 2, 1)
    assert m.astype(int).tolist() == [[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 1, 1, 0, 0, 0], [1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0],
                                      [1, 0, 0, 0, 1, 1]]
    assert F32 < U


def _refusal(status, text, fwd_only=False, **kw):
    a = dict(q=0x1000, k=0x1000, v=0x1000, o=0x1000, lse=0x1000, ldq=128, ldkv=64, ldo=128, nq=2, nkv=1, d=64, scale=0.125, window=4,
             sinks=1, dtype=0, ws=0x1000, ws_bytes=1 << 30, cu=(0, 10))
    a.update(kw)
    seg = ob.Segments(np.array(a["cu"], dtype=np.int32), device=None)
    seg.c.cu_dev = 0x1000
    p = lambda n: C.c_void_p(a[n])
    tail = (a["ldq"], a["ldkv"], a["ldo"], C.byref(seg.c), a["nq"], a["nkv"], a["d"], a["scale"], a["window"], a["sinks"], a["dtype"])
    if not fwd_only:
        st = ob.lib.ob_varlen_attn_window_bwd(p("o"), p("q"), p("k"), p("v"), p("o"), p("lse"), p("q"), p("k"), p("v"), *tail, p("ws"),
                                              a["ws_bytes"], None)
        assert st == status and text in ob.ob_last_error(), ob.ob_last_error()
    if "ws" not in kw and "ws_bytes" not in kw:
        st = ob.lib.ob_varlen_attn_window_fwd(p("q"), p("k"), p("v"), p("o"), p("lse"), *tail, None)
        assert st == status and text in ob.ob_last_error(), ob.ob_last_error()


@pytest.mark.parametrize("status,text,kw", [
    (1, "window 0", {"window": 0}), (1, "window -3", {"window": -3}), (1, "sinks -1", {"sinks": -1}), (3, "sinks 65", {"sinks": 65}),
    (1, "scale", {"scale": 0.0}), (1, "scale", {"scale": -1.0}), (1, "scale", {"scale": float("nan")}), (1, "scale", {"scale": float("inf")}),
    (1, "scale", {"scale": 1e7}), (1, "scale", {"scale": 1e-21}),
    (3, "head_dim 96", {"d": 96}), (1, "multiple", {"nq": 3, "nkv": 2}), (1, "dtype", {"dtype": 2}), (1, "strides", {"ldq": 120}),
    (1, "strides", {"ldkv": 68}), (3, "stride", {"ldo": (1 << 24) + 8}), (2, "length", {"cu": (0, 5, 5)}), (1, "null", {"q": None}),
    (1, "null", {"lse": None}), (1, "aligned", {"k": 0x1008}), (4, "workspace", {"ws": None}), (4, "workspace", {"ws_bytes": 100}),
    (4, "workspace", {"ws": 0x1004}),
])
def test_refusals(status, text, kw):
    _refusal(status, text, **kw)


def test_workspace_bytes():
    seg = lambda *lens: _host_segments(lens)
    size = lambda s, *a: ob.ob_varlen_attn_window_bwd_workspace_bytes(s, *a)
    up = lambda n: (n + 255) // 256 * 256
    rows = 2 * up(1000 * 2 * 4)
    assert size(seg(1000), 2, 1, 64, 1000, 4) == rows                      # no segment is longer than the window
    assert size(seg(1000), 2, 1, 64, 100, 0) == rows                       # no sinks
    assert size(seg(1000), 2, 1, 64, 100, 4) == rows + up(8 * 2 * 4 * 64 * 4)      # eight chunks of 128 queries
    assert size(seg(5000), 2, 1, 64, 100, 4) == 2 * up(5000 * 2 * 4) + up(20 * 2 * 4 * 64 * 4)      # twenty of 256
    assert size(seg(1000), 2, 1, 64, 100, 4, ob.OB_FP32) == up(1000 * 2 * 4)
    assert size(seg(1000), 2, 1, 64, 0, 4) == 0 and size(seg(1000), 2, 1, 96, 5, 4) == 0


def _host_segments(lens):
    s = ob.Segments(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=None)
    s.c.cu_dev = 0x1000
    return s


def _plan(lens, *a):
    launch, threads, chunks = ob.ob_varlen_attn_window_bwd_plan(_host_segments(lens), *a)
    return launch.key_rows, launch.query_rows, threads, chunks


# every kernel of dK / dV has cases in test_forward_and_backward: (its case) -> key rows, query rows, threads, chunks of the sinks
REACHED = [
    (([1100], 2, 1, 64, 200, 3), (64, 64, 256, 9)), (([1500, 257], 4, 1, 64, 513, 16), (64, 64, 256, 12)),
    (([1100], 2, 1, 128, 200, 3), (64, 64, 512, 9)), (([2101], 1, 1, 128, 700, 8), (64, 64, 512, 0)),
    (([900], 6, 1, 128, 447, 64), (64, 64, 512, 8)),
    # a full chip
    (([2000] * 4, 16, 8, 64, 600, 4), (64, 32, 256, 64)), (([2000] * 4, 16, 8, 128, 600, 4), (128, 64, 512, 64)),
    (([1100] * 4, 16, 8, 128, 600, 4), (64, 64, 512, 0)),
]


@pytest.mark.parametrize("case,want", REACHED)
def test_which_kernel_a_case_reaches(case, want):
    lens, nq, nkv, d, window, sinks = case
    assert _plan(lens, nq, nkv, d, window, sinks) == want


@gpu
@pytest.mark.parametrize("lens,nq,nkv,d,window,sinks", [c for c, _ in REACHED[5:]])
def test_full_chip(lens, nq, nkv, d, window, sinks):
    _call(lens, nq, nkv, d, window, sinks).run().check()


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_launch_shapes_give_the_same_bits(d):
    """a segment alone and among enough others to fill the chip, in another shape of dK / dV"""
    lens, nq, nkv, window, sinks = [700, 333, 1290] + [2000] * 5, 16, 8, 600, 20
    assert _plan(lens, nq, nkv, d, window, sinks)[:3] != _plan(lens[:1], nq, nkv, d, window, sinks)[:3]
    c = _call(lens, nq, nkv, d, window, sinks).run()
    for a, n in zip(np.concatenate([[0], np.cumsum(lens)])[:3], lens[:3]):
        one = Call(c.qkv[a:a + n].clone(), c.d_o[a:a + n].clone(), [0, n], nq, nkv, d, window, sinks).run()
        assert torch.equal(one.dqkv[:, :-16], c.dqkv[a:a + n, :-16])
