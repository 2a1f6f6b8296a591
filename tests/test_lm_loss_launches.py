"""Which launches the cross entropy over a vocabulary takes, and each of them against the definition in 64 bits."""
import ctypes as C

import pytest
import torch

import paper_2407_20761_amd as ob
from test_lm_loss import DEV, U, Call, _some_rows, expected

gpu = pytest.mark.gpu


def _plan(n, H, V):
    return ob.ob_lm_loss_plan(ob.make_lm_loss_desc(H, V), n)


# ---- every kind of tile ------------------------------------------------------------------------------

# (rows, all tokens, hidden, vocabulary) -> tiles of the forward's logits, pieces, tiles of the logits of a piece, of the last, of dx's sums, of dw
LAUNCHES = [
    ((2100, 2100, 1024, 16384), (256, 1, 256, 256, 0, 256)),           # whole columns of tiles, ragged rows
    ((2060, 5000, 1024, 16385), (256, 1, 256, 256, 0, 128)),           # ragged both ways, listed rows
    ((2049, 2049, 4096, 8200), (256, 1, 256, 256, 0, 128)),
    ((2100, 2100, 256, 16384), (128, 1, 128, 128, 0, 128)),
    ((257, 300, 768, 2001), (64, 1, 64, 64, 0, 128)),
    ((4100, 4100, 64, 131080), (128, 2, 128, 128, 64, 128)),
    ((4100, 4200, 1024, 131080), (256, 2, 256, 256, 128, 256)),
    ((4100, 4100, 2048, 131080), (256, 2, 256, 256, 256, 256)),
    ((9000, 9000, 1024, 120001), (256, 3, 256, 256, 256, 256)),        # the sums of three pieces
    ((4800, 4800, 512, 1009), (128, 1, 128, 128, 0, 64)),
]


@pytest.mark.parametrize("sizes,want", LAUNCHES)
def test_which_launches_a_case_takes(sizes, want):
    n, _, H, V = sizes
    p = _plan(n, H, V)
    assert (p.fwd_tile, p.pieces, p.piece_tile, p.last_tile, p.dx_tile, p.dw_tile) == want


@gpu
@pytest.mark.parametrize("sizes", [s for s, _ in LAUNCHES])
def test_every_launch(sizes):
    n, T, H, V = sizes
    c = Call(T, H, V, rows=None if n == T else _some_rows(T, n), seed=n).run()
    c.check()
    first = c.dx.clone(), c.dw.clone()
    for t in (c.dx, c.dw):
        t.fill_(float("nan"))
    c.bwd()
    assert torch.equal(first[0], c.dx) and torch.equal(first[1], c.dw)


@gpu
def test_accumulation_over_pieces_in_the_largest_tiles():
    c = Call(4100, 2048, 131080, seed=3)
    old = torch.randn(c.dw.shape, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).bfloat16() * 0.1
    c.fwd()
    c.dw.copy_(old)
    c.bwd(ob.OB_BWD_ACCUMULATE)
    value, bound = expected(c.w, c.x, c.labels, c.dnll, U)["dw"]
    value = value + old.double()
    assert float(((c.dw.double() - value).abs() / (bound + U * value.abs())).max()) <= 1


# ---- limits ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("H", [64, 128, 256, 320, 4096])
@pytest.mark.parametrize("n,V", [(1 << 22, 1 << 17), (1 << 18, 1 << 21), ((1 << 21) + 1, (1 << 17) + 3), (1 << 22, 1 << 16)])
def test_every_size_that_is_taken_can_be_launched(n, V, H):
    """a launch has fewer than 2^32 threads, 256 to a workgroup: one of more is an error when the call comes to it"""
    assert n * V <= 1 << 39
    assert _plan(n, H, V).fwd_workgroups * 256 < 1 << 32


@gpu
def test_more_logits_than_a_launch_of_small_tiles_has_threads_for():
    """17 GB of maxima and sums: the forward, a few of its rows"""
    n, H, V = (1 << 21) + 3, 64, (1 << 17) + 5
    assert n * V > 1 << 38
    print(f"lm loss: n={n} H={H} V={V}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, w = (torch.randn(s, generator=gen, device=DEV).bfloat16() for s in ((n, H), (V, H)))
    w /= 8
    labels = torch.randint(0, V, (n,), generator=gen, device=DEV, dtype=torch.int32)
    desc = ob.make_lm_loss_desc(H, V)
    nll, lse = (torch.full((n,), float("nan"), device=DEV) for _ in range(2))
    ws = torch.empty(ob.ob_lm_loss_workspace_bytes(desc, n), dtype=torch.uint8, device=DEV)
    ob.ob_lm_loss_fwd(desc, w, x, n, None, labels, nll, lse, ws)
    at = torch.cat([torch.arange(40, device=DEV), torch.randint(0, n, (60,), generator=gen, device=DEV), torch.arange(n - 40, n, device=DEV)])
    want = expected(w, x[at], labels[at], torch.zeros(len(at), device=DEV), U)
    for name, got in (("nll", nll), ("lse", lse)):
        value, bound = want[name]
        assert float(((got[at].double() - value).abs() / bound).max()) <= 1, name
    assert torch.isfinite(nll).all() and torch.isfinite(lse).all()


def test_refusals_of_the_plan():
    out, desc = ob.ob_lm_loss_launch(), ob.make_lm_loss_desc(64, 100)
    call = lambda d, n, o: ob.lib.ob_lm_loss_plan(d, n, o)
    assert call(C.byref(desc), 5, C.byref(out)) == ob.OB_OK and out.fwd_tile > 0
    assert call(C.byref(desc), 5, None) == ob.OB_EINVAL and call(None, 5, C.byref(out)) == ob.OB_EINVAL
    assert call(C.byref(desc), 0, C.byref(out)) == ob.OB_EINVAL and call(C.byref(desc), (1 << 22) + 1, C.byref(out)) == ob.OB_EINVAL
    assert call(C.byref(ob.make_lm_loss_desc(64, 100, ob.OB_FP32)), 5, C.byref(out)) == ob.OB_EINVAL
    assert call(C.byref(ob.make_lm_loss_desc(100, 100)), 5, C.byref(out)) == ob.OB_EUNSUPPORTED
