"""The gradients of the cross entropy over a vocabulary in norm: no more than the rounding of the results and of the entries of G beside the labels, whatever the rows'
weights, and the same label in many rows."""
import pytest
import torch

import paper_2407_20761_amd as ob
from test_lm_loss import DEV, Call

gpu = pytest.mark.gpu


def _bf16(t):
    return t.bfloat16().double()


def _bounds(c, x, w):
    """(value, error in norm that G's rounding to bf16 leaves everywhere but at the labels) of dx and dw, from the inputs"""
    z = x @ w.t()
    P = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
    has = (c.labels >= 0) & (c.labels < c.V)
    hot = torch.zeros_like(z).scatter_(1, torch.where(has, c.labels, 0).long()[:, None], has.double()[:, None])
    weight = torch.where(has, c.dnll.double(), torch.zeros_like(c.dnll.double()))[:, None]
    G = torch.where(has[:, None], (P - hot) * weight, 0.0)
    lost = (_bf16(G) - G) * (1 - hot)
    return {"dx": (G @ w, (lost @ w).norm()), "dw": (G.t() @ x, (lost.t() @ x).norm())}


def _factor(c, name):
    """What is left besides is 2^-8 of what a label's entry lost, fp32's sums and the exponentials' errors: 2 % cover them.  And the roundings of a value and of one next to it
    are two samples: the norm of N errors spread evenly scatters by 0.45 / sqrt(N) of itself, the difference of two by 0.63; six times that"""
    has = (c.labels >= 0) & (c.labels < c.V)
    rows = int(has.sum()) if name == "dx" else len(c.labels[has].unique())
    return 1.02 + 4 / (rows * c.x.shape[1]) ** 0.5


def _off(got, value, number=True):
    e = (got.double() - value).norm()
    return float(e) if number else e


def _check(c):
    rows = c.listed()
    want = _bounds(c, c.x[rows].double(), c.w.double())
    for n, got in (("dx", c.dx[rows]), ("dw", c.dw)):
        value, err = want[n]
        assert _off(got, value) <= _factor(c, n) * float(torch.hypot(_off(_bf16(value), value, False), err)) + 3e-5 * float(value.norm()), n


SIZES = [(60, 256, 32003), (990, 768, 32003), (4800, 512, 1009), (2100, 1024, 16384), (300, 64, 7), (5, 128, 100), (700, 1088, 900)]


@gpu
@pytest.mark.parametrize("n,H,V", SIZES)
@pytest.mark.parametrize("weight", [1 / 1000, 1 / 1020, 1.0039 / 1024, None])
def test_weights(n, H, V, weight):
    """1 / 1020 and 1.0039 / 1024 are what bf16 scales most: by 2^-8, every gradient alike; None: weights of their own"""
    c = Call(n, H, V, seed=n, ignored=0.05)
    if weight is None:
        c.dnll = 0.5 + torch.rand(n, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    else:
        c.dnll.fill_(weight)
    c.run()
    _check(c)
    c.check()


@gpu
def test_pieces():
    c = Call(4100, 512, 131080, seed=4)
    c.dnll.fill_(1 / 1020)
    c.run()
    _check(c)


# labels in many rows: all of them, few and many of a long list, neighbours, ends
def _labels(kind, n, V):
    i = torch.arange(n)
    return {"one": 0 * i + V - 1, "two": i % 2 * (V - 1), "runs": i * 7 // n % V, "far": torch.where(i % 2049 == 0, 5, 6 + i % (V - 6)), "most": torch.where(i % 3 == 0, i % V, 4)}[kind]


@gpu
@pytest.mark.parametrize("kind", ["one", "two", "runs", "far", "most"])
@pytest.mark.parametrize("n,H,V", [(1, 64, 9), (257, 1024, 50), (4500, 192, 3000), (2049, 2112, 64), (1, 1088, 300), (600, 1088, 40), (300, 1984, 9), (300, 4160, 20), (40, 8192, 9)])
def test_rows_of_one_label(n, H, V, kind):
    c = Call(n, H, V, seed=7)
    c.labels = _labels(kind, n, V).to(DEV).int()
    c.dnll.fill_(1 / 1020)
    c.run()
    _check(c)
    c.check()
    first = c.dx.clone(), c.dw.clone()
    for t in (c.dx, c.dw):
        t.fill_(float("nan"))
    c.ws.fill_(0)
    c.bwd()
    assert torch.equal(first[0], c.dx) and torch.equal(first[1], c.dw)


@gpu
@pytest.mark.parametrize("n,H,V,tile", [(4800, 512, 1009, 64), (990, 768, 3200, 128), (2100, 1024, 16384, 256)])
def test_accumulated(n, H, V, tile):
    """the sum with what was there is rounded once: off by that and by G's roundings beside the labels"""
    c = Call(n, H, V, seed=5)
    assert ob.ob_lm_loss_plan(c.desc, n).dw_tile == tile
    c.dnll.fill_(1 / 1020)
    old = (torch.randn(c.dw.shape, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV) * 1e-3).bfloat16()
    c.fwd()
    c.dw.copy_(old)
    c.bwd(ob.OB_BWD_ACCUMULATE)
    value, err = _bounds(c, c.x.double(), c.w.double())["dw"]
    value = value + old.double()
    assert _off(c.dw, value) <= _factor(c, "dw") * float(torch.hypot(_off(_bf16(value), value, False), err)) + 3e-5 * float(value.norm())
