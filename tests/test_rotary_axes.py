"""Rotary positions with several axes: against the definition in 80 bits, and what is refused."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2407_20761_amd as ob

gpu = pytest.mark.gpu
DEV = "cuda"


def _axes(d, kind):
    half = d // 2
    if kind == "one":
        return [0] * half
    if kind == "runs":
        return [0] * (half // 4) + [1] * (3 * half // 8) + [2] * (half - half // 4 - 3 * half // 8)
    if kind == "turns":
        return [i % 3 for i in range(half)]
    if kind == "part":                      # half of the head passes, and one axis has no pair
        return [0] * (half // 2 - 1) + [2] + [-1] * (half // 2)
    return [-1] * half


def _expected(x, pos, axes, base, per_axis, inverse):
    """x [T, heads, d] in 64 bits -> (y, |a| + |b| of every element's pair); angles in 80 bits (positions of 2^31 have no digits to
    spare in 64)"""
    d, base = x.shape[2], np.float32(base)          # (a float of the description)
    y, size = x.copy(), np.zeros_like(x)
    for i, a in enumerate(axes):
        if a < 0:
            continue
        power = np.longdouble(axes[:i].count(a)) / axes.count(a) if per_axis else np.longdouble(2 * i) / d
        ang = pos[a].astype(np.longdouble) * np.longdouble(base) ** -power * (-1 if inverse else 1)
        c, s = np.cos(ang).astype(np.float64)[:, None], np.sin(ang).astype(np.float64)[:, None]
        p, q = x[:, :, i], x[:, :, i + d // 2]
        y[:, :, i], y[:, :, i + d // 2] = p * c - q * s, q * c + p * s
        size[:, :, i] = size[:, :, i + d // 2] = np.abs(p) + np.abs(q)
    return y, size


def _run(T, heads, d, kind, base=10000.0, per_axis=False, inverse=False, dtype=torch.bfloat16, extra=8, in_place=False, seed=0, pos=None):
    print(f"rotary axes: T={T} heads={heads} d={d} {kind} base={base} per_axis={per_axis} inverse={inverse} {dtype}", flush=True)
    rng = np.random.default_rng(seed)
    axes = _axes(d, kind)
    x = torch.from_numpy(rng.standard_normal((T, heads * d + extra)).astype(np.float32)).to(dtype).to(DEV)
    if pos is None:
        pos = rng.integers(-50, 1 << 20, (max(axes) + 1 if max(axes) >= 0 else 1, T)).astype(np.int32)
        pos[:, 0] = 0
    y = x if in_place else torch.full((T, heads * d + 2 * extra), float("nan"), dtype=dtype, device=DEV)
    keep = x.clone()
    desc = ob.make_rotary_axes_desc(axes, d, base, per_axis)
    code = ob.OB_BF16 if dtype == torch.bfloat16 else ob.OB_FP32
    ob.ob_rotary_axes(desc, x, x.shape[1], y, y.shape[1], T, heads, torch.from_numpy(pos).to(DEV), inverse, code)
    np64 = lambda t: t.float().cpu().numpy().astype(np.float64)
    got, xin = np64(y[:, :heads * d]).reshape(T, heads, d), np64(keep[:, :heads * d]).reshape(T, heads, d)
    want, size = _expected(xin, pos, axes, base, per_axis, inverse)
    # one rounding to the type, and of the fp32 arithmetic: a sine or cosine off by 3e-7 (its argument has 24 bits of a half turn, 9.4e-8
    # rad, and it is good to 2 ulp), two products and a sum
    bound = torch.finfo(dtype).eps / 2 * np.abs(want) + 5e-7 * size
    worst = float((np.abs(got - want) / np.maximum(bound, 1e-30)).max())
    assert worst <= 1
    if in_place:
        assert torch.equal(y[:, heads * d:], keep[:, heads * d:])
    else:
        assert torch.equal(x, keep)
        assert torch.isnan(y[:, heads * d:].float()).all()
    return y


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["one", "runs", "turns", "part", "none"])
def test_axes(d, dtype, kind):
    _run(37, 5, d, kind, dtype=dtype)
    _run(5, 3, d, kind, base=1e6, per_axis=True, inverse=True, dtype=dtype, seed=1)


@gpu
@pytest.mark.parametrize("T,heads,d", [(1, 1, 64), (1, 40, 128), (2, 1, 128), (3, 20, 64), (4, 7, 64), (5, 40, 128), (301, 30, 64), (1029, 56, 128),
                                       (4, 4096, 64), (70000, 1, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sizes(T, heads, d, dtype):
    _run(T, heads, d, "runs", dtype=dtype, in_place=True)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_position(dtype):
    edge = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 2 ** 24 + 1, 1000003, -999999, 65537], dtype=np.int32)
    _run(10, 2, 128, "turns", base=1000000.0, dtype=dtype, pos=np.stack([edge, edge[::-1], np.roll(edge, 3)]))
    _run(10, 2, 64, "one", base=1.0001, dtype=dtype, pos=edge[None])


@gpu
def test_back_and_forth_in_fp32():
    """the inverse is the transpose: <R x, g> = <x, R^T g>, and R^T R x = x"""
    T, heads, d, axes = 50, 3, 64, _axes(64, "runs")
    gen = torch.Generator().manual_seed(0)
    x, g = (torch.randn((T, heads * d), generator=gen).to(DEV) for _ in range(2))
    pos = torch.randint(0, 100000, (3, T), generator=gen, dtype=torch.int32).to(DEV)
    desc = ob.make_rotary_axes_desc(axes, d, 500000.0)
    rx, rg, back = (torch.empty_like(x) for _ in range(3))
    turn = lambda a, b, inv: ob.ob_rotary_axes(desc, a, heads * d, b, heads * d, T, heads, pos, inv, ob.OB_FP32)
    turn(x, rx, False)
    turn(g, rg, True)
    turn(rx, back, True)
    # every element within 1e-6 of its pair's size, twice
    assert (back - x).abs().max() <= 2e-6 * 2 * x.abs().max()
    a, b = (rx.double() * g.double()).sum(), (x.double() * rg.double()).sum()
    assert abs(float(a - b)) <= 2e-6 * float((x.double().abs() * g.double().abs()).sum()) * 2


@gpu
def test_a_pair_without_an_axis_passes_anything():
    x = torch.full((3, 64), float("inf"), dtype=torch.bfloat16, device=DEV)
    x[:, 5] = float("nan")
    y = torch.zeros_like(x)
    pos = torch.zeros((1, 3), dtype=torch.int32, device=DEV)
    ob.ob_rotary_axes(ob.make_rotary_axes_desc([-1] * 32, 64), x, 64, y, 64, 3, 1, pos)
    assert torch.equal(y.view(torch.int16), x.view(torch.int16))


@gpu
def test_captured():
    T, heads, d = 33, 6, 128
    x = torch.randn((T, heads * d), device=DEV).bfloat16()
    pos = torch.randint(0, 1000, (3, T), dtype=torch.int32, device=DEV)
    desc, y = ob.make_rotary_axes_desc(_axes(d, "turns"), d), torch.empty_like(x)
    call = lambda: ob.ob_rotary_axes(desc, x, heads * d, y, heads * d, T, heads, pos)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        x.normal_()
        pos.add_(i)
        graph.replay()
        got = y.clone()
        call()
        assert torch.equal(got, y)


# ---- refusals: no GPU ------------------------------------------------------------------------------

@pytest.mark.parametrize("status,text,kw", [
    (3, "head_dim", {"d": 96}), (1, "n_axes", {"n_axes": 0}), (1, "n_axes", {"n_axes": 9}), (1, "base", {"base": 1.0}),
    (1, "base", {"base": float("nan")}), (1, "base", {"base": float("inf")}), (1, "pair 3 has axis 2", {"axis3": 2}), (1, "axis -2", {"axis3": -2}),
    (1, "null", {"x": None}), (1, "null", {"pos": None}), (1, "dtype", {"dtype": 5}), (1, "total_tokens", {"T": 0}),
    (1, "total_tokens", {"T": (1 << 22) + 1}), (1, "n_heads", {"heads": 0}), (1, "n_heads", {"heads": 4097}), (1, "strides", {"ldx": 120}),
    (1, "strides", {"ldy": 132}), (1, "aligned", {"y": 0x2008}), (1, "in place", {"y": 0x1000, "ldy": 136}),
])
def test_refusals(status, text, kw):
    a = dict(d=64, n_axes=2, base=10000.0, axis3=1, x=0x1000, y=0x2000, pos=0x3000, ldx=128, ldy=128, T=4, heads=2, dtype=0)
    a.update(kw)
    desc = ob.ob_rotary_axes_desc(a["d"], a["n_axes"], a["base"], 0, (C.c_int8 * 64)(*([0, 0, 0, a["axis3"]] + [0] * 60)))
    st = ob.lib.ob_rotary_axes(C.byref(desc), C.c_void_p(a["x"]), a["ldx"], C.c_void_p(a["y"]), a["ldy"], a["T"], a["heads"],
                               C.c_void_p(a["pos"]), 0, a["dtype"], None)
    assert st == status and text in ob.ob_last_error(), ob.ob_last_error()


def test_make_desc_counts_the_pairs():
    with pytest.raises(ValueError):
        ob.make_rotary_axes_desc([0] * 31, 64)
    with pytest.raises(ValueError):
        ob.make_rotary_axes_desc([0] * 100, 200)
    for axis in (-2, -257, 127, 256):      # (the description holds 8 bits of it)
        with pytest.raises(ValueError):
            ob.make_rotary_axes_desc([axis] + [0] * 31, 64)
    assert ob.make_rotary_axes_desc([-1] * 32, 64).n_axes == 1


def test_positions_of_64_bits():
    x, pos, desc = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros((1, 4), dtype=torch.int64), ob.make_rotary_axes_desc([0] * 32, 64)
    with pytest.raises(TypeError, match="int32"):
        ob.ob_rotary_axes(desc, x, 64, x, 64, 4, 1, pos)
    with pytest.raises(TypeError, match="int32"):
        ob.BlockAttn(rotary=desc, pos=pos)
