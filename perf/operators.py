"""The operators of the language-model side of a training step: what is timed of them, and their plain forms.

A case is a dict of plain values.  Three kinds:

  rotary   rotary positions with several axes over the query and key heads of a packed batch's [T, (nq + 2 nkv) d] rows.
           op "fwd" rotates, "bwd" rotates a gradient back.
  window   varlen attention with a sliding window and sinks.  op "fwd", or "step": forward, then backward.
  loss     cross entropy over a vocabulary, from the hidden rows of the supervised tokens.  op "fwd", or "step":
           forward, then the gradients of the hidden rows and of the output weights.

Segment layouts: "samples" = 256 visual tokens per image tile plus log-normal text (median 300); "text" = text-only
samples; "one" = a single segment.

With `own` false, run() computes the operators in their plain form, elementary operations in 32 bits; with `own` true it
calls the library.  exact() is the definition in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
PER_TILE = 256       # visual tokens of a tile on the LLM side, 16 x 16
TILE_PMF = (0.22, 0.20, 0.16, 0.14, 0.07, 0.06, 0.04, 0.03, 0.03, 0.02, 0.015, 0.015)
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _rotary(name, op, dtype, layout, tokens, nq, nkv, d, pairs, order, base, start=0, seed=0):
    """pairs: pairs per axis, as a text; order: "runs" or "turns" (the axes take turns), "apart": runs, each axis with a
    spectrum of its own; start: the first position of every sample"""
    return {"name": name, "kind": "rotary", "op": op, "dtype": dtype, "layout": layout, "tokens": tokens, "nq": nq, "nkv": nkv, "d": d,
            "pairs": pairs, "order": order, "base": base, "start": start, "lens_seed": seed}


def _window(name, op, dtype, layout, tokens, nq, nkv, d, window, sinks, seed=0):
    return {"name": name, "kind": "window", "op": op, "dtype": dtype, "layout": layout, "tokens": tokens, "nq": nq, "nkv": nkv, "d": d,
            "window": window, "sinks": sinks, "lens_seed": seed}


def _loss(name, op, dtype, layout, tokens, share, hidden, vocab, seed=0):
    """share: of the tokens, in percent, that are supervised"""
    return {"name": name, "kind": "loss", "op": op, "dtype": dtype, "layout": layout, "tokens": tokens, "share": share, "hidden": hidden,
            "vocab": vocab, "lens_seed": seed}


def listed():
    return [
        # one image tile's patches through a small vision tower: two axes, half of the pairs each; bound by the launch
        _rotary("rotary-tile-fwd", "fwd", "bf16", "one", 256, 10, 10, 64, "16,16", "apart", 10000.0),
        # the balanced mini-batch of the 7B language model: time, height and width
        _rotary("rotary-16k-fwd", "fwd", "bf16", "samples", 16327, 32, 8, 128, "16,24,24", "runs", 1000000.0, 0, 2),
        # gradients of a long stream's frames in fp32, far from the start, a quarter of the pairs without positions
        _rotary("rotary-far-bwd-fp32", "bwd", "fp32", "samples", 8191, 12, 4, 64, "8,8,8", "turns", 500000.0, 1 << 20, 3),
        # one short sample (a tile and a question), evaluated: bound by latency
        _window("window-short-fwd", "fwd", "bf16", "one", 557, 32, 8, 128, 256, 4),
        # the balanced mini-batch of the 7B language model in training
        _window("window-16k-step", "step", "bf16", "samples", 16327, 32, 8, 128, 1024, 4, 2),
        # one long document in training, small heads, a wide window
        _window("window-long-step", "step", "bf16", "one", 65521, 16, 4, 64, 4096, 64),
        # a long evaluation with the heads of the 20B model
        _window("window-long-fwd", "fwd", "bf16", "samples", 32741, 48, 8, 128, 2048, 16, 4),
        # checking a model in fp32: short texts, an odd window
        _window("window-texts-step-fp32", "step", "fp32", "text", 411, 4, 2, 64, 33, 1, 5),
        # one short sample of a small language model, evaluated: the output weights pass once
        _loss("loss-short-fwd", "fwd", "bf16", "one", 301, 20, 768, 32003),
        # the balanced mini-batch of the 7B language model in training, the supervised third of it
        _loss("loss-16k-step", "step", "bf16", "samples", 16327, 33, 4096, 65536, 2),
        # the balanced mini-batch of the 20B language model: the largest call
        _loss("loss-32k-step", "step", "bf16", "samples", 32741, 25, 6144, 131072, 4),
        # checking a model in fp32
        _loss("loss-texts-step-fp32", "step", "fp32", "text", 200, 60, 256, 1009, 5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    seed = rng.randrange(1 << 20)
    kind = rng.choice(("rotary", "window", "window", "loss"))
    dtype = "fp32" if rng.random() < (0.3 if kind == "rotary" else 0.12) else "bf16"
    layout = rng.choice(("samples", "samples", "text", "one"))
    if kind == "rotary":
        d = rng.choice((64, 128))
        nkv = rng.choice((1, 2, 3, 4, 8, 10))
        nq = nkv * rng.choice((1, 2, 4, 6) if nkv <= 8 else (1, 2))
        axes, left = rng.randint(1, 4), d // 2
        pairs = [left // axes] * axes
        if rng.random() < 0.5:        # some pairs without positions, or uneven shares
            pairs = [max(1, p - rng.randint(0, p - 1)) for p in pairs]
        c = _rotary("", rng.choice(("fwd", "bwd")), dtype, layout, _log_int(rng, 1, 16384), nq, nkv, d, ",".join(map(str, pairs)),
                    rng.choice(("runs", "turns", "apart")), rng.choice((10000.0, 500000.0, 1000000.0)),
                    rng.choice((0, 0, _log_int(rng, 1, 1 << 20))), seed)
    elif kind == "window":
        d = rng.choice((64, 128))
        nkv = rng.choice((1, 2, 4, 8))
        nq = nkv * rng.choice((1, 2, 4, 6))
        if dtype == "fp32":
            nkv = rng.choice((1, 2))
            c = _window("", rng.choice(("fwd", "step")), dtype, layout, _log_int(rng, 1, 600), nkv * rng.choice((1, 2, 4)), nkv, d,
                        _log_int(rng, 1, 600), rng.choice((0, 1, 4, 16)), seed)
        else:
            c = _window("", rng.choice(("fwd", "step", "step")), dtype, layout, _log_int(rng, 1, 32768), nq, nkv, d,
                        _log_int(rng, 16, 4096), rng.choice((0, 1, 4, 16, 64)), seed)
    elif dtype == "fp32":
        c = _loss("", rng.choice(("fwd", "step")), dtype, layout, _log_int(rng, 1, 600), rng.choice((20, 33, 60, 100)), 64 * _log_int(rng, 1, 8),
                  _log_int(rng, 17, 4096), seed)
    else:
        c = _loss("", rng.choice(("fwd", "step", "step")), dtype, layout, _log_int(rng, 1, 16384), rng.choice((20, 33, 60, 100)),
                  64 * _log_int(rng, 4, 64), _log_int(rng, 257, 131072), seed)
        if c["tokens"] * c["share"] > 819200:
            c["share"] = 33
    del c["name"]
    return c


# ---- layouts and positions -------------------------------------------------------------------------

def _text(rng):
    return max(1, min(4096, int(round(math.exp(math.log(300.0) + rng.gauss(0.0, 1.0))))))


def _samples(case):
    """(visual tokens, all tokens) of every sample"""
    T = case["tokens"]
    if case["layout"] == "one":
        return [(T // PER_TILE * PER_TILE, T)] if case["kind"] == "rotary" else [(0, T)]
    rng = random.Random(case["lens_seed"])
    out, total = [], 0
    while total < T:
        seen = PER_TILE * rng.choices(range(1, 13), TILE_PMF)[0] if case["layout"] == "samples" else 0
        n = min(seen + _text(rng), T - total)
        out.append((min(seen, n), n))
        total += n
    return out


def _cu(case):
    return np.concatenate([[0], np.cumsum([n for _, n in _samples(case)])]).astype(np.int32)


def _positions(case, axes):
    """[axes, T] int32: visual tokens of tile k at (k, row, column, 0), text behind them counts all axes up; two axes are row and column"""
    parts = []
    for seen, n in _samples(case):
        j = np.arange(seen)
        p = np.stack([j // PER_TILE, j % PER_TILE // 16, j % 16, 0 * j])
        first = max(seen // PER_TILE, 16) if seen else 0
        text = np.broadcast_to(first + np.arange(n - seen), (4, n - seen))
        parts.append(np.concatenate([p, text], 1))
    p = np.concatenate(parts, 1) + case["start"]
    return np.ascontiguousarray(p[1:3] if axes == 2 else p[:axes], dtype=np.int32)


def _pair_axes(case):
    """the axis of every pair (-1: none)"""
    pairs, half = [int(p) for p in case["pairs"].split(",")], case["d"] // 2
    if case["order"] != "turns":
        out = [a for a, n in enumerate(pairs) for _ in range(n)]
    else:
        out, left = [], list(pairs)
        while any(left):
            for a in range(len(left)):
                if left[a]:
                    out.append(a)
                    left[a] -= 1
    return out + [-1] * (half - len(out))


def _supervised(case):
    """the rows that have a label, ascending: text, never a visual token"""
    rng = np.random.default_rng(case["lens_seed"])
    at, rows = 0, []
    for seen, n in _samples(case):
        rows.append(at + np.arange(seen, n))
        at += n
    text = np.concatenate(rows)
    if len(text) == 0:
        text = np.arange(case["tokens"])
    n = max(1, min(len(text), case["tokens"] * case["share"] // 100))
    return np.sort(rng.permutation(text)[:n]).astype(np.int32)


# ---- inputs ----------------------------------------------------------------------------------------

def _randn(gen, shape, dtype, std=1.0):
    t = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)
    return (t * std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "rotary":
        axes = len(case["pairs"].split(","))
        s["x"] = _randn(gen, (case["tokens"], (case["nq"] + 2 * case["nkv"]) * case["d"]), dtype)
        s["pos"] = torch.from_numpy(_positions(case, axes)).to(DEV)
        s["pair_axes"] = _pair_axes(case)
    elif case["kind"] == "window":
        T, nq, nkv, d = case["tokens"], case["nq"], case["nkv"], case["d"]
        s["qkv"] = _randn(gen, (T, (nq + 2 * nkv) * d), dtype)
        if case["op"] == "step":
            s["d_o"] = _randn(gen, (T, nq * d), dtype)
        s["cu"] = _cu(case)
    else:
        rows = _supervised(case)
        n = len(rows)
        s["x"] = _randn(gen, (case["tokens"], case["hidden"]), dtype)
        s["w"] = _randn(gen, (case["vocab"], case["hidden"]), dtype, 0.02)
        # a few rows of a batch are cut off by the sample's length limit: no label
        labels = torch.randint(0, case["vocab"], (n,), generator=gen, device=DEV, dtype=torch.int32)
        drop = torch.rand(n, generator=gen, device=DEV) < 0.03
        s["labels"] = torch.where(drop, -100, labels).to(torch.int32)
        s["dnll"] = (0.5 + torch.rand(n, generator=gen, device=DEV)) / n         # per-sample weights of a mean
        s["rows_host"] = rows
        s["rows"] = torch.from_numpy(rows).to(DEV)
    if own:
        _prepare_own(case, s, dtype)
    return s


def _prepare_own(case, s, dtype):
    import paper_2407_20761_amd as ob
    code = ob.OB_BF16 if dtype == torch.bfloat16 else ob.OB_FP32
    s["ob"], s["dtype"] = ob, code
    buffer = lambda n: torch.empty(max(int(n), 256), dtype=torch.uint8, device=DEV)
    if case["kind"] == "rotary":
        s["desc"] = ob.make_rotary_axes_desc(s["pair_axes"], case["d"], case["base"], per_axis=case["order"] == "apart")
        s["y"] = torch.empty((case["tokens"], (case["nq"] + case["nkv"]) * case["d"]), dtype=dtype, device=DEV)
    elif case["kind"] == "window":
        T, nq, nkv, d = case["tokens"], case["nq"], case["nkv"], case["d"]
        s["seg"] = ob.Segments(s["cu"], device=DEV)
        s["o"] = torch.empty((T, nq * d), dtype=dtype, device=DEV)
        s["lse"] = torch.empty((nq, T), dtype=torch.float32, device=DEV)
        if case["op"] == "step":
            s["dqkv"] = torch.empty_like(s["qkv"])
            s["ws"] = buffer(ob.ob_varlen_attn_window_bwd_workspace_bytes(s["seg"], nq, nkv, d, case["window"], case["sinks"], code))
    else:
        n = len(s["rows_host"])
        s["desc"] = ob.make_lm_loss_desc(case["hidden"], case["vocab"], code)
        s["index"] = ob.RowIndex(s["rows_host"], device=DEV)
        s["ws"] = buffer(ob.ob_lm_loss_workspace_bytes(s["desc"], n))
        s["nll"], s["lse"] = (torch.empty(n, dtype=torch.float32, device=DEV) for _ in range(2))
        if case["op"] == "step":
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else {"rotary": _plain_rotary, "window": _plain_window, "loss": _plain_loss}[s["case"]["kind"]](s)


def _run_own(s):
    case, ob = s["case"], s["ob"]
    if case["kind"] == "rotary":
        heads = case["nq"] + case["nkv"]
        ob.ob_rotary_axes(s["desc"], s["x"], s["x"].shape[1], s["y"], s["y"].shape[1], case["tokens"], heads, s["pos"],
                          case["op"] == "bwd", s["dtype"])
        return {"y": s["y"]}
    if case["kind"] == "window":
        nq, nkv, d = case["nq"], case["nkv"], case["d"]
        qkv, ld = s["qkv"], s["qkv"].shape[1]
        q, k, v = qkv[:, :nq * d], qkv[:, nq * d:(nq + nkv) * d], qkv[:, (nq + nkv) * d:]
        ob.ob_varlen_attn_window_fwd(q, k, v, s["o"], s["lse"], ld, ld, nq * d, s["seg"], nq, nkv, d, d ** -0.5, case["window"],
                                     case["sinks"], s["dtype"])
        if case["op"] == "fwd":
            return {"o": s["o"], "lse": s["lse"]}
        dqkv = s["dqkv"]
        dq, dk, dv = dqkv[:, :nq * d], dqkv[:, nq * d:(nq + nkv) * d], dqkv[:, (nq + nkv) * d:]
        ob.ob_varlen_attn_window_bwd(s["d_o"], q, k, v, s["o"], s["lse"], dq, dk, dv, ld, ld, nq * d, s["seg"], nq, nkv, d, d ** -0.5,
                                     case["window"], case["sinks"], s["ws"], s["dtype"])
        return {"o": s["o"], "lse": s["lse"], "dqkv": dqkv}
    ob.ob_lm_loss_fwd(s["desc"], s["w"], s["x"], case["tokens"], s["index"], s["labels"], s["nll"], s["lse"], s["ws"])
    if case["op"] == "fwd":
        return {"nll": s["nll"], "lse": s["lse"]}
    ob.ob_lm_loss_bwd(s["desc"], 0, s["w"], s["x"], case["tokens"], s["index"], s["labels"], s["lse"], s["dnll"], s["dx"], s["dw"], s["ws"])
    return {"nll": s["nll"], "lse": s["lse"], "dx": s["dx"], "dw": s["dw"]}


def _plain_rotary(s):
    case, x, pos = s["case"], s["x"], s["pos"]
    d, heads = case["d"], case["nq"] + case["nkv"]
    axes = torch.tensor(s["pair_axes"], device=DEV)
    i = torch.arange(d // 2, device=DEV, dtype=torch.float64)
    if case["order"] == "apart":      # the pair's place among those of its axis, and how many there are
        same = (axes[:, None] == axes[None, :]).double()
        theta = case["base"] ** (-torch.tril(same, -1).sum(1) / same.sum(1))
    else:
        theta = case["base"] ** (-2 * i / d)
    # (angles in 64 bits: a million radians have no fraction left in 32)
    angle = pos.double()[axes.clamp(min=0)].t() * torch.where(axes < 0, 0.0, theta)
    if case["op"] == "bwd":
        angle = -angle
    c, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    h = x[:, :heads * d].float().view(-1, heads, d)
    a, b = h[..., :d // 2], h[..., d // 2:]
    return {"y": torch.cat([a * c - b * sn, b * c + a * sn], -1).reshape(-1, heads * d).to(x.dtype)}


def _bands(cu, window, sinks, rows=512):
    """(query rows, key rows of the sinks in front, key rows of the band) of every block of queries, as ranges"""
    for a, b in zip(cu[:-1].tolist(), cu[1:].tolist()):
        for q0 in range(a, b, rows):
            q1 = min(b, q0 + rows)
            k0 = max(a, q0 - window + 1)
            if k0 <= a + sinks:
                k0 = a
            yield a, q0, q1, min(a + sinks, k0), k0


def _plain_window(s):
    case, qkv, cu = s["case"], s["qkv"], s["cu"]
    T, nq, nkv, d, g = case["tokens"], case["nq"], case["nkv"], case["d"], case["nq"] // case["nkv"]
    window, sinks, scale = case["window"], case["sinks"], d ** -0.5
    f = qkv.float().view(T, nq + 2 * nkv, d).transpose(0, 1)      # [heads, T, d]
    q, k, v = f[:nq].reshape(nkv, g, T, d), f[nq:nq + nkv], f[nq + nkv:]
    o, lse = torch.empty((nkv, g, T, d), device=DEV), torch.empty((nkv, g, T), device=DEV)
    step = case["op"] == "step"
    if step:
        d_o = s["d_o"].float().view(T, nkv, g, d).permute(1, 2, 0, 3)
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a, q0, q1, s1, k0 in _bands(cu, window, sinks):
        j = torch.cat([torch.arange(a, s1, device=DEV), torch.arange(k0, q1, device=DEV)])
        i = torch.arange(q0, q1, device=DEV)[:, None]
        seen = (j <= i) & ((i - j < window) | (j - a < sinks))
        n, m = q1 - q0, len(j)
        kj, vj, qi = k[:, j], v[:, j], q[:, :, q0:q1].reshape(nkv, g * n, d)
        z = (qi @ kj.transpose(1, 2)).view(nkv, g, n, m) * scale
        z = z.masked_fill(~seen, -math.inf)
        top = z.max(-1, keepdim=True).values
        e = torch.exp(z - top)
        total = e.sum(-1, keepdim=True)
        p = e / total
        out = (p.view(nkv, g * n, m) @ vj).view(nkv, g, n, d)
        o[:, :, q0:q1] = out
        lse[:, :, q0:q1] = (top + torch.log(total))[..., 0]
        if step:
            go = d_o[:, :, q0:q1]
            dp = (go.reshape(nkv, g * n, d) @ vj.transpose(1, 2)).view(nkv, g, n, m)
            ds = (p * (dp - (go * out).sum(-1, keepdim=True))).view(nkv, g * n, m)
            dq[:, :, q0:q1] = (ds @ kj).view(nkv, g, n, d) * scale
            dk.index_add_(1, j, ds.transpose(1, 2) @ qi * scale)
            dv.index_add_(1, j, p.view(nkv, g * n, m).transpose(1, 2) @ go.reshape(nkv, g * n, d))
    back = lambda t: t.reshape(-1, T, d).transpose(0, 1).reshape(T, -1).to(qkv.dtype)
    res = {"o": back(o), "lse": lse.view(nq, T)}
    if step:
        res["dqkv"] = torch.cat([back(dq), back(dk), back(dv)], 1)
    return res


def _plain_loss(s):
    case, x, w, labels = s["case"], s["x"], s["w"], s["labels"].long()
    rows = s["rows"].long()
    xs, wf = x[rows].float(), w.float()
    z = xs @ wf.t()
    top = z.max(1, keepdim=True).values
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    has = (labels >= 0) & (labels < case["vocab"])
    safe = torch.where(has, labels, 0)[:, None]
    nll = torch.where(has, lse - z.gather(1, safe)[:, 0], 0.0)
    if case["op"] == "fwd":
        return {"nll": nll, "lse": lse}
    weight = torch.where(has, s["dnll"], 0.0)[:, None]
    g = torch.exp(z.sub_(lse[:, None])).mul_(weight)
    g.scatter_add_(1, safe, -weight)
    dx = torch.zeros_like(x)
    dx[rows] = (g @ wf).to(x.dtype)
    return {"nll": nll, "lse": lse, "dx": dx, "dw": (g.t() @ xs).to(w.dtype)}


# ---- work ------------------------------------------------------------------------------------------

def _area(case):
    """(query, key) pairs that see each other"""
    total, w, s = 0, case["window"], case["sinks"]
    for _, n in _samples(case):
        i = np.arange(n, dtype=np.int64)
        total += int(np.minimum(i + 1, np.minimum(i + 1, w) + np.minimum(np.maximum(i + 1 - w, 0), s)).sum())
    return float(total)


def work(case):
    size = 2.0 if case["dtype"] == "bf16" else 4.0
    T = case["tokens"]
    if case["kind"] == "rotary":
        values = float(T) * (case["nq"] + case["nkv"]) * case["d"]
        return {"bytes": 2 * size * values + 4.0 * T * len(case["pairs"].split(",")), "flops": 3 * values}
    if case["kind"] == "window":
        nq, nkv, d = case["nq"], case["nkv"], case["d"]
        pair = 4.0 * nq * d * _area(case)
        if case["op"] == "fwd":       # q, k, v in; o and the log-sum-exp out
            return {"bytes": size * T * d * 2 * (nq + nkv) + 4.0 * nq * T, "flops": pair}
        # and d_o in; dq, dk, dv out
        return {"bytes": size * T * d * 4 * (nq + nkv) + 4.0 * nq * T, "flops": 3 * pair}
    n, H, V = len(_supervised(case)), case["hidden"], case["vocab"]
    if case["op"] == "fwd":           # the supervised rows, the weights, labels; the losses and log-sum-exps
        return {"bytes": size * H * (n + V) + 16.0 * n, "flops": 2.0 * n * H * V}
    return {"bytes": size * H * (n + T + 2 * V) + 20.0 * n, "flops": 6.0 * n * H * V}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"rotary": _exact_rotary, "window": _exact_window, "loss": _exact_loss}[case["kind"]](case, s)


def _exact_rotary(case, s):
    """every pair as a complex number, turned by exp(i pos theta)"""
    d, heads, T = case["d"], case["nq"] + case["nkv"], case["tokens"]
    x = s["x"][:, :heads * d].double().view(T, heads, d)
    z = torch.complex(x[..., :d // 2], x[..., d // 2:])
    axes, place, turn = s["pair_axes"], {}, []
    for i, a in enumerate(axes):
        if a < 0:
            turn.append(torch.ones(T, dtype=torch.complex128, device=DEV))
            continue
        j = place.get(a, 0)
        place[a] = j + 1
        power = j / axes.count(a) if case["order"] == "apart" else 2 * i / d
        phi = s["pos"][a].double() / math.pow(case["base"], power)
        turn.append(torch.polar(torch.ones_like(phi), phi if case["op"] == "fwd" else -phi))
    z = z * torch.stack(turn, 1)[:, None]
    return {"y": torch.cat([z.real, z.imag], -1).reshape(T, heads * d)}


def _exact_window(case, s):
    """head by head and segment by segment, 2048 query rows at a time against every key in front of them"""
    T, nq, nkv, d, g = case["tokens"], case["nq"], case["nkv"], case["d"], case["nq"] // case["nkv"]
    if 10.0 * nq * d * sum(float(n) * n for _, n in _samples(case)) > 3e14:
        return None
    x = s["qkv"].double()
    o, lse = torch.zeros((T, nq * d), dtype=torch.float64, device=DEV), torch.zeros((nq, T), dtype=torch.float64, device=DEV)
    grad = torch.zeros_like(x)
    step = case["op"] == "step"
    for h in range(nq):
        cq, ck, cv = (slice(c * d, (c + 1) * d) for c in (h, nq + h // g, nq + nkv + h // g))
        for a, b in zip(s["cu"][:-1].tolist(), s["cu"][1:].tolist()):
            for q0 in range(a, b, 2048):
                q1 = min(b, q0 + 2048)
                dist = torch.arange(q0, q1, device=DEV)[:, None] - torch.arange(a, q1, device=DEV)
                hide = (dist < 0) | (dist >= case["window"])
                hide[:, :case["sinks"]] &= dist[:, :case["sinks"]] < 0
                z = (x[q0:q1, cq] @ x[a:q1, ck].t()) / math.sqrt(d)
                z[hide] = -math.inf
                ls = torch.logsumexp(z, 1)
                p = torch.exp(z - ls[:, None])
                o[q0:q1, h * d:(h + 1) * d] = p @ x[a:q1, cv]
                lse[h, q0:q1] = ls
                if step:
                    go = s["d_o"][q0:q1, h * d:(h + 1) * d].double()
                    dp = go @ x[a:q1, cv].t()
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                    grad[q0:q1, cq] += ds @ x[a:q1, ck]
                    grad[a:q1, ck] += ds.t() @ x[q0:q1, cq]
                    grad[a:q1, cv] += p.t() @ go
    res = {"o": o, "lse": lse}
    if step:
        res["dqkv"] = grad
    return res


def _exact_loss(case, s):
    """a few hundred rows of the batch at a time, the whole vocabulary"""
    rows, labels, V = s["rows"].long(), s["labels"].tolist(), case["vocab"]
    w, n = s["w"].double(), len(labels)
    if 6.0 * n * V * case["hidden"] > 2.5e14:
        return None
    nll, lse = (torch.zeros(n, dtype=torch.float64, device=DEV) for _ in range(2))
    step = case["op"] == "step"
    dx = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEV) if step else None
    dw = torch.zeros_like(w) if step else None
    for i0 in range(0, n, 512):
        i1 = min(n, i0 + 512)
        xs = s["x"][rows[i0:i1]].double()
        logp = torch.log_softmax(xs @ w.t(), 1)
        kept = [i for i in range(i0, i1) if 0 <= labels[i] < V]
        at = torch.tensor([i - i0 for i in kept], device=DEV, dtype=torch.long)
        to = torch.tensor([labels[i] for i in kept], device=DEV, dtype=torch.long)
        nll[i0 + at] = -logp[at, to]
        lse[i0:i1] = (xs * w[0]).sum(1) - logp[:, 0]
        if step:
            g = torch.zeros_like(logp)
            g[at] = torch.exp(logp[at])
            g[at, to] -= 1
            g *= s["dnll"][i0:i1].double()[:, None]
            dx[rows[i0:i1]] = g @ w
            dw += g.t() @ xs
    res = {"nll": nll, "lse": lse}
    if step:
        res["dx"], res["dw"] = dx, dw
    return res
