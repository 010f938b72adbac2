"""The operators of a hidden layer whose rows are of several kinds, as a list of measurable cases.

A layer of a typed encoder sorts its rows by kind once (``rows``), multiplies each kind by its own weights (``dense``),
normalises groups of channels with an activation (``norm``) and drops elements (``dropout``).  ``prepare`` makes what a
program holds before such a call, ``run`` is one call in the direction that the case names.  Where ``own`` is false the
same results come from elementary torch operations in 32 bits, sums over many rows and random bits in 64.

Directions
  fwd    the forward call
  bwd    the backward call, with the forward results that it takes as inputs
  both   the forward call, then the backward one on what it saved
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5


def _dense(name, direction, n, kinds, f_in, f_out, dtype, relu=True, listed_rows=True):
    return dict(name=name, op="dense", direction=direction, n=n, kinds=kinds, f_in=f_in, f_out=f_out, dtype=dtype,
                relu=relu, order=listed_rows)


def _norm(name, direction, n, width, groups, act, dtype, segments="row", count=0):
    return dict(name=name, op="norm", direction=direction, n=n, width=width, groups=groups, act=act, dtype=dtype,
                segments=segments, count=count)


def listed():
    return [
        # the rows of a mini-batch by node type, once per step: launches and latency
        dict(name="rows_batch", op="rows", n=5_000, kinds=8, loose=0.1),
        # the rows of the largest share (12.5 M nodes) by kind
        dict(name="rows_share", op="rows", n=12_500_000, kinds=64, loose=0.0),
        # a few nodes asked for at serving time, each of its own kind: bound by the weights that they touch
        _dense("dense_few_bf16", "fwd", 24, 16, 256, 256, "bf16", listed_rows=False),
        # the headline part (125,237 nodes, 128 -> 256) with five node types, rows where they are
        _dense("dense_part_f32", "fwd", 125_237, 5, 128, 256, "f32"),
        _dense("dense_part_bwd_f32", "bwd", 125_237, 5, 128, 256, "f32"),
        # hidden layers over many nodes, bf16: rows laid out by kind, and rows where they are
        _dense("dense_nodes_bf16", "fwd", 1_000_003, 16, 256, 256, "bf16", listed_rows=False),
        _dense("dense_nodes_bwd_bf16", "bwd", 604_000, 16, 256, 256, "bf16"),
        # each node's channels by themselves, hidden width 256, as an encoder uses it
        _norm("norm_nodes_bf16", "fwd", 1_000_000, 256, 32, "prelu", "bf16"),
        _norm("norm_nodes_bwd_bf16", "bwd", 604_000, 256, 32, "silu", "bf16"),
        # a batch of graphs of ragged sizes, statistics over a graph's nodes: a training pass through the layer
        _norm("norm_graphs_f32", "both", 125_237, 128, 8, "silu", "f32", segments="ragged", count=1_200),
        # a hidden layer of odd width of a mid-size part
        dict(name="dropout_part_f32", op="dropout", direction="fwd", n=120_011, width=150, dtype="f32", p=0.5, step=False),
        # the hidden rows of a large graph, the step's number on the device
        dict(name="dropout_nodes_bwd_bf16", op="dropout", direction="bwd", n=2_400_000, width=256, dtype="bf16", p=0.1, step=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    return min(hi, _log(rng, lo, hi) // rng.choice([8, 8, 4, 1]) * rng.choice([8, 8, 4, 1]) + lo)


def draw(rng):
    """One more case: one row to some million rows, 1 to 256 kinds, widths 8 to 384."""
    op = rng.choice(["rows", "dense", "dense", "dense", "norm", "norm", "norm", "dropout"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "rows":
        return dict(op=op, n=_log(rng, 1, 8_000_000), kinds=_log(rng, 1, 1_000), loose=rng.choice([0.0, 0.05, 0.5]))
    if op == "dense":
        few = rng.random() < 0.25
        n, kinds = (_log(rng, 1, 200), _log(rng, 1, 64)) if few else (_log(rng, 500, 400_000), _log(rng, 1, 256))
        f_in, f_out = _width(rng, 16, 384), _width(rng, 8, 384)
        return dict(op=op, direction=rng.choice(["fwd", "bwd"]), n=n, kinds=kinds, f_in=f_in, f_out=f_out, dtype=dtype,
                    relu=rng.random() < 0.6, order=rng.random() < 0.5)
    if op == "norm":
        groups = rng.choice([1, 2, 4, 8, 16, 32])
        width = groups * max(4, min(256 // groups, _log(rng, 4, 64)))     # (of two channels normalised alone little but rounding is left)
        segments = rng.choice(["row", "row", "run", "ragged"])
        direction = rng.choice(["fwd", "bwd", "both"])
        acts = ["none", "relu", "prelu", "silu"] if direction == "fwd" else ["none", "silu"]
        n = _log(rng, 1, 600_000)
        count = 0
        if segments == "run":
            count = _log(rng, 1, max(1, n // 2))
            n = count * max(2, n // count)
        elif segments == "ragged":
            count = _log(rng, 1, max(1, n // 3))
        return dict(op=op, direction=direction, n=n, width=width, groups=groups, act=rng.choice(acts), dtype=dtype,
                    segments=segments, count=count)
    return dict(op=op, direction=rng.choice(["fwd", "bwd"]), n=_log(rng, 1, 1_500_000), width=_width(rng, 8, 384), dtype=dtype,
                p=round(rng.uniform(0.05, 0.8), 3), step=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(g, n, width, dtype, scale=1.0, shift=0.0):
    """[n, width] normal values in rows padded to 16 bytes, as the trainers hold activations."""
    per16 = 16 // torch.empty(0, dtype=dtype).element_size()
    ld = (width + per16 - 1) // per16 * per16
    return torch.randn((n, ld), generator=g, device=DEV).mul_(scale).add_(shift).to(dtype)[:, :width]


def _kinds(g, n, kinds, loose=0.0):
    """A kind for each row: shares between a half and one and a half of the mean, one kind of four without rows where
    there are many; -1 for rows of no kind."""
    share = torch.rand(kinds, generator=g, device=DEV) + 0.5
    if kinds >= 8:
        share[torch.rand(kinds, generator=g, device=DEV) < 0.25] = 0.0
        share[kinds // 2] = 1.0
    edge = share.double().cumsum(0)
    ids = torch.searchsorted(edge, torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * edge[-1], right=True)
    ids = ids.clamp_(max=kinds - 1).int()
    if loose:
        ids[torch.rand(n, generator=g, device=DEV) < loose] = -1
    return ids


def _ragged(g, n, count):
    """Offsets of `count` segments over n rows, some of them empty or of one row."""
    cuts = torch.randint(0, n + 1, (max(count - 1, 0),), generator=g, device=DEV).sort().values
    edge = torch.tensor([0, n], device=DEV)
    return torch.cat([edge[:1], cuts, edge[1:]]).int()


def prepare(case, seed):
    g = _generator(seed)
    op, n = case["op"], case["n"]
    s = dict(case=case)
    if op == "rows":
        s["ids"] = _kinds(g, n, case["kinds"], case["loose"])
        s["offsets"] = torch.zeros(case["kinds"] + 1, dtype=torch.int32, device=DEV)
        s["order"] = torch.full((n,), -1, dtype=torch.int32, device=DEV)
        return s
    dtype = _dtype(case)
    if op == "dense":
        E, fi, fo = case["kinds"], case["f_in"], case["f_out"]
        ids = _kinds(g, n, E)
        sizes = torch.bincount(ids.long(), minlength=E)
        s["offsets"] = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)]).int()
        s["order"] = ids.long().argsort(stable=True).int() if case["order"] else None
        s["X"] = _rows(g, n, fi, dtype)
        s["W"] = torch.randn((E, fi, fo), generator=g, device=DEV) * math.sqrt(2.0 / (fi + fo))
        s["b"] = torch.randn((E, fo), generator=g, device=DEV) * 0.1
        s["act"] = 1 if case["relu"] else 0
        # the plain form's plan: the largest kind, and each listed row's place among E times that many
        s["most"] = int(sizes.max())
        kind = ids.long().sort().values
        s["place"] = kind * s["most"] + torch.arange(n, device=DEV) - s["offsets"].long()[kind]
        if case["direction"] == "bwd":
            s["dY"] = _rows(g, n, fo, dtype, scale=1.0 / n)
            s["Y"] = _rows(g, n, fo, dtype)        # what the forward call left: positive or zero
            s["Y"].clamp_(min=0)
            s["dW"], s["db"] = torch.empty_like(s["W"]), torch.empty_like(s["b"])
            s["out"] = torch.empty_like(s["X"])
        else:
            s["out"] = _rows(g, n, fo, dtype)
        return s
    width = case["width"]
    s["X"] = _rows(g, n, width, dtype, shift=0.3 if op == "norm" else 0.0)
    s["out"] = torch.empty_like(s["X"])
    if op == "dropout":
        s["seed"] = int(torch.randint(1 << 62, (1,), generator=g, device=DEV))
        s["step"] = torch.randint(1 << 20, (1,), generator=g, device=DEV) if case["step"] else None
        return s
    s["gamma"] = 1.0 + 0.3 * torch.randn(width, generator=g, device=DEV)
    s["beta"] = 0.3 * torch.randn(width, generator=g, device=DEV)
    s["slope"] = torch.full((1,), 0.25, device=DEV) if case["act"] == "prelu" else None
    if case["segments"] == "ragged":
        s["offsets"] = _ragged(g, n, case["count"])
        s["of"] = torch.repeat_interleave(torch.arange(case["count"], device=DEV), s["offsets"].long().diff())
    elif case["segments"] == "run":
        s["of"] = torch.arange(n, device=DEV) // (n // case["count"])
    if case["direction"] != "fwd":
        s["dY"] = _rows(g, n, width, dtype)
        s["dX"] = torch.empty_like(s["X"])
        if case["segments"] != "row":
            s["stats"] = _statistics(case, s)       # what the forward call left
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _plain_rows(case, s):
    ids, E = s["ids"].long(), case["kinds"]
    key = torch.where((ids >= 0) & (ids < E), ids, torch.full_like(ids, E))
    sorted_key, order = key.sort(stable=True)
    offsets = torch.searchsorted(sorted_key, torch.arange(E + 1, device=ids.device))
    return offsets.int(), torch.where(sorted_key < E, order, torch.full_like(order, -1)).int()


def _padded(case, s, rows):
    """The kinds' rows as [kinds, largest kind, width] in 32 bits, zeros behind a kind's last row."""
    rows = rows.float()
    out = rows.new_zeros((case["kinds"] * s["most"], rows.shape[1]))
    out[s["place"]] = rows if s["order"] is None else rows[s["order"].long()]
    return out.view(case["kinds"], s["most"], -1)


def _unpadded(s, padded):
    rows = padded.flatten(0, 1)[s["place"]]
    return rows if s["order"] is None else torch.empty_like(rows).index_copy_(0, s["order"].long(), rows)


def _plain_dense(case, s):
    dtype, X = _dtype(case), _padded(case, s, s["X"])
    if case["direction"] == "fwd":
        Z = torch.bmm(X, s["W"]) + s["b"][:, None, :]
        return _unpadded(s, Z.clamp_(min=0) if case["relu"] else Z).to(dtype)
    dZ = s["dY"].float()
    dZ = _padded(case, s, torch.where(s["Y"] > 0, dZ, torch.zeros_like(dZ)) if case["relu"] else dZ)
    dX = _unpadded(s, torch.bmm(dZ, s["W"].transpose(1, 2).contiguous()))
    return torch.bmm(X.transpose(1, 2).contiguous(), dZ), dZ.sum(1), dX.to(dtype)


def _segment_sums(s, per_row, count):
    """[rows, groups] -> [segments, groups], in 64 bits: segments may be long."""
    return per_row.new_zeros((count, per_row.shape[1])).index_add_(0, s["of"], per_row)


def _statistics(case, s):
    """[segments, groups, 2]: mean and 1/sqrt(variance + EPS), zeros of a segment without rows"""
    G, count, cg = case["groups"], case["count"], case["width"] // case["groups"]
    x = s["X"].double().unflatten(1, (G, cg))
    held = torch.bincount(s["of"], minlength=count)[:, None]
    rows = held.clamp(min=1) * cg
    mean = _segment_sums(s, x.sum(2), count) / rows
    var = _segment_sums(s, (x - mean[s["of"]][:, :, None]).square().sum(2), count) / rows
    return torch.stack([mean, (var + EPS).rsqrt() * (held > 0)], 2).float()


def _activation(case, s, y):
    """act(y) and its derivative"""
    if case["act"] == "silu":
        t = torch.sigmoid(y)
        return y * t, t * (1 + y * (1 - t))
    slope = {"none": 1.0, "relu": 0.0, "prelu": 0.25}[case["act"]]
    return torch.where(y > 0, y, slope * y), torch.where(y > 0, torch.ones_like(y), torch.full_like(y, slope))


def _plain_norm(case, s):
    dtype, G, cg = _dtype(case), case["groups"], case["width"] // case["groups"]
    x = s["X"].float().unflatten(1, (G, cg))
    whole = case["segments"] == "row"
    if whole:
        mean = x.mean(2, keepdim=True)
        stats = None
        rstd = ((x - mean).square().mean(2, keepdim=True) + EPS).rsqrt()
    else:
        stats = s["stats"] if case["direction"] == "bwd" else _statistics(case, s)
        mean, rstd = stats[s["of"], :, :1], stats[s["of"], :, 1:]
    xh = (x - mean) * rstd
    gamma = s["gamma"].view(G, cg)
    y = gamma * xh + s["beta"].view(G, cg)
    a, slope = _activation(case, s, y)
    out = [] if case["direction"] == "bwd" else [a.flatten(1).to(dtype)] + ([] if whole else [stats])
    if case["direction"] == "fwd":
        return out
    dy = s["dY"].float().unflatten(1, (G, cg)) * slope
    dxh = dy * gamma
    if whole:
        m1, m2 = dxh.mean(2, keepdim=True), (dxh * xh).mean(2, keepdim=True)
    else:
        rows = torch.bincount(s["of"], minlength=case["count"]).clamp(min=1)[:, None] * cg
        m1 = (_segment_sums(s, dxh.double().sum(2), case["count"]) / rows).float()[s["of"]][:, :, None]
        m2 = (_segment_sums(s, (dxh * xh).double().sum(2), case["count"]) / rows).float()[s["of"]][:, :, None]
    dx = (dxh - m1 - xh * m2) * rstd
    return out + [dx.flatten(1).to(dtype), (dy * xh).double().sum(0).flatten().float(), dy.double().sum(0).flatten().float()]


_M1, _M2, _STEP = (c - (1 << 64) for c in (0xBF58476D1CE4E5B9, 0x94D049BB133111EB, 0x9E3779B97F4A7C15))


def _split_mix(seed, unit):
    """The library's generator in wrapping 64-bit integers; `seed`: a number or a tensor."""
    shift = lambda z, k: (z >> k) & ((1 << (64 - k)) - 1)
    z = (unit + 1) * _STEP + seed
    z = (z ^ shift(z, 30)) * _M1
    z = (z ^ shift(z, 27)) * _M2
    return z ^ shift(z, 31)


def _plain_dropout(case, s):
    n, F = case["n"], case["width"]
    x = s["X"].float()
    seed = s["seed"] if s["step"] is None else _split_mix(s["seed"], s["step"])
    units = -(-F // 4)
    z = _split_mix(seed, torch.arange(n * units, device=x.device))
    field = torch.stack([(z >> (16 * k)) & 0xFFFF for k in range(4)], 1).view(n, 4 * units)[:, :F]
    limit = math.floor(case["p"] * 65536 + 0.5)
    return torch.where(field >= limit, x * (65536 / (65536 - limit)), torch.zeros_like(x)).to(_dtype(case))


# ---------------------------------------------------------------------------------------------------- a pass
def run(s):
    case = s["case"]
    if not own:
        return {"rows": _plain_rows, "dense": _plain_dense, "norm": _plain_norm, "dropout": _plain_dropout}[case["op"]](case, s)
    from paper_2305_09887_amd import binding as B
    op, direction = case["op"], case.get("direction")
    if op == "rows":
        return B.tma_group_rows(s["ids"], case["kinds"], offsets_out=s["offsets"], order_out=s["order"])
    if op == "dense":
        if direction == "fwd":
            return B.tma_grouped_dense_fwd(s["X"], s["W"], s["b"], s["offsets"], s["act"], order=s["order"], Y_out=s["out"])
        return B.tma_grouped_dense_bwd(s["X"], s["Y"], s["dY"], s["W"], s["offsets"], s["act"], order=s["order"],
                                       dW=s["dW"], dbias=s["db"], dX_out=s["out"])
    if op == "dropout":
        call = B.tma_dropout_fwd if direction == "fwd" else B.tma_dropout_bwd
        return call(s["X"], case["p"], s["seed"], step=s["step"], out=s["out"])
    act = {"none": B.TMA_ACT_NONE, "relu": B.TMA_ACT_RELU, "prelu": B.TMA_ACT_PRELU, "silu": B.TMA_ACT_SILU}[case["act"]]
    plan = dict(slope=s["slope"], eps=EPS)
    if case["segments"] == "ragged":
        plan["segments"] = s["offsets"]
    elif case["segments"] == "run":
        plan["rows_per_segment"] = case["n"] // case["count"]
    out, stats = [], s.get("stats")
    if direction != "bwd":
        Y, stats = B.tma_groupnorm_act_fwd(s["X"], case["groups"], s["gamma"], s["beta"], act, out=s["out"],
                                           need_stats=case["segments"] != "row", **plan)
        out = [Y] if stats is None else [Y, stats]
    if direction == "fwd":
        return out
    return out + list(B.tma_groupnorm_act_bwd(s["X"], s["dY"], case["groups"], s["gamma"], s["beta"], act, stats=stats,
                                              dX_out=s["dX"], **plan)[:3])


def work(case):
    n, op = case["n"], case["op"]
    if op == "rows":
        return {"bytes": 8.0 * n + 4.0 * (case["kinds"] + 1), "flops": 0.0}
    size = 2 if case["dtype"] == "bf16" else 4
    if op == "dense":
        fi, fo = case["f_in"], case["f_out"]
        touched = min(case["kinds"], n)
        weights = touched * (fi + 1.0) * fo * 4
        index = 4.0 * (case["kinds"] + 1 + (n if case["order"] else 0))
        if case["direction"] == "fwd":
            return {"bytes": size * n * float(fi + fo) + weights + index, "flops": 2.0 * n * fi * fo}
        grads = case["kinds"] * (fi + 1.0) * fo * 4
        return {"bytes": size * n * float(2 * fi + fo * (2 if case["relu"] else 1)) + weights + grads + index,
                "flops": 4.0 * n * fi * fo}
    cells = float(n) * case["width"]
    if op == "dropout":
        return {"bytes": 2 * size * cells, "flops": 0.0}
    tensors = {"fwd": 2, "bwd": 3, "both": 4}[case["direction"]]
    return {"bytes": tensors * size * cells + 8.0 * case["width"], "flops": 10.0 * cells}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_dense(case, s):
    """Kind by kind, in the order of the list."""
    E, fi, fo, n = case["kinds"], case["f_in"], case["f_out"], case["n"]
    edge = s["offsets"].tolist()
    rows = torch.arange(n, device=DEV) if s["order"] is None else s["order"].long()
    X, W = s["X"], s["W"]
    if case["direction"] == "fwd":
        Y = torch.zeros((n, fo), dtype=torch.float64, device=DEV)
        for e in range(E):
            r = rows[edge[e]:edge[e + 1]]
            z = X[r].double().mm(W[e].double()) + s["b"][e].double()
            Y[r] = z * (z > 0) if case["relu"] else z
        return Y
    dW, db = torch.zeros((E, fi, fo), dtype=torch.float64, device=DEV), torch.zeros((E, fo), dtype=torch.float64, device=DEV)
    dX = torch.zeros((n, fi), dtype=torch.float64, device=DEV)
    for e in range(E):
        r = rows[edge[e]:edge[e + 1]]
        dz = s["dY"][r].double()
        if case["relu"]:
            dz = dz * (s["Y"][r] > 0)
        dW[e], db[e], dX[r] = X[r].double().t().mm(dz), dz.sum(0), dz.mm(W[e].double().t())
    return dW, db, dX


def _exact_norm(case, s):
    """Moments from running sums over the rows, the gradients by differentiating the forward form."""
    n, F, G = case["n"], case["width"], case["groups"]
    cg, back = F // G, case["direction"] != "fwd"
    x = s["X"].double().clone().requires_grad_(back)
    gamma, beta = (s[k].double().clone().requires_grad_(back) for k in ("gamma", "beta"))
    if case["segments"] == "row":
        v = x.view(n, G, cg)
        mean, var = v.mean(2), v.var(2, unbiased=False)
        stats = None
    else:
        if case["segments"] == "ragged":
            edge = s["offsets"].long()
        else:
            edge = torch.arange(case["count"] + 1, device=DEV) * (n // case["count"])
        size = (edge[1:] - edge[:-1]).double()[:, None] * cg
        row = torch.searchsorted(edge, torch.arange(n, device=DEV), right=True) - 1

        def per_segment(t):
            run = torch.cat([t.new_zeros((1, G)), t.view(n, G, cg).sum(2).cumsum(0)])
            return (run[edge[1:]] - run[edge[:-1]]) / size.clamp(min=1)

        mean_s = per_segment(x)
        mean = mean_s[row]
        var_s = per_segment((x - mean.repeat_interleave(cg, 1)).square())
        var = var_s[row]
        stats = torch.stack([mean_s, 1 / (var_s + EPS).sqrt()], 2).detach() * (size > 0)[:, :, None]
    y = (x - mean.repeat_interleave(cg, 1)) / (var.repeat_interleave(cg, 1) + EPS).sqrt() * gamma + beta
    a = y / (1 + torch.exp(-y)) if case["act"] == "silu" else y.clamp(min=0) + {"none": 1.0, "relu": 0.0, "prelu": 0.25}[case["act"]] * y.clamp(max=0)
    out = [] if case["direction"] == "bwd" else [a.detach()] + ([] if stats is None else [stats])
    if not back:
        return out
    return out + list(torch.autograd.grad(a, (x, gamma, beta), s["dY"].double()))


def _exact_dropout(case, s):
    """The generator in unsigned host integers, the rows in blocks."""
    n, F = case["n"], case["width"]
    units = (F + 3) // 4

    def mix(seed, unit):
        with np.errstate(over="ignore"):
            z = np.uint64(seed) + (unit + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            return z ^ (z >> np.uint64(31))

    seed = s["seed"]
    if s["step"] is not None:
        seed = int(mix(seed, np.array([int(s["step"])], dtype=np.uint64))[0])
    limit = int(round(case["p"] * 65536))
    keep = torch.empty((n, F), dtype=torch.bool, device=DEV)
    per = max(1, (1 << 23) // units)
    for a in range(0, n, per):
        b = min(n, a + per)
        z = mix(seed, np.arange(a * units, b * units, dtype=np.uint64))
        fields = z.view(np.uint16).reshape(b - a, 4 * units)[:, :F]      # little-endian: the low field first
        keep[a:b] = torch.from_numpy(fields >= limit).to(DEV)
    return s["X"].double() / (1 - limit / 65536) * keep


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rows":
        return None
    return {"dense": _exact_dense, "norm": _exact_norm, "dropout": _exact_dropout}[case["op"]](case, s)
