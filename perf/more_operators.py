"""The operators of wide residual layers and of the step that trains them, as a list of measurable cases.

A gated layer multiplies the rows by two weights and one result by the activation of the other (``gated``), a dense layer
adds its result to what went past it (``residual``), and before the optimizer the gradients of all tensors are held to one
norm (``clip``).  ``prepare`` makes what a program holds before such a call, ``run`` is one call in the direction that the
case names.  Where ``own`` is false the same results come from elementary torch operations in 32 bits, sums over a whole
model in 64.

Directions
  fwd    the forward call; ``save``: with what the backward call will ask for
  bwd    the backward call, with the forward results that it takes as inputs
  both   the forward call, then the backward one on what it saved
  norm   the norm alone (clip)
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"


def _layer(op, name, direction, n, f_in, f_out, dtype, act="silu", bias=True, save=True, dense=False):
    return dict(name=name, op=op, direction=direction, n=n, f_in=f_in, f_out=f_out, dtype=dtype, act=act, bias=bias, save=save,
                dense=dense)


def _clip(name, direction, tensors, total, dtype, ratio):
    return dict(name=name, op="clip", direction=direction, tensors=tensors, total=total, dtype=dtype, ratio=ratio)


def listed():
    return [
        # one token, or one node, asked for at serving time: bound by the weights
        _layer("gated", "gated_token_bf16", "fwd", 1, 1024, 4096, "bf16", bias=False, save=False),
        # a few requests served together
        _layer("gated", "gated_batch_bf16", "fwd", 24, 2048, 5632, "bf16", bias=False, save=False),
        # the rows of a training step through a wide layer, and their gradients: bound by the matrix units
        _layer("gated", "gated_rows_bf16", "fwd", 8_192, 2048, 8192, "bf16"),
        _layer("gated", "gated_rows_bwd_bf16", "bwd", 8_192, 2048, 8192, "bf16"),
        # the headline part (125,237 nodes, 128 -> 256): a training pass through the layer
        _layer("gated", "gated_part_f32", "both", 125_237, 128, 256, "f32"),
        # one row out of a wide layer
        _layer("residual", "residual_token_f32", "fwd", 1, 4096, 1024, "f32", act="none", save=False),
        # the way back from a wide layer to the rows that went past it
        _layer("residual", "residual_rows_bf16", "fwd", 8_192, 8192, 2048, "bf16", act="none", save=False),
        # hidden layers over many nodes: bound by memory
        _layer("residual", "residual_nodes_bf16", "fwd", 1_000_003, 256, 256, "bf16", act="relu"),
        # odd widths in rows that lie behind each other
        _layer("residual", "residual_odd_bwd_f32", "bwd", 30_011, 301, 777, "f32", dense=True),
        # the tensors of a small encoder: launches and latency
        _clip("clip_encoder_f32", "clip", 14, 202_031, "f32", 0.5),
        # a deep model's gradients in half the bytes
        _clip("clip_model_bf16", "clip", 290, 400_000_007, "bf16", 0.25),
        # a large model's gradients, watched only
        _clip("norm_model_f32", "norm", 120, 500_000_003, "f32", 1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    return max(lo, min(hi, _log(rng, lo, hi) // (m := rng.choice([64, 64, 8, 1])) * m))


def draw(rng):
    """One more case: one row to a quarter of a million, widths 8 to 8192; one tensor to 400, one gradient to 200 million."""
    op = rng.choice(["gated", "gated", "residual", "residual", "clip"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "clip":
        return dict(op=op, direction=rng.choice(["clip", "clip", "norm"]), tensors=_log(rng, 1, 400), total=_log(rng, 400, 200_000_000),
                    dtype=dtype, ratio=round(rng.choice([0.1, 0.7, 3.0]) * rng.uniform(0.9, 1.2), 3))
    f_in, f_out = _width(rng, 8, 4096), _width(rng, 8, 8192)
    few = rng.random() < 0.3
    most = int(2.5e11 / (f_in * f_out))
    n = _log(rng, 1, 64) if few else _log(rng, 65, max(66, min(250_000, most)))
    # (a ReLU is decided by a value's sign: where one call's rounding is the next one's decision no two forms agree)
    direction = rng.choice(["fwd", "bwd", "both"] if dtype == "f32" else ["fwd", "bwd"])
    act = rng.choice(["none", "silu", "gelu"] if direction == "both" else ["none", "relu", "silu", "gelu"])
    return dict(op=op, direction=direction, n=n, f_in=f_in, f_out=f_out, dtype=dtype, act=act, bias=rng.random() < 0.7,
                save=direction != "fwd" or rng.random() < 0.5, dense=rng.random() < 0.3)


# ---------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(g, case, n, width, scale=1.0):
    """[n, width] normal values: in rows padded to 16 bytes, as the trainers hold activations, or behind each other."""
    dtype = _dtype(case)
    per16 = 1 if case["dense"] else 16 // torch.empty(0, dtype=dtype).element_size()
    ld = (width + per16 - 1) // per16 * per16
    return torch.randn((n, ld), generator=g, device=DEV).mul_(scale).to(dtype)[:, :width]


def _prepare_clip(case, g, s):
    """The tensors one behind the other in one buffer, of sizes that differ by up to some hundred times, one of a single
    value among them."""
    count, total, dtype = case["tensors"], case["total"], _dtype(case)
    count = min(count, total)
    share = torch.rand(count, generator=g, device=DEV, dtype=torch.float64).mul_(5).exp_()
    edge = share.cumsum(0).div_(share.sum()).mul_(total - count).long().tolist()
    edge[-1] = total - count
    edge = [0] + [e + i + 1 for i, e in enumerate(edge)]
    s["flat"] = torch.empty(total, dtype=dtype, device=DEV)
    for a in range(0, total, 1 << 26):
        b = min(total, a + (1 << 26))
        s["flat"][a:b] = torch.randn(b - a, generator=g, device=DEV).mul_(1e-3)
    s["max_norm"] = case["ratio"] * 1e-3 * math.sqrt(total)
    s["out"] = torch.empty_like(s["flat"]) if case["direction"] == "clip" else None
    s["grads"] = [s["flat"][a:b] for a, b in zip(edge[:-1], edge[1:])]
    s["outs"] = [s["out"][a:b] for a, b in zip(edge[:-1], edge[1:])] if case["direction"] == "clip" else None
    return s


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case=case)
    if case["op"] == "clip":
        return _prepare_clip(case, g, s)
    n, fi, fo, gated = case["n"], case["f_in"], case["f_out"], case["op"] == "gated"
    back = case["direction"] != "fwd"
    s["X"] = _rows(g, case, n, fi)
    weight = lambda: torch.randn((fi, fo), generator=g, device=DEV) * math.sqrt(1.0 / fi)
    bias = lambda: torch.randn(fo, generator=g, device=DEV) * 0.1 if case["bias"] else None
    s["W"], s["b"] = weight(), bias()
    if gated:
        s["W_up"], s["b_up"] = weight(), bias()
    else:
        s["R"] = _rows(g, case, n, fo)             # what goes past the layer
    if back:
        s["dY"] = _rows(g, case, n, fo, scale=1.0 / n)
        s["dR"] = _rows(g, case, n, fi, scale=1.0 / n)      # the gradient that went past it
        if case["direction"] == "bwd":             # what the forward call left
            s["Z"] = _rows(g, case, n, fo)
            if gated:
                s["U"] = _rows(g, case, n, fo)
        s["dX"] = _rows(g, case, n, fi)
        s["dW"], s["db"] = torch.empty_like(s["W"]), torch.empty(fo, device=DEV) if case["bias"] else None
        if gated:
            s["dW_up"], s["db_up"] = torch.empty_like(s["W"]), torch.empty(fo, device=DEV) if case["bias"] else None
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _activation(name, z):
    """act(z) and its derivative"""
    if name == "silu":
        t = 1 / (1 + torch.exp(-z))
        return z * t, t * (1 + z * (1 - t))
    if name == "gelu":
        p = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    return z, torch.ones_like(z)


def _affine(X, W, b):
    return X.mm(W) if b is None else X.mm(W) + b


def _sums(d, wanted):
    """Sums over the rows, in 64 bits: there may be many."""
    return [d.sum(0, dtype=torch.float64).float()] if wanted else []


def _plain_gated(case, s):
    dtype, X, out = _dtype(case), s["X"].float(), []
    G, U = s.get("Z"), s.get("U")
    if case["direction"] != "bwd":
        G, U = _affine(X, s["W"], s["b"]), _affine(X, s["W_up"], s["b_up"])
        out = [(_activation(case["act"], G)[0] * U).to(dtype)] + ([G.to(dtype), U.to(dtype)] if case["save"] else [])
    if case["direction"] == "fwd":
        return out
    a, slope = _activation(case["act"], G.float())
    d = s["dY"].float()
    dG, dU = d * U.float() * slope, d * a
    dX = dG.mm(s["W"].t()) + dU.mm(s["W_up"].t()) + s["dR"].float()
    return out + [X.t().mm(dG), X.t().mm(dU)] + _sums(dG, case["bias"]) + _sums(dU, case["bias"]) + [dX.to(dtype)]


def _plain_residual(case, s):
    dtype, X, out, Z = _dtype(case), s["X"].float(), [], s.get("Z")
    if case["direction"] != "bwd":
        Z = _affine(X, s["W"], s["b"])
        out = [(_activation(case["act"], Z)[0] + s["R"].float()).to(dtype)] + ([Z.to(dtype)] if case["save"] else [])
    if case["direction"] == "fwd":
        return out
    dZ = s["dY"].float() * _activation(case["act"], Z.float())[1]
    dX = dZ.mm(s["W"].t()) + s["dR"].float()
    return out + [X.t().mm(dZ)] + _sums(dZ, case["bias"]) + [dX.to(dtype)]


def _plain_clip(case, s):
    norm = s["flat"].float().square().sum(dtype=torch.float64).sqrt()
    if case["direction"] == "norm":
        return [norm.float().view(1)]
    factor = (s["max_norm"] / norm).clamp(max=1.0).float()
    return [norm.float().view(1), (s["flat"].float() * factor).to(_dtype(case))]


# ---------------------------------------------------------------------------------------------------- a pass
def run(s):
    case = s["case"]
    if not own:
        return {"gated": _plain_gated, "residual": _plain_residual, "clip": _plain_clip}[case["op"]](case, s)
    from paper_2305_09887_amd import binding as B
    if case["op"] == "clip":
        if case["direction"] == "norm":
            return [B.tma_grad_norm(s["grads"])]
        return [B.tma_grad_clip(s["grads"], s["max_norm"], out=s["outs"]), s["out"]]
    act = {"none": B.TMA_ACT_NONE, "relu": B.TMA_ACT_RELU, "silu": B.TMA_ACT_SILU, "gelu": B.TMA_ACT_GELU}[case["act"]]
    back, out, Z, U = case["direction"] != "fwd", [], s.get("Z"), s.get("U")
    if case["op"] == "gated":
        if case["direction"] != "bwd":
            H, Z, U = B.tma_gated_dense_fwd(s["X"], s["W"], s["W_up"], s["b"], s["b_up"], act, save=case["save"])
            out = [H] + ([Z, U] if case["save"] else [])
        if not back:
            return out
        got = B.tma_gated_dense_bwd(s["X"], Z, U, s["dY"], s["W"], s["W_up"], act, R=s["dR"], dW_gate=s["dW"], dW_up=s["dW_up"],
                                    db_gate=s["db"], db_up=s["db_up"], dX_out=s["dX"], need_dbias=case["bias"])
    else:
        if case["direction"] != "bwd":
            Y, Z = B.tma_dense_residual_fwd(s["X"], s["W"], s["b"], act, R=s["R"], save=case["save"])
            out = [Y] + ([Z] if case["save"] else [])
        if not back:
            return out
        got = B.tma_dense_residual_bwd(s["X"], Z, s["dY"], s["W"], act, R=s["dR"], dW=s["dW"], dbias=s["db"], dX_out=s["dX"],
                                       need_dbias=case["bias"])
    return out + [t for t in got if t is not None]


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "clip":
        return {"bytes": size * float(case["total"]) * (2 if case["direction"] == "clip" else 1) + 4, "flops": 2.0 * case["total"]}
    n, fi, fo, gated = float(case["n"]), case["f_in"], case["f_out"], case["op"] == "gated"
    sides = 2 if gated else 1
    weights = 4.0 * sides * fo * (fi + (1 if case["bias"] else 0))
    product = 2.0 * n * fi * fo * sides
    saved = sides * fo
    bytes_, flops = 0.0, 0.0
    if case["direction"] != "bwd":
        past = 0 if gated else fo
        bytes_ += size * n * (fi + past + fo + (saved if case["save"] else 0)) + weights
        flops += product
    if case["direction"] != "fwd":
        seen = 0 if case["direction"] == "both" else saved * n * size + weights + size * n * fi     # (what a pass has seen already)
        bytes_ += seen + size * n * (fo + 2 * fi) + weights
        flops += 2 * product
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _act64(name, z):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z * (z > 0) if name == "relu" else z


def _by_blocks(rows, forms):
    """forms(a, b) of blocks of rows: lists of results to be put behind each other."""
    step = max(1, min(rows, 1 << 15))
    parts = [forms(a, min(rows, a + step)) for a in range(0, rows, step)]
    return [torch.cat(p) for p in zip(*parts)]


def exact(case, seed):
    """Forward by its formula, gradients of it by differentiation where a pass begins with it, else of the stored values."""
    s = prepare(case, seed)
    if case["op"] == "clip":
        parts = [t.double().pow(2).sum() for t in s["flat"].split(1 << 26)]
        norm = torch.stack(parts).sum().sqrt()
        if case["direction"] == "norm":
            return [norm.view(1)]
        c = min(1.0, s["max_norm"] / float(norm))
        return [norm.view(1), s["flat"].double() * c]
    n, gated, name = case["n"], case["op"] == "gated", case["act"]
    W, b = s["W"].double(), 0 if s["b"] is None else s["b"].double()
    Wu, bu = (s["W_up"].double(), 0 if s["b_up"] is None else s["b_up"].double()) if gated else (None, 0)

    def forward(lo, hi):
        x = s["X"][lo:hi].double()
        z = x @ W + b
        if not gated:
            return [_act64(name, z) + s["R"][lo:hi].double()] + ([z] if case["save"] else [])
        u = x @ Wu + bu
        return [_act64(name, z) * u] + ([z, u] if case["save"] else [])

    if case["direction"] == "fwd":
        return _by_blocks(n, forward)
    out = _by_blocks(n, forward) if case["direction"] == "both" else []
    sums = None

    def backward(lo, hi):
        nonlocal sums
        x, d = s["X"][lo:hi].double(), s["dY"][lo:hi].double()
        z = (x @ W + b if "Z" not in s else s["Z"][lo:hi].double()).requires_grad_()
        u = ((x @ Wu + bu if "U" not in s else s["U"][lo:hi].double()) if gated else torch.ones((), device=DEV).double()).requires_grad_()
        y = _act64(name, z) * u
        dz, du = torch.autograd.grad(y, (z, u), d)
        dx = dz @ W.t() + s["dR"][lo:hi].double()
        mine = [x.t() @ dz] + ([x.t() @ du] if gated else []) + ([dz.sum(0)] + ([du.sum(0)] if gated else []) if case["bias"] else [])
        sums = mine if sums is None else [p + q for p, q in zip(sums, mine)]
        return [dx + du @ Wu.t() if gated else dx]

    dX = _by_blocks(n, backward)
    return out + sums + dX
