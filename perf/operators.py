"""The products around a feed-forward block that a user of this package has it do, as cases that can be timed and compared.

Four kinds.  `linear`: one layer in the structured-only form (dense rows of the neurons that are not ablated) with bias, activation and
residual behind the product.  `linear_bwd`: its gradients, from the gradient of its result and the pre-activations that the
forward pass left.  `gated`: act(x Wg^T + bg) * (x Wu^T + bu).  `gated_bwd`: its gradients, from the gradient of its result and both
projections that the forward pass left.  Sizes are those of the package's configurations (the 768 <-> 3072 projections of a
ViT-B/16 block, the 4096 -> 16384 layer) and ragged ones between and below them.  Weights N(0, 1/d_in), activations N(0, 1).
"""
from __future__ import annotations

import math

import torch

own = False

# Multiply-adds of one projection in what draw() gives: the largest listed cases have as many.
MAX_TERMS = 2048 * 4096 * 16384


def _case(kind, d_in, d_out, batch, dtype, act, ablated=0, residual=False, bias=True, save=False, out=None):
    return {"kind": kind, "d_in": d_in, "d_out": d_out, "batch": batch, "dtype": dtype, "act": act, "ablated": ablated, "residual": residual, "bias": bias,
            "save": save, "out": out or dtype}


def listed():
    return [
        # Online inference, one sample through the up-projection of a ViT-B/16 block with its GELU: the smallest call.
        dict(_case("linear", 768, 3072, 1, "f32", "gelu"), name="linear_1_768x3072_f32"),
        # A small serving batch through the down-projection, 30 % of its neurons ablated, added to the residual stream, which is kept in fp32.
        dict(_case("linear", 3072, 768, 16, "bf16", "none", ablated=30, residual=True, out="f32"), name="linear_16_3072x768_bf16"),
        # A ragged layer and batch: nothing is a multiple of a tile, rows are not 16-byte aligned.
        dict(_case("linear", 1001, 777, 37, "bf16", "relu", ablated=10, residual=True), name="linear_37_1001x777_bf16"),
        # A training step's forward pass through the large layer with a fifth of its neurons ablated; the pre-activations are kept for the backward pass.
        dict(_case("linear", 4096, 16384, 2048, "bf16", "gelu", ablated=20, save=True), name="linear_2048_4096x16384_bf16"),
        # The weight gradient that a connectivity update of a ViT projection ranks, in fp32 as the update takes it, and the other gradients of that step.
        dict(_case("linear_bwd", 768, 3072, 512, "f32", "gelu"), name="linear_bwd_512_768x3072_f32"),
        # The large layer's backward pass.
        dict(_case("linear_bwd", 4096, 16384, 2048, "bf16", "gelu", ablated=20), name="linear_bwd_2048_4096x16384_bf16"),
        # One token through the gated projections of a large block: two weight matrices have to be streamed.
        dict(_case("gated", 4096, 16384, 1, "bf16", "silu", bias=False), name="gated_1_4096x16384_bf16"),
        # A ragged gated block in fp32, with biases.
        dict(_case("gated", 1000, 777, 100, "f32", "gelu", save=True), name="gated_100_1000x777_f32"),
        # A training step's forward pass through a large gated block, both projections kept.
        dict(_case("gated", 4096, 16384, 2048, "bf16", "silu", bias=False, save=True), name="gated_2048_4096x16384_bf16"),
        # The backward pass of a small gated block in fp32.
        dict(_case("gated_bwd", 768, 2048, 300, "f32", "silu"), name="gated_bwd_300_768x2048_f32"),
        # A ragged one in bf16: rows that begin anywhere.
        dict(_case("gated_bwd", 1001, 2731, 333, "bf16", "gelu"), name="gated_bwd_333_1001x2731_bf16"),
        # The backward pass of the large gated block.
        dict(_case("gated_bwd", 4096, 16384, 2048, "bf16", "silu", bias=False), name="gated_bwd_2048_4096x16384_bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def _width(rng, lo, hi):
    """Widths over the logarithm of the range: two of three a multiple of 64 as in trained models, the others any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 1 / 3 or n < 64 else (n + 32) // 64 * 64


def draw(rng):
    kind = rng.choice(["linear", "linear_bwd", "gated", "gated_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    c = _case(kind, _width(rng, 100, 4096), _width(rng, 100, 16384), _log_int(rng, 1, 2048), dtype, rng.choice(["relu", "gelu", "silu"]))
    if kind.startswith("linear"):
        c["act"] = rng.choice(["none", c["act"]])
        c["ablated"] = rng.choice([0, 0, rng.randint(1, 50)])
        c["residual"] = kind == "linear" and rng.random() < 0.5
        c["out"] = rng.choice([dtype, dtype, "f32"])
    c["bias"] = rng.random() < 0.7
    c["save"] = kind in ("linear", "gated") and rng.random() < 0.5
    return c


def _stored(case):
    return case["d_out"] - case["d_out"] * case["ablated"] // 100


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(shape, std, dtype=torch.float32):
        return (torch.randn(shape, device="cuda", generator=gen) * std).to(dtype)

    d, m, B, n, t, o = case["d_in"], case["d_out"], case["batch"], _stored(case), _type(case["dtype"]), _type(case["out"])
    s = {"kind": case["kind"], "d_in": d, "d_out": m, "n": n, "act": case["act"], "save": case["save"], "out": o, "x": normal((B, d), 1.0, t)}
    if case["kind"].startswith("linear"):
        s["W"] = normal((n, d), d ** -0.5, t)
        s["active"] = None if n == m else torch.randperm(m, device="cuda", generator=gen)[:n].sort().values.int()
        s["bias"] = normal((m,), 0.1) if case["bias"] else None
        if case["kind"] == "linear":
            s["residual"] = normal((B, m), 1.0, o) if case["residual"] else None
        else:
            s["dy"] = normal((B, m), 1e-2, o)
            bias = 0.0 if s["bias"] is None else s["bias"] if n == m else s["bias"][s["active"].long()]
            s["z"] = (s["x"].float() @ s["W"].float().T + bias).to(t)
    else:
        s["Wg"], s["Wu"] = normal((m, d), d ** -0.5, t), normal((m, d), d ** -0.5, t)
        s["bg"], s["bu"] = (normal((m,), 0.1), normal((m,), 0.1)) if case["bias"] else (None, None)
        if case["kind"] == "gated_bwd":
            s["dh"] = normal((B, m), 1e-2, t)
            s["g"] = (s["x"].float() @ s["Wg"].float().T + (s["bg"] if case["bias"] else 0.0)).to(t)
            s["u"] = (s["x"].float() @ s["Wu"].float().T + (s["bu"] if case["bias"] else 0.0)).to(t)
    return s


# ---- the framework's calls ----
def _own(s):
    from paper_2305_02299_amd import ACT_GELU, ACT_NONE, ACT_RELU, ACT_SILU, GatedLinear, StructuredLinear
    act = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "silu": ACT_SILU}[s["act"]]
    if s["kind"].startswith("linear"):
        layer = StructuredLinear(s["d_in"], s["d_out"], s["W"], s["active"], s["bias"])
        if s["kind"] == "linear":
            return layer.forward(s["x"], act=act, residual=s["residual"], out_dtype=s["out"], save=s["save"])
        return layer.backward(s["dy"], s["x"], s["z"], act=act)
    layer = GatedLinear(s["d_in"], s["d_out"], s["Wg"], s["Wu"], s["bg"], s["bu"], act)
    if s["kind"] == "gated":
        return layer.forward(s["x"], save=s["save"])
    return layer.backward(s["dh"], s["x"], s["g"], s["u"])


# ---- the plain form ----
def _act(v, act):
    if act == "relu":
        return torch.clamp(v, min=0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _slope(v, act):
    if act == "relu":
        return (v > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-v))
        return p * (1.0 + v * (1.0 - p))
    return torch.ones_like(v)


def _linear(s):
    bias = s["bias"] if s["bias"] is not None else torch.zeros(s["d_out"], device=s["x"].device)
    z = s["x"].float() @ s["W"].float().T
    if s["active"] is None:
        z = z + bias
        y = _act(z, s["act"])
    else:
        stored = s["active"].long()
        z = z + bias[stored]
        y = _act(bias, s["act"]).repeat(z.shape[0], 1)
        y[:, stored] = _act(z, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(s["out"])
    return (y, z.to(s["x"].dtype)) if s["save"] else y


def _linear_bwd(s):
    t = s["x"].dtype
    dy, x = s["dy"].float(), s["x"].float()
    dz = (dy if s["active"] is None else dy[:, s["active"].long()]) * _slope(s["z"].float(), s["act"])
    dx, dW = dz @ s["W"].float(), dz.T @ x
    if s["bias"] is None:
        return dx.to(t), dW.to(t), None
    db = dz.sum(0)
    if s["active"] is not None:
        every = dy.sum(0) * _slope(s["bias"], s["act"])
        every[s["active"].long()] = db
        db = every
    return dx.to(t), dW.to(t), db


def _gated(s):
    x, t = s["x"].float(), s["x"].dtype
    g, u = x @ s["Wg"].float().T, x @ s["Wu"].float().T
    if s["bg"] is not None:
        g, u = g + s["bg"], u + s["bu"]
    h = (_act(g, s["act"]) * u).to(t)
    return (h, g.to(t), u.to(t)) if s["save"] else h


def _gated_bwd(s):
    t = s["x"].dtype
    dh, x, g, u = s["dh"].float(), s["x"].float(), s["g"].float(), s["u"].float()
    dg, du = dh * u * _slope(g, s["act"]), dh * _act(g, s["act"])
    dx = dg @ s["Wg"].float() + du @ s["Wu"].float()
    db = (dg.sum(0), du.sum(0)) if s["bg"] is not None else (None, None)
    return (dx.to(t), (dg.T @ x).to(t), (du.T @ x).to(t)) + db


def run(state):
    if own:
        return _own(state)
    return {"linear": _linear, "linear_bwd": _linear_bwd, "gated": _gated, "gated_bwd": _gated_bwd}[state["kind"]](state)


def work(case):
    """Each input read once and each output written once; 2 operations per weight and batch row of a product."""
    d, m, B, n = case["d_in"], case["d_out"], case["batch"], _stored(case)
    e, o = (4 if case["dtype"] == "f32" else 2), (4 if case["out"] == "f32" else 2)
    listed_rows = 4 * n if n < m else 0
    biases = 4 * m if case["bias"] else 0
    if case["kind"] == "linear":
        moved = e * (B * d + n * d) + o * B * m * (2 if case["residual"] else 1) + (e * B * n if case["save"] else 0) + listed_rows + biases
        return {"bytes": moved, "flops": 2 * B * n * d}
    if case["kind"] == "linear_bwd":
        z = e * B * n if case["act"] != "none" else 0
        # with a bias its gradient is written, and its values are read where neurons are ablated
        return {"bytes": 2 * e * (B * d + n * d) + o * B * (m if case["bias"] else n) + z + listed_rows + biases * (2 if n < m else 1), "flops": 4 * B * n * d}
    if case["kind"] == "gated":
        return {"bytes": e * (B * d + 2 * m * d) + e * B * m * (3 if case["save"] else 1) + 2 * biases, "flops": 4 * B * m * d}
    return {"bytes": 2 * e * (B * d + 2 * m * d) + 3 * e * B * m + 2 * biases, "flops": 8 * B * m * d}


# ---- what the definitions give in 64 bits ----
def _value_and_slope(v, act):
    if act == "none":
        return v, torch.ones_like(v)
    if act == "relu":
        return torch.where(v > 0, v, 0.0), torch.where(v > 0, 1.0, 0.0).double()
    if act == "gelu":   # v Phi(v), Phi from the complementary error function, which keeps its digits far below zero
        below = 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
        return v * below, below + v * torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi)
    p = torch.sigmoid(v)
    return v * p, p + v * p * torch.sigmoid(-v)


def exact(case, seed):
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    x, act, B = wide["x"], case["act"], case["batch"]
    if case["kind"].startswith("linear"):
        W, m = wide["W"], case["d_out"]
        bias = wide.get("bias", torch.zeros(m, dtype=torch.float64, device="cuda"))
        place = s["active"].long() if s["active"] is not None else torch.arange(m, device="cuda")
        if case["kind"] == "linear":
            z = torch.addmm(bias[place], x, W.T)
            y = _value_and_slope(bias, act)[0].expand(B, m).clone()
            y[:, place] = _value_and_slope(z, act)[0]
            if case["residual"]:
                y += wide["residual"]
            return (y, z) if case["save"] else y
        whole = _value_and_slope(bias, act)[1].expand(B, m).clone()
        whole[:, place] = _value_and_slope(wide["z"], act)[1]
        whole *= wide["dy"]
        dz = whole[:, place]
        return torch.mm(dz, W), torch.mm(dz.T.contiguous(), x), whole.sum(dim=0) if case["bias"] else None
    if case["kind"] == "gated":
        zero = torch.zeros(case["d_out"], dtype=torch.float64, device="cuda")
        g, u = torch.addmm(wide.get("bg", zero), x, wide["Wg"].T), torch.addmm(wide.get("bu", zero), x, wide["Wu"].T)
        h = _value_and_slope(g, act)[0] * u
        return (h, g, u) if case["save"] else h
    value, slope = _value_and_slope(wide["g"], act)
    dg, du = wide["dh"] * wide["u"] * slope, wide["dh"] * value
    dx = torch.addmm(torch.mm(dg, wide["Wg"]), du, wide["Wu"])
    sums = (dg.sum(dim=0), du.sum(dim=0)) if case["bias"] else (None, None)
    return (dx, torch.mm(dg.T.contiguous(), x), torch.mm(du.T.contiguous(), x)) + sums
