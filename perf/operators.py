"""The passes by which the operators of a wider per-Gaussian decoder and its clipped training step are measured.

A decoder that is too wide for the fused preprocess runs over the Gaussians' embeddings, one row each: layer norm, a
matrix product with its bias, activation and residual, and the backward of both; its gradients and the scene's are
clipped by their global norm and taken by the Adam step. A case is one pass through one of these: ``norm_fwd``,
``norm_bwd``, ``linear_fwd``, ``linear_bwd``, ``clip`` (norm and clipping) or ``clip_step`` (norm, and the Adam step that
takes the clipping coefficient). Rows are Gaussians (one, when a single embedding is looked at; 3,000,000 in the
scenes of ``inputs.CONFIGS``), widths those of a decoder (from 3 outputs) up to 4,096.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5                      # layer norm
CLIP_EPS = 1e-6                 # beside the norm in the clipping coefficient
BETA1, BETA2, ADAM_EPS, STEP = 0.9, 0.999, 1e-15, 101
SCENE_ROWS = (3, 3, 4, 1, 48)   # means, log-scales, quaternions, opacity logits, SH coefficients
LR = (1.6e-4, 5e-3, 1e-3, 0.05, 1.25e-4)


def _norm(op, type_, rows, dim, add=False):
    return {"op": op, "type": type_, "rows": rows, "dim": dim, "add": add}


def _linear(op, type_, rows, n_in, n_out, act, residual=False, keep=False, grad="f32"):
    case = {"op": op, "type": type_, "rows": rows, "in": n_in, "out": n_out, "act": act}
    case.update({"residual": residual, "keep": keep} if op == "linear_fwd" else {"grad": grad})
    return case


def listed():
    return [
        # one embedding normalised: the latency of a call
        dict(_norm("norm_fwd", "f16", 1, 256), name="norm_row"),
        # training in fp32 with an odd width and an odd count of rows
        dict(_norm("norm_bwd", "f32", 100_003, 333), name="norm_odd_bwd"),
        # training in bfloat16 with wide rows; the skip connection's gradient joins dx
        dict(_norm("norm_bwd", "bf16", 16_384, 4_096, add=True), name="norm_wide_bwd"),
        # a single row through a wide layer, as when one embedding is decoded: the weights are read once
        dict(_linear("linear_fwd", "bf16", 1, 4_096, 4_096, "gelu", residual=True), name="linear_row"),
        # a decoder's hidden layer over every Gaussian of a 3M scene, keeping what its backward needs
        dict(_linear("linear_fwd", "f16", 3_000_000, 64, 128, "relu", keep=True), name="linear_scene"),
        # a wide layer over many rows: the matrix cores' rate
        dict(_linear("linear_fwd", "bf16", 8_192, 4_096, 4_096, "gelu", residual=True), name="linear_wide"),
        # fp32 with odd sizes, nothing aligned
        dict(_linear("linear_fwd", "f32", 5_003, 777, 333, "silu", residual=True), name="linear_odd_f32"),
        # a decoder's hidden layer in training over a million Gaussians, weight gradients in fp32 for Adam
        dict(_linear("linear_bwd", "f16", 1_000_000, 128, 128, "relu"), name="linear_scene_bwd"),
        # a wide layer in training, weight gradients in the weights' type
        dict(_linear("linear_bwd", "bf16", 8_192, 4_096, 4_096, "gelu", grad="same"), name="linear_wide_bwd"),
        # a small decoder's gradients, below the bound, as in most steps: the latency of a call (clipped in place, a
        # second pass on the same state would find the norm at the bound)
        {"op": "clip", "name": "clip_decoder", "type": "f32", "tensors": 8, "n": 2_144, "hit": False, "to32": False},
        # many ragged 16-bit gradients clipped into the fp32 arrays that the optimiser takes
        {"op": "clip", "name": "clip_many", "type": "bf16", "tensors": 60, "n": 1_000_000, "hit": True, "to32": True},
        # the clipped optimiser step of a 3M-Gaussian SH3 scene
        {"op": "clip_step", "name": "step_scene", "n": 3_000_000, "hit": True},
    ]


def draw(rng):
    """Sizes over the logarithm of the listed range, odd ones among them, every type and direction; bytes and flops are
    held below those of the largest listed cases of the operator."""
    def size(lo, hi, odd):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return v if odd or v < 16 else max(16, v // 16 * 16)

    op = rng.choice(("norm_fwd", "norm_bwd", "linear_fwd", "linear_bwd", "clip", "clip_step"))
    type_, odd = rng.choice(("f32", "f16", "bf16")), rng.random() < 0.4
    if op == "clip_step":
        return {"op": op, "n": size(1_000, 3_000_000, odd), "hit": rng.random() < 0.5}
    if op == "clip":
        tensors = size(1, 60, True)
        to32 = type_ != "f32" and rng.random() < 0.5
        return {"op": op, "type": type_, "tensors": tensors, "n": size(100, min(2_000_000, 60_000_000 // tensors), odd),
                "hit": to32, "to32": to32}
    if op.startswith("norm"):
        dim = size(3, 4_096, odd)
        rows = size(1, min(3_000_000, (1 << 25) // dim), True)
        return _norm(op, type_, rows, dim, add=op == "norm_bwd" and rng.random() < 0.5)
    n_in, n_out = size(16, 4_096, odd), size(3, 4_096, odd)
    # fp32 products run at a sixteenth of the 16-bit rate
    flops = 2.0e10 if type_ == "f32" else 1.2e11
    most = min(3_000_000.0, flops / (2.0 * n_in * n_out), 2.5e8 / (n_in + n_out))
    rows = size(1, max(2.0, most), True)
    act = rng.choice(("none", "relu", "gelu", "silu", "tanh", "sigmoid"))
    if op == "linear_fwd":
        return _linear(op, type_, rows, n_in, n_out, act, residual=rng.random() < 0.5, keep=rng.random() < 0.5)
    return _linear(op, type_, rows, n_in, n_out, act, grad=rng.choice(("f32", "same")))


# ---- a user's program -----------------------------------------------------------


def _normal(g, shape, sigma, mu=0.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEVICE).mul_(sigma).add_(mu).to(dtype)


def _lengths(case):
    """Lengths of the gradient tensors: weights of about n values with biases of odd lengths between them."""
    return [case["n"] if k % 2 == 0 else 1 + (case["n"] // 64 + 37 * k) % (case["n"] + 1) for k in range(case["tensors"])]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    op, t = case["op"], TYPES[case.get("type", "f32")]
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEVICE)  # noqa: E731
    s = {"case": case}
    if op.startswith("norm"):
        rows, dim = case["rows"], case["dim"]
        s.update(x=_normal(g, (rows, dim), 1.5, 0.5, t), w=_normal(g, (dim,), 0.2, 1.0), b=_normal(g, (dim,), 0.1))
        if op == "norm_fwd":
            s.update(y=empty(rows, dim, dtype=t), mean=empty(rows), rstd=empty(rows))
        else:
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt()
            s.update(dy=_normal(g, (rows, dim), 1e-2, 0.0, t), dx=empty(rows, dim, dtype=t), dw=empty(dim), db=empty(dim))
            s["add"] = _normal(g, (rows, dim), 1e-2, 0.0, t) if case["add"] else None
    elif op.startswith("linear"):
        rows, n_in, n_out = case["rows"], case["in"], case["out"]
        s.update(x=_normal(g, (rows, n_in), 1.0, 0.0, t), w=_normal(g, (n_out, n_in), n_in ** -0.5, 0.0, t))
        if op == "linear_fwd":
            s.update(b=_normal(g, (n_out,), 0.1), y=empty(rows, n_out, dtype=t))
            s["r"] = _normal(g, (rows, n_out), 1.0, 0.0, t) if case["residual"] else None
            s["z"] = empty(rows, n_out, dtype=t) if case["keep"] else None
        else:
            s.update(z=_normal(g, (rows, n_out), 1.0, 0.0, t), dy=_normal(g, (rows, n_out), 1e-2, 0.0, t),
                     dx=empty(rows, n_in, dtype=t), db=empty(n_out),
                     dw=empty(n_out, n_in, dtype=t if case["grad"] == "same" else torch.float32))
    elif op == "clip":
        lengths = _lengths(case)
        s["grads"] = [_normal(g, (n,), 10.0 ** (-3 + k % 3), 0.0, t) for k, n in enumerate(lengths)]
        s["out"] = [empty(n) for n in lengths] if case["to32"] else None
        s["result"] = empty(2)
        size = math.sqrt(sum(n * 10.0 ** (2 * (-3 + k % 3)) for k, n in enumerate(lengths)))
        s["max_norm"] = size * (0.25 if case["hit"] else 4.0)
    else:
        n = case["n"]
        s["tensors"] = []
        for rows, lr in zip(SCENE_ROWS, LR):
            s["tensors"].append(dict(param=_normal(g, (rows, n), 1.0), grad=_normal(g, (rows, n), 1e-4),
                                     exp_avg=_normal(g, (rows, n), 1e-5), param_half=None, rows=rows, n=n, beta2=BETA2,
                                     exp_avg_sq=torch.rand((rows, n), generator=g, device=DEVICE).add_(0.1).mul_(1e-9),
                                     lr=[lr] * rows))
        s["result"] = empty(2)
        s["max_norm"] = 1e-4 * math.sqrt(n * sum(SCENE_ROWS)) * (0.25 if case["hit"] else 4.0)
    return s


def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "tanh":
        return torch.tanh(z)
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name in ("silu", "sigmoid"):
        p = 1 / (1 + torch.exp(-z))
        return p * (1 - p) if name == "sigmoid" else p * (1 + z * (1 - p))
    if name == "tanh":
        t = torch.tanh(z)
        return 1 - t * t
    return torch.ones_like(z)


def _plain(s):
    case = s["case"]
    op, t = case["op"], TYPES[case.get("type", "f32")]
    f = lambda name: None if s[name] is None else s[name].float()  # noqa: E731
    if op == "norm_fwd":
        x = f("x")
        mean = x.sum(1, keepdim=True) / case["dim"]
        d = x - mean
        rstd = 1 / torch.sqrt((d * d).sum(1, keepdim=True) / case["dim"] + EPS)
        y = d * rstd * s["w"] + s["b"]
        return {"y": y.to(t), "mean": mean.view(-1), "rstd": rstd.view(-1)}
    if op == "norm_bwd":
        rstd, dy = s["rstd"].unsqueeze(1), f("dy")
        xh = (f("x") - s["mean"].unsqueeze(1)) * rstd
        gr = dy * s["w"]
        dx = rstd * (gr - gr.sum(1, keepdim=True) / case["dim"] - xh * ((gr * xh).sum(1, keepdim=True) / case["dim"]))
        if s["add"] is not None:
            dx = dx + f("add")
        return {"dx": dx.to(t), "dw": (dy * xh).sum(0), "db": dy.sum(0)}
    if op == "linear_fwd":
        z = f("x") @ f("w").t() + s["b"]
        y = _act(case["act"], z)
        if s["r"] is not None:
            y = y + f("r")
        return {"y": y.to(t), "z": z.to(t)} if case["keep"] else {"y": y.to(t)}
    if op == "linear_bwd":
        dz = f("dy") * _act_slope(case["act"], f("z"))
        return {"dx": (dz @ f("w")).to(t), "dw": (dz.t() @ f("x")).to(s["dw"].dtype), "db": dz.sum(0)}
    grads = [p["grad"] for p in s["tensors"]] if op == "clip_step" else s["grads"]
    total = sum((v.float() * v.float()).sum() for v in grads)
    norm = torch.sqrt(total)
    c = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0)
    result = torch.stack([norm, c])
    if op == "clip":
        if case["to32"]:
            return {"result": result, "grads": [v.float() * c for v in grads]}
        for v in grads:
            v.copy_(v.float() * c)
        return {"result": result, "grads": grads}
    out = {"result": result}
    for k, p in enumerate(s["tensors"]):
        gr = p["grad"] * c
        p["exp_avg"].mul_(BETA1).add_(gr * (1 - BETA1))
        p["exp_avg_sq"].mul_(BETA2).add_(gr * gr * (1 - BETA2))
        denom = torch.sqrt(p["exp_avg_sq"]) / math.sqrt(1 - BETA2 ** STEP) + ADAM_EPS
        p["param"].sub_(p["exp_avg"] / denom * (p["lr"][0] / (1 - BETA1 ** STEP)))
        out.update({"param%d" % k: p["param"], "m%d" % k: p["exp_avg"], "v%d" % k: p["exp_avg_sq"]})
    return out


def _scratch(s, size):
    """The workspace that a program sizes once and keeps."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(size(), 256), dtype=torch.uint8, device=DEVICE)
    return s["workspace"]


def _kernels(s):
    from paper_2609_05255_amd import gsraster as gs
    case = s["case"]
    op = case["op"]
    if op == "norm_fwd":
        gs.gs_layer_norm_fwd(s["x"], s["w"], s["b"], EPS, s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "norm_bwd":
        ws = _scratch(s, lambda: gs.gs_layer_norm_workspace_size(s["x"]))
        gs.gs_layer_norm_bwd(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], ws, add=s["add"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if op == "linear_fwd":
        ws = _scratch(s, lambda: gs.gs_linear_workspace_size(s["x"], s["w"], case["act"]))
        gs.gs_linear_fwd(s["x"], s["w"], s["b"], s["y"], ws, act=case["act"], residual=s["r"], z=s["z"])
        return {"y": s["y"], "z": s["z"]} if case["keep"] else {"y": s["y"]}
    if op == "linear_bwd":
        ws = _scratch(s, lambda: gs.gs_linear_workspace_size(s["x"], s["w"], case["act"]))
        gs.gs_linear_bwd(s["dy"], s["x"], s["w"], s["z"], s["dx"], s["dw"], s["db"], ws, act=case["act"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if "set" not in s:
        grads = [p["grad"] for p in s["tensors"]] if op == "clip_step" else s["grads"]
        s["set"] = gs.GradSet(grads, out=s.get("out"))
    ws = _scratch(s, lambda: gs.gs_grad_workspace_size(s["set"]))
    if op == "clip":
        gs.gs_grad_clip(s["set"], s["max_norm"], s["result"], ws)
        return {"result": s["result"], "grads": s["out"] if case["to32"] else s["grads"]}
    gs.gs_grad_norm(s["set"], s["max_norm"], s["result"], ws)
    gs.gs_adam_step(s["tensors"], BETA1, ADAM_EPS, STEP, grad_scale=s["result"][1:])
    out = {"result": s["result"]}
    for k, p in enumerate(s["tensors"]):
        out.update({"param%d" % k: p["param"], "m%d" % k: p["exp_avg"], "v%d" % k: p["exp_avg_sq"]})
    return out


def run(state):
    return _kernels(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------


def work(case):
    op, e = case["op"], 4 if case.get("type", "f32") == "f32" else 2
    if op.startswith("norm"):
        v = case["rows"] * case["dim"]
        if op == "norm_fwd":
            return {"bytes": 2 * v * e + 8 * case["rows"] + 8 * case["dim"], "flops": 8.0 * v}
        return {"bytes": (3 + case["add"]) * v * e + 8 * case["rows"] + 12 * case["dim"], "flops": 14.0 * v}
    if op.startswith("linear"):
        rows, n_in, n_out = case["rows"], case["in"], case["out"]
        product = 2.0 * rows * n_in * n_out
        if op == "linear_fwd":
            return {"bytes": e * (rows * n_in + n_in * n_out + rows * n_out * (1 + case["residual"] + case["keep"]))
                    + 4 * n_out, "flops": product}
        return {"bytes": e * (2 * rows * n_in + n_in * n_out + rows * n_out * (1 if case["act"] == "none" else 2))
                + (4 if case["grad"] == "f32" else e) * n_in * n_out + 4 * n_out, "flops": 2 * product}
    if op == "clip":
        v = sum(_lengths(case))
        return {"bytes": v * (e + (4 if case["to32"] else e if case["hit"] else 0)) + 8, "flops": 3.0 * v}
    v = case["n"] * sum(SCENE_ROWS)
    return {"bytes": 28 * v + 8, "flops": 16.0 * v}


# ---- the same in 64 bits ----------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    d = lambda name: s[name].double()  # noqa: E731
    if op == "norm_fwd":
        x = d("x")
        mean, var = x.mean(dim=1), x.var(dim=1, unbiased=False)
        rstd = (var + EPS) ** -0.5
        return {"y": torch.addcmul(d("b"), (x - mean[:, None]) * rstd[:, None], d("w")), "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        # dx is the gradient's part that is orthogonal, in each row, to the ones and to x's deviations
        rstd = d("rstd")[:, None]
        xh = (d("x") - d("mean")[:, None]) * rstd
        up = d("dy") * d("w")
        dx = (up - up.mean(dim=1, keepdim=True) - xh * (up * xh).mean(dim=1, keepdim=True)) * rstd
        dx = dx if s["add"] is None else dx + d("add")
        return {"dx": dx, "dw": torch.einsum("rd,rd->d", d("dy"), xh), "db": d("dy").sum(dim=0)}
    if op == "linear_fwd":
        z = torch.addmm(d("b"), d("x"), d("w").T.contiguous())
        y = {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * torch.special.ndtr(v),
             "silu": lambda v: v * torch.sigmoid(v), "tanh": torch.tanh, "sigmoid": torch.sigmoid}[case["act"]](z)
        y = y if s["r"] is None else y + d("r")
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    if op == "linear_bwd":
        z = d("z")
        pdf = lambda v: torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi)  # noqa: E731
        slope = {"none": torch.ones_like, "relu": lambda v: torch.heaviside(v, torch.zeros_like(v)),
                 "gelu": lambda v: torch.special.ndtr(v) + v * pdf(v),
                 "silu": lambda v: torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v),
                 "tanh": lambda v: torch.cosh(v) ** -2, "sigmoid": lambda v: torch.sigmoid(v) * torch.sigmoid(-v)}
        dz = d("dy") * slope[case["act"]](z)
        return {"dx": dz @ d("w"), "dw": dz.T.contiguous() @ d("x"), "db": dz.sum(dim=0)}
    grads = [p["grad"].double() for p in s["tensors"]] if op == "clip_step" else [v.double() for v in s["grads"]]
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(v) for v in grads]))
    c = (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
    out = {"result": torch.stack([norm, c])}
    if op == "clip":
        out["grads"] = [v * c for v in grads]
        return out
    # what the optimiser is given as fp32 values
    f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    b1, b2 = f32(BETA1), f32(BETA2)
    for k, (p, v) in enumerate(zip(s["tensors"], grads)):
        m = b1 * p["exp_avg"].double() + (1 - b1) * c * v
        q = b2 * p["exp_avg_sq"].double() + (1 - b2) * (c * v) ** 2
        step = f32(p["lr"][0]) * (m / (1 - b1 ** STEP)) / ((q / (1 - b2 ** STEP)).sqrt() + f32(ADAM_EPS))
        out.update({"param%d" % k: p["param"].double() - step, "m%d" % k: m, "v%d" % k: q})
    return out
