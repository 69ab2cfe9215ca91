"""The passes by which the operators of a codebook and of a mixture of decoders are measured.

A scene's embeddings may come from a codebook, one index for each Gaussian (``lookup_fwd``, ``lookup_bwd``: the codebook's
gradient, with the sort of the rows by their entry that it needs). A mixture of decoders sends each Gaussian's row to a few
of its experts: ``route_fwd`` and ``route_bwd`` choose and weigh them from a row of logits, ``dispatch_fwd`` sorts the rows
by expert and copies them there, ``dispatch_bwd`` adds their gradients up, ``combine_fwd`` and ``combine_bwd`` bring the
experts' results back with their weights, and ``experts_fwd`` and ``experts_bwd`` are the experts' layers over the sorted
rows. Rows are Gaussians, from one that is looked at to the 3,000,000 of the scenes of ``inputs.CONFIGS``; widths are those
of embeddings and decoders.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _lookup(op, type_, rows, dim, entries, grad="f32"):
    case = {"op": op, "type": type_, "rows": rows, "dim": dim, "entries": entries}
    return dict(case, grad=grad) if op == "lookup_bwd" else case


def _route(op, type_, rows, experts, k, normalise, masked=False):
    return {"op": op, "type": type_, "rows": rows, "experts": experts, "k": k, "normalise": normalise, "masked": masked}


def _move(op, type_, rows, dim, experts, k, add=False, dropped=False):
    return {"op": op, "type": type_, "rows": rows, "dim": dim, "experts": experts, "k": k, "add": add, "dropped": dropped}


def _experts(op, type_, rows, experts, n_in, n_out, act, keep=False, grad="f32"):
    case = {"op": op, "type": type_, "rows": rows, "experts": experts, "in": n_in, "out": n_out, "act": act}
    return dict(case, keep=keep) if op == "experts_fwd" else dict(case, grad=grad)


def listed():
    return [
        # the embedding of one Gaussian that is looked at: the latency of a call
        dict(_lookup("lookup_fwd", "f16", 1, 256, 4_096), name="lookup_one"),
        # training a codebook over a 3M scene, entries used as unevenly as words are; the gradient in fp32 for Adam
        dict(_lookup("lookup_bwd", "f16", 3_000_000, 64, 65_536), name="lookup_scene_bwd"),
        # a codebook of more entries than there are rows, an odd width, the gradient in the codebook's type
        dict(_lookup("lookup_bwd", "bf16", 50_001, 333, 150_007, grad="same"), name="lookup_odd_bwd"),
        # the router of a mixture over a million Gaussians
        dict(_route("route_fwd", "f16", 1_000_000, 64, 2, True), name="route_scene"),
        # weights out of the softmax over all experts, some of which are masked; odd sizes; the logits' gradient
        dict(_route("route_bwd", "bf16", 100_003, 37, 3, False, masked=True), name="route_odd_bwd"),
        # a million Gaussians' rows sorted by expert and copied there
        dict(_move("dispatch_fwd", "f16", 1_000_000, 128, 16, 2), name="dispatch_scene"),
        # results of experts added up in fp32, odd sizes, some choices dropped (an expert that takes no more rows)
        dict(_move("combine_fwd", "f32", 20_003, 333, 37, 3, add=True, dropped=True), name="combine_odd"),
        # wide rows in training: the gradients of the experts' results and of their weights
        dict(_move("combine_bwd", "bf16", 8_192, 4_096, 8, 2), name="combine_wide_bwd"),
        # four Gaussians decoded by two experts each: the weights of the experts that have a row are read once
        dict(_experts("experts_fwd", "bf16", 8, 16, 2_048, 2_048, "gelu"), name="experts_few"),
        # wide experts over many rows: the matrix cores' rate
        dict(_experts("experts_fwd", "bf16", 16_384, 8, 2_048, 2_048, "gelu", keep=True), name="experts_wide"),
        # a mixture's hidden layer in training over a million Gaussians, weight gradients in fp32 for Adam
        dict(_experts("experts_bwd", "f16", 1_000_000, 16, 64, 128, "silu"), name="experts_scene_bwd"),
        # fp32 with odd sizes, nothing aligned
        dict(_experts("experts_bwd", "f32", 5_003, 7, 333, 215, "tanh"), name="experts_odd_bwd"),
    ]


def draw(rng):
    """Sizes over the logarithm of the listed range, odd ones among them, every operator, type and direction; bytes and
    flops are held below those of the largest listed cases of the operator."""
    def size(lo, hi, odd=True):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return v if odd or v < 16 else max(16, v // 16 * 16)

    op = rng.choice(("lookup_fwd", "lookup_bwd", "route_fwd", "route_bwd", "dispatch_fwd", "dispatch_bwd", "combine_fwd",
                     "combine_bwd", "experts_fwd", "experts_bwd"))
    type_, odd, flag = rng.choice(("f32", "f16", "bf16")), rng.random() < 0.4, rng.random() < 0.5
    most = 2 if type_ == "f32" else 1   # fp32 values are twice the bytes
    if op.startswith("lookup"):
        dim = size(3, 1_024, odd)
        rows = size(1, min(3_000_000, 190_000_000 // most // dim))
        return _lookup(op, type_, rows, dim, size(1, min(1_000_000, 50_000_000 // dim)), rng.choice(("f32", "same")))
    if op.startswith("route"):
        experts = size(2, 256, odd)
        k = rng.randint(1, min(8, experts))   # (the weight of one choice, normalised, is 1: its gradient is 0)
        return _route(op, type_, size(1, min(1_000_000, 64_000_000 // most // experts)), experts, k,
                      rng.random() < 0.5 and (k > 1 or op == "route_fwd"), masked=flag)
    if op[:8] in ("dispatch", "combine_"):
        k, dim = rng.randint(1, 4), size(3, 4_096, odd)
        rows = size(1, min(1_000_000, 67_000_000 // most // (k * dim)))
        return _move(op, type_, rows, dim, size(4, 256), k, add=flag and op in ("dispatch_bwd", "combine_fwd"),
                     dropped=rng.random() < 0.3)
    experts, n_in, n_out = size(2, 64), size(16, 2_048, odd), size(3, 2_048, odd)
    while experts * n_in * n_out > 67_000_000:
        experts //= 2
    # fp32 products run at a sixteenth of the 16-bit rate
    flops = 1.0e10 if type_ == "f32" else 6.0e10
    rows = size(1, max(2, min(1_000_000, int(flops / (2.0 * n_in * n_out)), 190_000_000 // most // (n_in + n_out))))
    act = rng.choice(("none", "relu", "gelu", "silu", "tanh", "sigmoid"))
    return _experts(op, type_, rows, experts, n_in, n_out, act, keep=flag, grad=rng.choice(("f32", "same")))


# ---- a user's program -----------------------------------------------------------


def _normal(g, shape, sigma, mu=0.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEVICE).mul_(sigma).add_(mu).to(dtype)


def _lengths(case):
    """Rows of each expert: as uneven as the shares 1, 1/2, 1/3, ... are, the first experts' rows rounded up; the last ones
    of a few rows have none."""
    left, out = case["rows"], []
    total = sum(1.0 / (e + 1) for e in range(case["experts"]))
    for e in range(case["experts"]):
        out.append(min(left, math.ceil(case["rows"] / total / (e + 1))))
        left -= out[-1]
    out[0] += left
    return out


def _argsort(keys):
    return torch.sort(keys, stable=True).indices


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    op, t = case["op"], TYPES[case["type"]]
    rows = case["rows"]
    empty = lambda *shape, dtype=t: torch.empty(shape, dtype=dtype, device=DEVICE)  # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=g, device=DEVICE)  # noqa: E731
    s = {"case": case}
    if op.startswith("lookup"):
        entries, dim = case["entries"], case["dim"]
        # entry v is used in proportion to 1 / (v + 1); one row in 64 has none
        index = torch.exp(uniform(rows).double() * math.log(entries + 1)).long().clamp_(1, entries) - 1
        s["index"] = torch.where(uniform(rows) < 1 / 64, -1, index).int() if rows > 1 else index.int()
        s["scale"] = math.sqrt(dim)
        if op == "lookup_fwd":
            s.update(table=_normal(g, (entries, dim), dim ** -0.5, 0.0, t), y=empty(rows, dim))
        else:
            s.update(dy=_normal(g, (rows, dim), 1e-2, 0.0, t),
                     dtable=empty(entries, dim, dtype=t if case["grad"] == "same" else torch.float32))
        return s
    if op.startswith("route"):
        experts, k = case["experts"], case["k"]
        s["logits"] = _normal(g, (rows, experts), 1.5, 0.0, t)
        if case["masked"]:   # one expert in eight, and every expert of one row in 64
            hidden = (uniform(rows, experts) < 1 / 8) | (uniform(rows, 1) < 1 / 64)
            s["logits"].masked_fill_(hidden, -math.inf)
        s.update(expert=empty(rows, k, dtype=torch.int32), weight=empty(rows, k, dtype=torch.float32))
        if op == "route_bwd":
            expert, weight = _choose(s["logits"].float(), k, case["normalise"])
            s.update(expert=expert, weight=weight.float(), dweight=_normal(g, (rows, k), 1e-2),
                     dlogits=empty(rows, experts))
        return s
    if op.startswith("experts"):
        n, n_in, n_out = case["experts"], case["in"], case["out"]
        lengths = _lengths(case)
        s["ends"] = [sum(lengths[:e]) for e in range(n + 1)]
        s["offsets"] = torch.tensor(s["ends"], dtype=torch.int32, device=DEVICE)
        s.update(x=_normal(g, (rows, n_in), 1.0, 0.0, t), w=_normal(g, (n, n_out, n_in), n_in ** -0.5, 0.0, t))
        if op == "experts_fwd":
            s.update(b=_normal(g, (n, n_out), 0.1), y=empty(rows, n_out))
            s["z"] = empty(rows, n_out) if case["keep"] else None
        else:
            s.update(z=_normal(g, (rows, n_out), 1.0, 0.0, t), dy=_normal(g, (rows, n_out), 1e-2, 0.0, t),
                     dx=empty(rows, n_in), db=empty(n, n_out, dtype=torch.float32),
                     dw=empty(n, n_out, n_in, dtype=t if case["grad"] == "same" else torch.float32))
        return s
    # the k choices of a row are different experts, some of which are chosen far more often
    dim, experts, k = case["dim"], case["experts"], case["k"]
    expert = torch.topk(_normal(g, (experts,), 1.0) - torch.log(-torch.log(uniform(rows, experts))), k, dim=1).indices
    if case["dropped"]:
        expert = torch.where(uniform(rows, k) < 1 / 8, -1, expert)
    s["expert"] = expert.int()
    if op != "dispatch_fwd":
        flat = expert.reshape(-1)
        key = torch.where(flat < 0, experts, flat)
        order = _argsort(key)
        place = torch.empty_like(order)
        place[order] = torch.arange(rows * k, device=DEVICE)
        s["order"], s["place"] = order.int(), torch.where(flat < 0, -1, place).int()
        s["offsets"] = torch.searchsorted(key[order], torch.arange(experts + 1, device=DEVICE)).int()
    weight = uniform(rows, k)
    s["weight"] = weight / weight.sum(1, keepdim=True)
    if op == "dispatch_fwd":
        # (rows of experts' inputs behind the last chosen one stay as they are)
        s.update(x=_normal(g, (rows, dim), 1.0, 0.0, t), xs=torch.zeros(rows * k, dim, dtype=t, device=DEVICE))
    elif op == "dispatch_bwd":
        s.update(dxs=_normal(g, (rows * k, dim), 1e-2, 0.0, t), dx=empty(rows, dim))
        s["add"] = _normal(g, (rows, dim), 1e-2, 0.0, t) if case["add"] else None
    else:
        s["ys"] = _normal(g, (rows * k, dim), 1.0, 0.0, t)
        if op == "combine_fwd":
            s["y"] = empty(rows, dim)
            s["add"] = _normal(g, (rows, dim), 1.0, 0.0, t) if case["add"] else None
        else:
            s.update(dy=_normal(g, (rows, dim), 1e-2, 0.0, t), dweight=empty(rows, k, dtype=torch.float32),
                     dys=torch.zeros(rows * k, dim, dtype=t, device=DEVICE))
    return s


def _choose(logits, k, normalise):
    """Experts of the k largest logits of each row (the lowest of equal ones first; -1 where none is left) and their
    weights."""
    top, expert = torch.sort(logits, dim=1, descending=True, stable=True)
    top, none = top[:, :k], torch.isneginf(top[:, :k])
    most = torch.where(none[:, :1], 0.0, top[:, :1])
    e = torch.exp(top - most)
    total = e.sum(1, keepdim=True) if normalise else torch.exp(logits - most).sum(1, keepdim=True)
    return torch.where(none, -1, expert[:, :k]).int(), torch.where(none, 0.0, e / total)


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


def _gathered(rows, place, k):
    """Rows at the places of each row's k choices, [rows][k][dim], zero where there is none."""
    at = place.long().view(-1, k)
    return torch.where((at < 0).unsqueeze(2), 0.0, rows.float()[at.clamp(min=0)])


def _plain(s):
    case = s["case"]
    op, t = case["op"], TYPES[case["type"]]
    if op == "lookup_fwd":
        at = s["index"].long()
        y = s["table"][at.clamp(min=0)].float() * s["scale"]
        return torch.where((at < 0).unsqueeze(1), 0.0, y).to(t)
    if op == "lookup_bwd":
        # eight sums for each entry, added up at the end: some entries have hundreds of thousands of rows
        copy = torch.arange(case["rows"], device=DEVICE) % 8
        at = torch.where(s["index"] < 0, case["entries"], s["index"]) * 8 + copy
        sums = torch.zeros((case["entries"] + 1) * 8, case["dim"], device=DEVICE).index_add_(0, at, s["dy"].float())
        return (sums.view(-1, 8, case["dim"])[:-1].sum(1) * s["scale"]).to(s["dtable"].dtype)
    if op == "route_fwd":
        expert, weight = _choose(s["logits"].float(), case["k"], case["normalise"])
        return {"expert": expert, "weight": weight}
    if op == "route_bwd":
        logits, w, dw = s["logits"].float(), s["weight"], s["dweight"]
        at, none = s["expert"].long().clamp(min=0), s["expert"] < 0
        inner = (dw * w).sum(1, keepdim=True)
        # (a row's choices are different experts: the places that are added to are, but for the zeros of those left out)
        chosen = torch.where(none, 0.0, w * dw)
        if case["normalise"]:
            dl = torch.zeros_like(logits).scatter_add_(1, at, torch.where(none, 0.0, w * (dw - inner)))
        else:
            most = logits.max(1, keepdim=True).values
            e = torch.exp(logits - torch.where(torch.isneginf(most), 0.0, most))
            total = e.sum(1, keepdim=True)
            p = e / torch.where(total > 0, total, 1.0)
            dl = (-p * inner).scatter_add_(1, at, chosen)
        return dl.to(t)
    if op == "dispatch_fwd":
        experts, flat = case["experts"], s["expert"].view(-1).long()
        key = torch.where(flat < 0, experts, flat)
        order = _argsort(key)
        place = torch.empty_like(order)
        place[order] = torch.arange(order.numel(), device=DEVICE)
        offsets = torch.searchsorted(key[order], torch.arange(experts + 1, device=DEVICE))
        moved = torch.where((key[order] < experts).unsqueeze(1), s["x"][order // case["k"]], s["xs"])
        return {"order": order.int(), "place": torch.where(flat < 0, -1, place).int(), "offsets": offsets.int(), "xs": moved}
    if op in ("dispatch_bwd", "combine_fwd"):
        v = _gathered(s["dxs"] if op == "dispatch_bwd" else s["ys"], s["place"], case["k"])
        v = (v if op == "dispatch_bwd" else v * s["weight"].unsqueeze(2)).sum(1)
        return (v if s["add"] is None else v + s["add"].float()).to(t)
    if op == "combine_bwd":
        dy, order = s["dy"].float(), s["order"].long()
        dweight = (_gathered(s["ys"], s["place"], case["k"]) * dy.unsqueeze(1)).sum(2)
        dys = s["weight"].view(-1)[order].unsqueeze(1) * dy[order // case["k"]]
        there = (s["place"][order] >= 0).unsqueeze(1)
        return {"dys": torch.where(there, dys.to(t), s["dys"]), "dweight": dweight}
    parts = zip(s["ends"][:-1], s["ends"][1:], s["w"])
    if op == "experts_fwd":
        z = torch.cat([s["x"][a:b].float() @ w.float().t() + v for (a, b, w), v in zip(parts, s["b"])])
        y = _act(case["act"], z).to(t)
        return {"y": y, "z": z.to(t)} if case["keep"] else {"y": y}
    dz = s["dy"].float() * _act_slope(case["act"], s["z"].float())
    dx, dw, db = zip(*((dz[a:b] @ w.float(), dz[a:b].t() @ s["x"][a:b].float(), dz[a:b].sum(0)) for a, b, w in parts))
    return {"dx": torch.cat(dx).to(t), "dw": torch.stack(dw).to(s["dw"].dtype), "db": torch.stack(db)}


def _scratch(s, name, size):
    """A workspace that a program sizes once and keeps."""
    if name not in s:
        s[name] = torch.empty(max(size(), 256), dtype=torch.uint8, device=DEVICE)
    return s[name]


def _order(s, count, groups, lookup=False):
    """The arrays that sorting rows fills, which a program keeps (a lookup's gradient takes the sorted keys, rows on their
    way back their places); with the sort's result where that was prepared."""
    from paper_2609_05255_amd import gsraster as gs
    if "plan" not in s:
        s["plan"] = gs.RowOrder(count, groups, device=DEVICE, sorted=lookup, place=not lookup)
        if "order" in s:
            s["plan"].order, s["plan"].place, s["plan"].offsets = s["order"], s["place"], s["offsets"]
    return s["plan"]


def _kernels(s):
    from paper_2609_05255_amd import gsraster as gs
    case = s["case"]
    op, rows = case["op"], case["rows"]
    if op == "lookup_fwd":
        gs.gs_embedding_fwd(s["table"], s["index"], s["scale"], s["y"])
        return s["y"]
    if op == "lookup_bwd":
        plan = _order(s, rows, case["entries"], lookup=True)
        gs.gs_sort_rows(s["index"], plan, _scratch(s, "sort", lambda: gs.gs_sort_rows_workspace_size(plan)))
        gs.gs_embedding_bwd(s["dy"], plan, s["scale"], s["dtable"],
                            _scratch(s, "sums", lambda: gs.gs_embedding_workspace_size(s["dy"])))
        return s["dtable"]
    if op == "route_fwd":
        gs.gs_route_fwd(s["logits"], s["expert"], s["weight"], normalise=case["normalise"])
        return {"expert": s["expert"], "weight": s["weight"]}
    if op == "route_bwd":
        gs.gs_route_bwd(s["dweight"], s["logits"], s["expert"], s["weight"], s["dlogits"], normalise=case["normalise"])
        return s["dlogits"]
    if op.startswith("experts"):
        ws = _scratch(s, "workspace", lambda: gs.gs_experts_workspace_size(s["x"], s["w"], case["act"]))
        if op == "experts_fwd":
            gs.gs_experts_fwd(s["x"], s["offsets"], s["w"], s["b"], s["y"], ws, act=case["act"], z=s["z"])
            return {"y": s["y"], "z": s["z"]} if case["keep"] else {"y": s["y"]}
        gs.gs_experts_bwd(s["dy"], s["x"], s["offsets"], s["w"], s["z"], s["dx"], s["dw"], s["db"], ws, act=case["act"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    plan = _order(s, rows * case["k"], case["experts"])
    if op == "dispatch_fwd":
        gs.gs_sort_rows(s["expert"], plan, _scratch(s, "sort", lambda: gs.gs_sort_rows_workspace_size(plan)))
        gs.gs_dispatch_fwd(s["x"], plan, s["xs"])
        return {"order": plan.order, "place": plan.place, "offsets": plan.offsets, "xs": s["xs"]}
    if op == "dispatch_bwd":
        gs.gs_dispatch_bwd(s["dxs"], plan, s["dx"], add=s["add"])
        return s["dx"]
    if op == "combine_fwd":
        gs.gs_combine_fwd(s["ys"], plan, s["weight"], s["y"], residual=s["add"])
        return s["y"]
    gs.gs_combine_bwd(s["dy"], s["ys"], plan, s["weight"], s["dys"], s["dweight"])
    return {"dys": s["dys"], "dweight": s["dweight"]}


def run(state):
    return _kernels(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------


def work(case):
    op, e, rows = case["op"], 4 if case["type"] == "f32" else 2, case["rows"]
    if op.startswith("lookup"):
        v, entries = rows * case["dim"], case["entries"]
        if op == "lookup_fwd":   # (entries that a row uses are read once: log-uniform ones, about as many as this)
            used = sum(-math.expm1(rows * math.log1p(-min(0.999, c / math.log(entries + 1)))) * n
                       for c, n in _shares(entries))
            return {"bytes": v * e + 4 * rows + used * case["dim"] * e, "flops": 1.0 * v}
        return {"bytes": v * e + 4 * rows + entries * case["dim"] * (4 if case["grad"] == "f32" else e), "flops": 1.0 * v}
    if op.startswith("route"):
        v, k = rows * case["experts"], case["k"]
        if op == "route_fwd":
            return {"bytes": v * e + 8 * rows * k, "flops": 4.0 * v}
        return {"bytes": v * e * (1 if case["normalise"] else 2) + 12 * rows * k, "flops": (1.0 if case["normalise"] else 6.0) * v}
    if op.startswith("experts"):
        n_in, n_out = case["in"], case["out"]
        used = sum(n > 0 for n in _lengths(case)) * n_in * n_out
        product = 2.0 * rows * n_in * n_out
        if op == "experts_fwd":
            return {"bytes": e * (rows * n_in + used + rows * n_out * (1 + case["keep"])) + 4 * case["experts"] * n_out,
                    "flops": product}
        return {"bytes": e * (2 * rows * n_in + used + rows * n_out * (1 if case["act"] == "none" else 2))
                + case["experts"] * n_out * (4 + n_in * (4 if case["grad"] == "f32" else e)), "flops": 2 * product}
    k, v = case["k"], rows * case["dim"]
    moved = k * v * (7 / 8 if case["dropped"] else 1)
    if op == "dispatch_fwd":
        return {"bytes": (v + moved) * e + 12 * rows * k + 4 * case["experts"], "flops": 0.0}
    if op == "dispatch_bwd":
        return {"bytes": (v * (1 + case["add"]) + moved) * e + 4 * rows * k, "flops": 1.0 * k * v}
    if op == "combine_fwd":
        return {"bytes": (v * (1 + case["add"]) + moved) * e + 8 * rows * k, "flops": 2.0 * k * v}
    return {"bytes": (v + 2 * moved) * e + 12 * rows * k, "flops": 3.0 * k * v}


def _shares(entries):
    """(share times log(entries + 1), how many) of the entries, in groups of like ones."""
    first, out = 0, []
    while first < entries:
        n = min(entries - first, max(1, first // 16))
        out.append((math.log1p(n / (first + 1)) / n, n))
        first += n
    return out


# ---- the same in 64 bits ----------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    d = lambda name: s[name].double()  # noqa: E731
    if op == "lookup_fwd":
        # the product with a zero row behind the table's
        table = torch.cat([d("table"), torch.zeros(1, case["dim"], dtype=torch.float64, device=DEVICE)])
        return table.index_select(0, s["index"].long() % (case["entries"] + 1)) * s["scale"]
    if op == "lookup_bwd":
        # each row added to its entry's, those without one to a row behind the table's
        out = torch.zeros(case["entries"] + 1, case["dim"], dtype=torch.float64, device=DEVICE)
        out.index_add_(0, s["index"].long() % (case["entries"] + 1), d("dy"))
        return out[:-1] * s["scale"]
    if op == "route_fwd":
        # the number of experts before each one, larger or equal and lower, by counting; then the ones below k
        logits, k, experts = d("logits"), case["k"], case["experts"]
        rank = torch.zeros(logits.shape, dtype=torch.int32, device=DEVICE)
        for j in range(experts):
            other = logits[:, j:j + 1]
            rank += other > logits
            rank[:, j + 1:] += other == logits[:, j + 1:]
        chosen = (rank < k) & ~torch.isneginf(logits)
        masked = logits.masked_fill(~chosen, -math.inf) if case["normalise"] else logits
        p = torch.exp(logits - torch.logsumexp(masked, 1, keepdim=True))
        expert = torch.full((case["rows"], k), -1, dtype=torch.int32, device=DEVICE)
        weight = torch.zeros(case["rows"], k, dtype=torch.float64, device=DEVICE)
        r, c = chosen.nonzero(as_tuple=True)
        expert[r, rank[r, c].long()] = c.int()
        weight[r, rank[r, c].long()] = p[r, c]
        return {"expert": expert, "weight": weight}
    if op == "route_bwd":
        # the gradient of sum w dw: of the weights as given where they are normalised, else of the softmax
        logits, dw, none = d("logits"), d("dweight"), s["expert"] < 0
        full = torch.zeros_like(logits)
        r, j = (~none).nonzero(as_tuple=True)
        full[r, s["expert"][r, j].long()] = dw[r, j]
        if case["normalise"]:
            p = torch.zeros_like(logits)
            p[r, s["expert"][r, j].long()] = d("weight")[r, j]
        else:
            p = torch.softmax(logits, 1).nan_to_num(nan=0.0)
        inner = (dw * d("weight")).sum(1, keepdim=True)
        return p * (full - inner)
    if op == "dispatch_fwd":
        experts, k = case["experts"], case["k"]
        flat = s["expert"].view(-1)
        order = torch.cat([(flat == e).nonzero().view(-1) for e in [*range(experts), -1]])
        counts = torch.bincount(flat[flat >= 0], minlength=experts)
        offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0)).int()
        used = int(offsets[-1])
        xs, place = s["xs"].clone(), torch.full_like(flat, -1)
        xs[:used] = s["x"][torch.div(order[:used], k, rounding_mode="floor")]
        place[order[:used]] = torch.arange(used, dtype=torch.int32, device=DEVICE)
        return {"order": order.int(), "place": place, "offsets": offsets, "xs": xs}
    if op in ("dispatch_bwd", "combine_fwd"):
        # from the sorted rows to theirs
        out = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device=DEVICE) if s["add"] is None else d("add")
        used, order = int(s["offsets"][-1]), s["order"].long()
        v = d("dxs" if op == "dispatch_bwd" else "ys")[:used]
        if op == "combine_fwd":
            v = v * d("weight").view(-1, 1)[order[:used]]
        return out.index_add_(0, torch.div(order[:used], case["k"], rounding_mode="floor"), v)
    if op == "combine_bwd":
        used, order = int(s["offsets"][-1]), s["order"].long()
        order = order[:used]
        dys, dweight = d("dys"), torch.zeros(case["rows"] * case["k"], dtype=torch.float64, device=DEVICE)
        up = d("dy")[torch.div(order, case["k"], rounding_mode="floor")]
        dys[:used] = d("weight").view(-1, 1)[order] * up
        dweight[order] = torch.linalg.vecdot(up, d("ys")[:used])
        return {"dys": dys, "dweight": dweight.view(case["rows"], case["k"])}
    z_of = lambda v: v.double()  # noqa: E731
    if op == "experts_fwd":
        z = torch.empty(case["rows"], case["out"], dtype=torch.float64, device=DEVICE)
        for e, (a, b) in enumerate(zip(s["ends"][:-1], s["ends"][1:])):
            z[a:b] = torch.addmm(d("b")[e], z_of(s["x"][a:b]), z_of(s["w"][e]).T.contiguous())
        y = {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * torch.special.ndtr(v),
             "silu": lambda v: v * torch.sigmoid(v), "tanh": torch.tanh, "sigmoid": torch.sigmoid}[case["act"]](z)
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    z = d("z")
    pdf = lambda v: torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi)  # noqa: E731
    slope = {"none": torch.ones_like, "relu": lambda v: torch.heaviside(v, torch.zeros_like(v)),
             "gelu": lambda v: torch.special.ndtr(v) + v * pdf(v),
             "silu": lambda v: torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v),
             "tanh": lambda v: torch.cosh(v) ** -2, "sigmoid": lambda v: torch.sigmoid(v) * torch.sigmoid(-v)}
    dz = d("dy") * slope[case["act"]](z)
    dx = torch.empty(case["rows"], case["in"], dtype=torch.float64, device=DEVICE)
    dw = torch.zeros(case["experts"], case["out"], case["in"], dtype=torch.float64, device=DEVICE)
    db = torch.zeros(case["experts"], case["out"], dtype=torch.float64, device=DEVICE)
    for e, (a, b) in enumerate(zip(s["ends"][:-1], s["ends"][1:])):
        dx[a:b] = dz[a:b] @ z_of(s["w"][e])
        dw[e] = dz[a:b].T.contiguous() @ z_of(s["x"][a:b])
        db[e] = dz[a:b].sum(dim=0)
    return {"dx": dx, "dw": dw, "db": db}
