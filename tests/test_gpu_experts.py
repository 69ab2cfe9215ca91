"""The experts' layers (gs_experts_fwd, gs_experts_bwd) against float64, expert by expert: every type and activation, sizes
on both sides of every change of kernel (few rows, narrow layers, tiles, units that share an expert's sum), experts without
rows, one expert with all of them, rows that are no expert's, odd sizes, strides and alignments. Bounds as for one linear
layer: the fp32 error of a sum of `length` products relative to the sum of their magnitudes, the activation's own 5e-7,
and one rounding to the type; a dz that is rounded to 16 bits adds that rounding to each product of dx (and of dw in a
16-bit type)."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from rows_reference import TINY, U32, UNIT, act, assert_close, slope, strided, sum_bound

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = ["none", "relu", "gelu", "silu", "tanh", "sigmoid"]
ACT_ERROR = 5e-7   # of an activation or its slope, relative to 1 + |z|
NAN = float("nan")


def magnitude(t):
    """What a product's operand counts as in the error of an fp32 sum on the matrix cores. These take a binary16 operand
    below 2^-14 at the exponent of 2^-14, without normalising it, so a sum that it joins has the grain of 2^-14's product:
    a gradient in two planes (high part h and, 2^-11 of it, low part l) for x = 2^-24 and x = 2^-20 alike is off by up to
    2^-44 where |h| is about 2^-4, 2^-26 of |h| 2^-14, which h x + l x alone, with x's own exponent, would not explain
    (2^-26 of |h| 2^-24). Without a second plane such a product alone is exact."""
    a = t.double().abs()
    return torch.where(t == 0, a, a.clamp(min=2.0 ** -14)) if t.dtype == torch.float16 else a


def lengths_of(rows, experts, spread):
    """Rows of each expert; with "spare" some rows are nobody's."""
    if spread == "one":
        return [rows if e == experts // 2 else 0 for e in range(experts)]
    share = [1.0 / (e + 1) if spread == "skewed" else 1.0 for e in range(experts)]
    have = rows - (rows // 7 if spread == "spare" else 0)
    out = [int(have * s / sum(share)) for s in share]
    if experts > 2:
        out[1] = 0
    out[0] += have - sum(out)
    return out


def make(rows, experts, n_in, n_out, dtype, seed, spread="skewed"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    n = lengths_of(rows, experts, spread)
    ends = [sum(n[:e]) for e in range(experts + 1)]
    d = dict(x=rand(rows, n_in).to(dtype), w=(rand(experts, n_out, n_in) * n_in ** -0.5).to(dtype),
             b=rand(experts, n_out) * 0.3, dy=(rand(rows, n_out) * 0.1).to(dtype), z=(rand(rows, n_out) * 1.5).to(dtype))
    for name in ("x", "dy", "z"):
        d[name][ends[-1]:] = NAN   # nobody's rows are not read
    for e in range(experts):
        if n[e] == 0:
            d["w"][e] = NAN        # nor are the weights of nobody's expert
    d.update(ends=ends, offsets=torch.tensor(ends, dtype=torch.int32, device="cuda"))
    return d


def space(d, name, dw_type=torch.float32):
    n = gs.gs_experts_workspace_size(d["x"], d["w"], name, dw_type)
    return torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device="cuda")


def forward(d, name, keep=True, bias=True, change=lambda t: t):
    rows, n_out, t = d["x"].shape[0], d["w"].shape[1], d["x"].dtype
    y, z = (change(torch.full((rows, n_out), NAN, dtype=t, device="cuda")) for _ in range(2))
    gs.gs_experts_fwd(change(d["x"]), d["offsets"], d["w"], d["b"] if bias else None, y, space(d, name, None), act=name,
                      z=z if keep else None)
    return y, z if keep else None


def check_forward(d, name, y, z, bias=True):
    dtype = d["x"].dtype
    for e, (a, b) in enumerate(zip(d["ends"][:-1], d["ends"][1:])):
        if a == b:
            continue
        x, w = d["x"][a:b].double(), d["w"][e].double()
        rz = x @ w.t()
        err = sum_bound(x.shape[1]) * (x.abs() @ w.abs().t())
        if bias:
            rz = rz + d["b"][e].double()
            err = err + 2 * U32 * (d["b"][e].double().abs() + rz.abs())
        if z is not None:
            assert_close("z of %d" % e, z[a:b], rz, err, dtype)
        err = 1.13 * err + (ACT_ERROR * (1 + rz.abs()) if name != "none" else 0)
        assert_close("y of %d" % e, y[a:b], act(name, rz), err, dtype)
    assert torch.isnan(y[d["ends"][-1]:]).all()
    if z is not None:
        assert torch.isnan(z[d["ends"][-1]:]).all()


def backward(d, name, dw_type, change=lambda t: t, want=("dx", "dw", "db")):
    experts, n_out, n_in = d["w"].shape
    t = d["x"].dtype
    dx = change(torch.full_like(d["x"], NAN)) if "dx" in want else None
    dw = torch.full((experts, n_out, n_in), NAN, dtype=dw_type, device="cuda") if "dw" in want else None
    db = torch.full((experts, n_out), NAN, device="cuda") if "db" in want else None
    gs.gs_experts_bwd(change(d["dy"]), change(d["x"]), d["offsets"], d["w"], None if name == "none" else change(d["z"]), dx,
                      dw, db, space(d, name, dw_type if dw is not None else t), act=name)
    return dx, dw, db


def check_backward(d, name, dx, dw, db):
    dtype = d["x"].dtype
    smooth = name not in ("none", "relu")
    for e, (a, b) in enumerate(zip(d["ends"][:-1], d["ends"][1:])):
        if a == b:
            assert dw is None or not dw[e].any()
            assert db is None or not db[e].any()
            continue
        x, w, dy, z = (t.double() for t in (d["x"][a:b], d["w"][e], d["dy"][a:b], d["z"][a:b]))
        dz = dy * slope(name, z)
        ez = dy.abs() * ACT_ERROR * (1 + z.abs()) if smooth else torch.zeros_like(dz)
        rounded = UNIT[dtype] * dz.abs() + TINY[dtype] if smooth and dtype != torch.float32 else torch.zeros_like(dz)
        if dx is not None:
            err = sum_bound(w.shape[0]) * (dz.abs() @ w.abs()) + (ez + rounded) @ w.abs()
            assert_close("dx of %d" % e, dx[a:b], dz @ w, err, dtype)
        if dw is not None:
            # in fp32 the planes keep 22 bits or more of dz (in binary16 to within 2^-36 where it is small)
            kept = 2.0 ** -22 * dz.abs() + 2.0 ** -36 if dw.dtype == torch.float32 and dtype != torch.float32 else rounded
            err = sum_bound(b - a) * (dz.abs().t() @ magnitude(d["x"][a:b])) + (ez + kept).t() @ x.abs()
            assert_close("dw of %d" % e, dw[e], dz.t() @ x, err, dw.dtype)
        if db is not None:
            assert_close("db of %d" % e, db[e], dz.sum(0), sum_bound(b - a) * dz.abs().sum(0) + ez.sum(0), torch.float32)
    if dx is not None:
        assert torch.isnan(dx[d["ends"][-1]:]).all()


# few rows, narrow layers, tiles of every size, odd widths
SHAPES = [(1, 1, 1, 1), (1, 4, 64, 32), (2, 3, 17, 5), (8, 16, 256, 130), (16, 5, 100, 40), (32, 3, 512, 200),
          (33, 4, 64, 64), (40, 70, 48, 24), (100, 3, 3, 3), (300, 5, 128, 128), (1000, 7, 32, 128), (2001, 3, 100, 60),
          (5000, 2, 17, 33), (33, 2, 256, 256), (100, 130, 200, 136), (500, 6, 136, 264), (1200, 4, 333, 215),
          (3000, 3, 520, 140), (700, 2, 1040, 96), (2500, 5, 129, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,n_in,n_out", SHAPES)
def test_forward(rows, experts, n_in, n_out, dtype):
    for k, spread in enumerate(("skewed", "spare", "one")):
        d = make(rows, experts, n_in, n_out, dtype, rows + n_in, spread)
        name = ACTS[(rows + k) % 6]
        y, z = forward(d, name, keep=k != 1, bias=k != 2)
        check_forward(d, name, y, z, bias=k != 2)


@pytest.mark.parametrize("same", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,n_in,n_out", SHAPES)
def test_backward(rows, experts, n_in, n_out, dtype, same):
    for k, spread in enumerate(("skewed", "spare", "one")):
        d = make(rows, experts, n_in, n_out, dtype, rows + n_out, spread)
        name = ACTS[(rows + k + n_in) % 6]
        check_backward(d, name, *backward(d, name, dtype if same else torch.float32))


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,n_in,n_out", [(20, 3, 96, 72), (900, 5, 96, 72), (900, 3, 264, 144)])
def test_activations(rows, experts, n_in, n_out, dtype, name):
    d = make(rows, experts, n_in, n_out, dtype, 5)
    check_forward(d, name, *forward(d, name))
    check_backward(d, name, *backward(d, name, torch.float32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,n_in,n_out", [(9000, 4, 512, 768), (40_000, 8, 256, 256), (70_001, 5, 64, 128),
                                                     (20_000, 1024, 64, 40), (3000, 1000, 160, 130)])
def test_larger(rows, experts, n_in, n_out, dtype):
    """The largest tiles, units that share an expert's sum, as many experts as there may be."""
    d = make(rows, experts, n_in, n_out, dtype, 6)
    check_forward(d, "gelu", *forward(d, "gelu"))
    check_backward(d, "relu", *backward(d, "relu", dtype))
    check_backward(d, "silu", *backward(d, "silu", torch.float32))


@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (3, 5), (8, 8)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(20, 70, 33), (500, 64, 64), (500, 77, 50), (600, 200, 150), (600, 333, 215)])
def test_strides(rows, n_in, n_out, dtype, pad, offset):
    d = make(rows, 4, n_in, n_out, dtype, 7, "spare")
    w, experts = d["w"], 4
    store = torch.full((experts * (n_out * (n_in + pad) + 3 * pad) + offset,), NAN, dtype=dtype, device="cuda")
    each = n_out * (n_in + pad) + 3 * pad
    view = torch.as_strided(store, (experts, n_out, n_in), (each, n_in + pad, 1), offset)
    view.copy_(w)
    d["w"] = view
    far = lambda t: strided(t, pad, offset)  # noqa: E731
    check_forward(d, "silu", *forward(d, "silu", change=far))
    dx, dw, db = backward(d, "silu", torch.float32, change=far)
    check_backward(d, "silu", dx, dw, db)
    # the gradient of the weights with strides of its own; what lies between is left alone
    gstore = torch.full_like(store, NAN, dtype=torch.float32)
    dw2 = torch.as_strided(gstore, (experts, n_out, n_in), (each, n_in + pad, 1), offset)
    gs.gs_experts_bwd(far(d["dy"]), far(d["x"]), d["offsets"], d["w"], far(d["z"]), None, dw2, None, space(d, "silu"),
                      act="silu")
    assert torch.equal(dw2, dw)
    assert int(torch.isfinite(gstore).sum()) == dw.numel()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(30, 64, 64), (700, 64, 96), (700, 256, 144)])
def test_parts_of_the_gradients(rows, n_in, n_out, dtype):
    """Each gradient alone is the one of the whole call, bit for bit; and so is a second call, whatever the workspace
    holds."""
    d = make(rows, 5, n_in, n_out, dtype, 8)
    whole = backward(d, "tanh", torch.float32)
    for k, name in enumerate(("dx", "dw", "db")):
        assert torch.equal(backward(d, "tanh", torch.float32, want=(name,))[k].nan_to_num(nan=7), whole[k].nan_to_num(nan=7))
    for a, b in zip(whole, backward(d, "tanh", torch.float32)):
        assert torch.equal(a.nan_to_num(nan=7), b.nan_to_num(nan=7))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(30, 64, 64), (900, 64, 96), (900, 264, 144)])
def test_some_of_the_experts(rows, n_in, n_out, dtype):
    """Offsets that begin behind the first row: the experts of a part of the order."""
    d = make(rows, 6, n_in, n_out, dtype, 13, "even")
    a, b = 2, 5
    first, last = d["ends"][a], d["ends"][b]
    y, z = forward(d, "silu")
    dx, dw, db = backward(d, "silu", torch.float32)
    part = dict(d, w=d["w"][a:b], b=d["b"][a:b], offsets=d["offsets"][a:b + 1], ends=d["ends"][a:b + 1])
    y2, z2 = forward(part, "silu")
    dx2, dw2, db2 = backward(part, "silu", torch.float32)
    for whole, some in ((y, y2), (z, z2), (dx, dx2)):
        assert torch.isnan(some[:first]).all() and torch.isnan(some[last:]).all()
        # (another number of tiles may be summed in another order)
        near = (whole[first:last].double() - some[first:last].double()).abs()
        assert (near <= 4 * UNIT[dtype] * whole[first:last].double().abs() + 64 * U32).all()
    check_forward(part, "silu", y2, z2)
    check_backward(part, "silu", dx2, dw2, db2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (264, 144)])
@pytest.mark.parametrize("rows", [0, 50])
def test_no_rows(rows, n_in, n_out, dtype):
    d = make(50, 3, n_in, n_out, dtype, 9)
    d = dict(d, x=d["x"][:rows], dy=d["dy"][:rows], z=d["z"][:rows], ends=[0, 0, 0, 0],
             offsets=torch.zeros(4, dtype=torch.int32, device="cuda"))
    check_forward(d, "gelu", *forward(d, "gelu"))
    check_backward(d, "gelu", *backward(d, "gelu", torch.float32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(24, 64, 40), (400, 64, 96), (600, 264, 144)])
def test_one_expert_is_a_linear_layer(rows, n_in, n_out, dtype):
    d = make(rows, 1, n_in, n_out, dtype, 10)
    y, z = forward(d, "gelu")
    check_forward(d, "gelu", y, z)
    ws = torch.empty(max(gs.gs_linear_workspace_size(d["x"], d["w"][0], "gelu"), 1), dtype=torch.uint8, device="cuda")
    yl, zl = torch.empty_like(y), torch.empty_like(z)
    gs.gs_linear_fwd(d["x"], d["w"][0], d["b"][0], yl, ws, act="gelu", z=zl)
    # two roundings of the same values to the type
    size = d["x"].double().abs() @ d["w"][0].double().abs().t() + 1
    assert ((z.double() - zl.double()).abs() <= 2 * (UNIT[dtype] * zl.double().abs() + sum_bound(n_in) * size + TINY[dtype])).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(24, 64, 40), (400, 64, 96), (600, 264, 144)])
def test_special_values_stay_with_their_rows_and_experts(rows, n_in, n_out, dtype):
    d = make(rows, 3, n_in, n_out, dtype, 11)
    clean_y, _ = forward(d, "none")
    clean = backward(d, "none", dtype)
    d["x"][2, 3] = float("inf")      # the first expert's
    d["dy"][4, 5] = NAN
    y, _ = forward(d, "none")
    others = [r for r in range(rows) if r != 2]
    assert torch.equal(y[others], clean_y[others]) and not torch.isfinite(y[2]).any()
    dx, dw, db = backward(d, "none", dtype)
    others = [r for r in range(rows) if r != 4]
    assert torch.equal(dx[others], clean[0][others]) and torch.isnan(dx[4]).all()
    assert torch.equal(dw[1:], clean[1][1:]) and torch.equal(db[1:], clean[2][1:])
    assert torch.isnan(db[0, 5]) and torch.isnan(dw[0, 5]).all()


def test_gradients_against_differences():
    rows, experts, n_in, n_out = 40, 3, 9, 7
    d = make(rows, experts, n_in, n_out, torch.float32, 12, "spare")
    used = d["ends"][-1]
    c = torch.randn(rows, n_out, device="cuda")

    def value(x, w, b):
        y, _ = forward(dict(d, x=x, w=w, b=b), "silu")
        return float((y[:used].double() * c[:used].double()).sum())

    w = d["w"].nan_to_num(nan=0.5)
    d["w"] = w
    _, z = forward(d, "silu")
    d.update(z=z, dy=c)
    dx, dw, db = backward(d, "silu", torch.float32)
    h = 2.0 ** -6
    size = float(c.abs().sum()) * 40   # of value's terms, generously; third derivatives of silu are below 1
    bound = size * (8 * U32 / h) + 30 * h * h
    for name, grad, places in (("x", dx, [(0, 0), (used - 1, 8)]), ("w", dw, [(0, 1, 2), (2, 6, 8)]),
                               ("b", db, [(0, 0), (2, 5)])):
        for at in places:
            moved = []
            for step in (h, -h):
                t = {k: d[k].clone() for k in ("x", "w", "b")}
                t[name][at] += step
                moved.append(value(**t))
            assert abs((moved[0] - moved[1]) / (2 * h) - float(grad[at])) <= bound, (name, at)


def test_long_rows_of_weights():
    """Experts whose weights begin more than 2^31 values behind the first's."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("9 GB of weights")
    experts, n_in, n_out = 65, 8192, 8192
    w = torch.zeros(experts, n_out, n_in, dtype=torch.bfloat16, device="cuda")
    w[-1, :, 0], w[0, :, 0] = 3.0, 1.0
    x = torch.ones(2, n_in, dtype=torch.bfloat16, device="cuda")
    offsets = torch.ones(experts + 1, dtype=torch.int32, device="cuda")
    offsets[0], offsets[-1] = 0, 2
    y = torch.full((2, n_out), NAN, dtype=torch.bfloat16, device="cuda")
    gs.gs_experts_fwd(x, offsets, w, None, y)
    assert (y[0] == 1).all() and (y[1] == 3).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(20, 96, 40), (700, 64, 96), (900, 264, 144), (900, 133, 61)])
def test_experts_with_the_same_weights(rows, n_in, n_out, dtype):
    """Weights a stride of 0 apart."""
    d = make(rows, 5, n_in, n_out, dtype, 21, "even")
    same = dict(d, w=d["w"][:1].expand(5, n_out, n_in))
    whole = dict(d, w=same["w"].contiguous())
    for a, b in zip((*forward(same, "silu"), *backward(same, "silu", torch.float32)),
                    (*forward(whole, "silu"), *backward(whole, "silu", torch.float32))):
        assert torch.equal(a.nan_to_num(nan=7), b.nan_to_num(nan=7))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,n_in,n_out", [(16, 16, 100, 530), (32, 20, 96, 520), (9, 70, 1000, 1100), (20, 40, 133, 400)])
def test_few_rows_and_many_columns(rows, experts, n_in, n_out, dtype):
    """More groups of columns than the compute units take at once."""
    d = make(rows, experts, n_in, n_out, dtype, 17)
    check_forward(d, "silu", *forward(d, "silu"))
