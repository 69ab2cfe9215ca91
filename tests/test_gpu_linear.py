"""The linear operators (gs_linear_fwd, gs_linear_bwd) against float64: every type and activation, sizes on both sides
of every change of kernel (few rows, tiles, split sums), odd sizes, strides and alignments, and no rows. Bounds: the
fp32 error of a sum of `length` products relative to the sum of their magnitudes (sum_bound), the activation's own
5e-7, and one rounding to the type; a dz that is rounded to 16 bits adds that rounding to each product of dx (and of
dw in a 16-bit type)."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from rows_reference import TINY, U32, UNIT, act, assert_close, slope, strided, sum_bound

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = ["none", "relu", "gelu", "silu", "tanh", "sigmoid"]
ACT_ERROR = 5e-7   # of an activation or its slope, relative to 1 + |z|


def make(rows, n_in, n_out, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return dict(x=rand(rows, n_in).to(dtype), w=(rand(n_out, n_in) * n_in ** -0.5).to(dtype), bias=rand(n_out) * 0.3,
                r=rand(rows, n_out).to(dtype), dy=(rand(rows, n_out) * 0.1).to(dtype),
                z=(rand(rows, n_out) * 1.5).to(dtype))


def space(x, w, name, dw_type=torch.float32):
    return torch.empty(max(gs.gs_linear_workspace_size(x, w, name, dw_type), 1), dtype=torch.uint8, device="cuda")


def check_forward(d, name, y, z=None, bias=True, residual=True):
    dtype = d["x"].dtype
    x, w = d["x"].double(), d["w"].double()
    rz = x @ w.t()
    err = sum_bound(x.shape[1]) * (x.abs() @ w.abs().t())
    if bias:
        rz = rz + d["bias"].double()
        err = err + 2 * U32 * (d["bias"].double().abs() + rz.abs())
    if z is not None:
        assert_close("z", z, rz, err, dtype)
    ry = act(name, rz)
    err = 1.13 * err + (ACT_ERROR * (1 + rz.abs()) if name != "none" else 0)
    if residual:
        ry = ry + d["r"].double()
        err = err + 2 * U32 * ry.abs()
    assert_close("y", y, ry, err, dtype)


def check_backward(d, name, dx, dw, db):
    dtype = d["x"].dtype
    x, w, dy, z = (d[k].double() for k in ("x", "w", "dy", "z"))
    dz = dy * slope(name, z)
    smooth = name not in ("none", "relu")
    ez = dy.abs() * ACT_ERROR * (1 + z.abs()) if smooth else torch.zeros_like(dz)
    rounded = UNIT[dtype] * dz.abs() + TINY[dtype] if smooth and dtype != torch.float32 else torch.zeros_like(dz)
    if dx is not None:
        err = sum_bound(w.shape[0]) * (dz.abs() @ w.abs()) + (ez + rounded) @ w.abs()
        assert_close("dx", dx, dz @ w, err, dtype)
    if dw is not None:
        # in fp32 the planes keep 22 bits or more of dz
        kept = rounded if dw.dtype != torch.float32 else 2.0 ** -21 * dz.abs() * (rounded > 0) + 2.0 ** -35
        err = sum_bound(x.shape[0]) * (dz.abs().t() @ x.abs()) + (ez + kept).t() @ x.abs()
        assert_close("dw", dw, dz.t() @ x, err, dw.dtype)
    if db is not None:
        assert_close("db", db, dz.sum(0), sum_bound(x.shape[0]) * dz.abs().sum(0) + ez.sum(0), torch.float32)


SHAPES = [(1, 1, 1), (1, 64, 3), (2, 17, 32), (5, 129, 16), (16, 256, 48), (17, 100, 100), (64, 31, 129), (64, 512, 64),
          (65, 64, 64), (65, 1000, 70), (100, 2048, 64), (129, 3, 5), (200, 17, 3), (1000, 40, 31), (1000, 64, 33),
          (4099, 96, 96), (5000, 16, 24), (777, 333, 222), (256, 1536, 260), (20000, 128, 256), (2100, 256, 2048)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_forward(rows, n_in, n_out, dtype):
    d = make(rows, n_in, n_out, dtype, rows + n_in + n_out)
    name = ACTS[(rows + n_out) % len(ACTS)]
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    ws = space(d["x"], d["w"], name, None)
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, ws, act=name, residual=d["r"], z=z)
    check_forward(d, name, y, z)
    gs.gs_linear_fwd(d["x"], d["w"], None, y, ws)
    check_forward(d, "none", y, bias=False, residual=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_backward(rows, n_in, n_out, dtype):
    d = make(rows, n_in, n_out, dtype, rows + n_in + n_out)
    for k, name in enumerate((ACTS[(rows + n_out) % len(ACTS)], "none", "gelu")):
        dx = torch.full_like(d["x"], float("nan"))
        dw = torch.full(d["w"].shape, float("nan"), dtype=dtype if k == 2 else torch.float32, device="cuda")
        db = torch.full((n_out,), float("nan"), device="cuda")
        ws = space(d["x"], d["w"], name, dw.dtype)
        z = None if name == "none" else d["z"]
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], z, dx, dw, db, ws, act=name)
        check_backward(d, name, dx, dw, db)
        again = [torch.empty_like(v) for v in (dx, dw, db)]
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], z, *again, ws, act=name)
        assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activations(name, dtype):
    # pre-activations over the whole line, through a layer that passes them on (w = 1 in one column)
    z = torch.cat([torch.linspace(-30, 30, 4001), torch.linspace(-1, 1, 999), torch.tensor([0.0, -0.0, 100.0, -100.0])])
    rows = z.numel()
    d = make(rows, 8, 8, dtype, 5)
    d["x"].zero_()
    d["x"][:, 0] = z.to(dtype)
    d["w"].zero_()
    d["w"][:, 0] = 1.0
    y = torch.empty_like(d["r"])
    gs.gs_linear_fwd(d["x"], d["w"], None, y, space(d["x"], d["w"], name, None), act=name)
    check_forward(d, name, y, bias=False, residual=False)
    d["z"] = d["x"][:, :1].expand(-1, 8).contiguous()
    dx, dw, db = torch.empty_like(d["x"]), torch.empty(8, 8, device="cuda"), torch.empty(8, device="cuda")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], name), act=name)
    check_backward(d, name, dx, dw, db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(3, 40, 24), (150, 104, 72), (3000, 64, 136)])
@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 0), (8, 1), (4, 4)])
def test_strides(rows, n_in, n_out, dtype, pad, offset):
    # rows further apart than their columns and operands off their vectors' alignment; what lies between is NaN
    d = make(rows, n_in, n_out, dtype, 3)
    s = {k: strided(v, pad, offset) if v.dim() == 2 else v for k, v in d.items()}
    y, z = (strided(torch.zeros_like(d["r"]), pad + 1, offset) for _ in range(2))
    gs.gs_linear_fwd(s["x"], s["w"], d["bias"], y, space(d["x"], d["w"], "silu"), act="silu", residual=s["r"], z=z)
    check_forward(d, "silu", y, z)
    for name in ("none", "tanh"):
        dx = strided(torch.zeros_like(d["x"]), pad, offset)
        dw = strided(torch.zeros(n_out, n_in, device="cuda"), pad, offset)
        db = torch.empty(n_out, device="cuda")
        gs.gs_linear_bwd(s["dy"], s["x"], s["w"], s["z"], dx, dw, db, space(d["x"], d["w"], name), act=name)
        check_backward(d, name, dx, dw, db)


def test_outputs_left_out():
    d = make(300, 48, 40, torch.bfloat16, 9)
    ws = space(d["x"], d["w"], "gelu")
    dx, dw, db = torch.empty_like(d["x"]), torch.empty(40, 48, device="cuda"), torch.empty(40, device="cuda")
    for keep in range(8):
        outs = [t if keep >> k & 1 else None for k, t in enumerate((dx, dw, db))]
        for t in (dx, dw, db):
            t.fill_(float("nan"))
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], *outs, ws, act="gelu")
        check_backward(d, "gelu", *outs)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    d = make(0, 24, 40, dtype, 1)
    dw, db = torch.full((40, 24), 3.0, device="cuda"), torch.full((40,), 3.0, device="cuda")
    ws = space(d["x"], d["w"], "gelu")
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], torch.empty_like(d["r"]), ws, act="gelu")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], torch.empty_like(d["x"]), dw, db, ws, act="gelu")
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [4, 300])
def test_undefined_values_stay_in_their_row(dtype, rows):
    # an infinity and an undefined value in x reach their rows of z alone, whatever the tiles read beside them
    d = make(rows, 72, 40, dtype, 2)
    d["x"][1, 70] = float("inf")
    d["x"][2, 0] = float("nan")
    y = torch.empty_like(d["r"])
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, space(d["x"], d["w"], "none"), residual=d["r"])
    assert not torch.isfinite(y[1]).any() and torch.isnan(y[2]).all()
    keep = [i for i in range(rows) if i not in (1, 2)]
    check_forward({**d, "x": d["x"][keep], "r": d["r"][keep]}, "none", y[keep])


@pytest.mark.parametrize("dtype", TYPES)
def test_infinite_gradient(dtype):
    # an infinite dy makes its row of dx and its column's dw and db infinite or undefined, and nothing else
    d = make(200, 24, 16, dtype, 6)
    d["dy"][7, 3] = float("inf")
    d["z"][7, 3] = 1.0
    dx, dw, db = torch.empty_like(d["x"]), torch.empty(16, 24, device="cuda"), torch.empty(16, device="cuda")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], "silu"), act="silu")
    assert torch.isinf(db[3]) and torch.isinf(dw[3]).all() and not torch.isfinite(dx[7]).any()
    rest = [c for c in range(16) if c != 3]
    keep = [r for r in range(200) if r != 7]
    assert torch.isfinite(dw[rest]).all() and torch.isfinite(dx[keep]).all() and torch.isfinite(db[rest]).all()


@pytest.mark.parametrize("name", ["gelu", "silu", "tanh", "sigmoid"])
def test_backward_against_differences(name):
    d = make(70, 30, 20, torch.float32, 4)
    y, z = torch.empty_like(d["r"]), torch.empty_like(d["r"])
    ws = space(d["x"], d["w"], name)
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, ws, act=name, z=z)
    dx, dw, db = torch.empty_like(d["x"]), torch.empty_like(d["w"]), torch.empty_like(d["bias"])
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], z, dx, dw, db, ws, act=name)

    def loss(x, w, b):
        gs.gs_linear_fwd(x, w, b, y, ws, act=name)
        return float((y.double() * d["dy"].double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(8)
    h = 2.0 ** -7
    for k, grad in enumerate((dx, dw, db)):
        args = [d["x"], d["w"], d["bias"]]
        v = torch.randn(args[k].shape, generator=gen, device="cuda")
        plus, minus = list(args), list(args)
        plus[k], minus[k] = args[k] + h * v, args[k] - h * v
        got = (loss(*plus) - loss(*minus)) / (2 * h)
        want = float((grad.double() * v.double()).sum())
        # the third derivative's h^2 / 6, and the fp32 rounding of 1,400 values of y times dy over 2 h
        limit = 2e-3 * float((grad.double() * v.double()).abs().sum()) + 1400 ** 0.5 * 0.1 * 8 * U32 / h
        assert abs(got - want) <= limit, (k, got, want)


def test_another_stream():
    d = make(3000, 200, 150, torch.float16, 13)
    side = torch.cuda.Stream()
    y, ws = torch.zeros_like(d["r"]), space(d["x"], d["w"], "relu")
    side.wait_stream(torch.cuda.current_stream())
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, ws, act="relu", residual=d["r"], stream=side)
    side.synchronize()
    check_forward(d, "relu", y)


def test_binding_refuses():
    d = make(40, 24, 16, torch.float16, 1)
    y, ws = torch.empty_like(d["r"]), space(d["x"], d["w"], "relu")

    def refused(*args, **kw):
        with pytest.raises((ValueError, gs.GsError)):
            gs.gs_linear_fwd(*args, **kw)

    refused(d["x"], d["w"][:, :23], None, y, ws)              # another width
    refused(d["x"], d["w"].float(), None, y, ws)              # another type
    refused(d["x"], d["w"], d["bias"].half(), y, ws)          # the bias is fp32
    refused(d["x"], d["w"], None, y.t().contiguous().t(), ws)   # columns apart
    refused(d["x"], d["w"], None, y[:39], ws)                 # fewer rows
    refused(d["x"][:1].expand(40, 24), d["w"], None, y, ws)   # rows on top of each other
    refused(d["x"], d["w"], None, y, ws, residual=y[:, :15])
    wide = torch.empty(100, 24, dtype=torch.float16, device="cuda")
    refused(wide, d["w"][:, :24].t().contiguous().t(), None, torch.empty(100, 16, dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):   # dw of a third type
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], None, torch.empty(16, 24, dtype=torch.bfloat16, device="cuda"),
                         None, ws, act="relu")
    with pytest.raises(gs.GsError) as e:   # a workspace that is too small
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], None, torch.empty(16, 24, device="cuda"), None, ws[:256],
                         act="relu")
    assert e.value.status == gs.GS_ERR_CAPACITY


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,n_in,n_out", [(4166, 520, 4104), (4100, 4104, 1032), (70, 4104, 4360), (300, 4096, 4608)])
def test_largest_tiles(rows, n_in, n_out, dtype):
    # products of enough tiles for the 256 x 256 ones: ends of rows, columns and sums inside a tile, an odd count of
    # halves, sums shorter than the tiles on their way
    d = make(rows, n_in, n_out, dtype, 17)
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, space(d["x"], d["w"], "silu", None), act="silu", residual=d["r"], z=z)
    check_forward(d, "silu", y, z)
    for name, dw_type in (("tanh", dtype), ("gelu", torch.float32), ("none", torch.float32)):
        dx = torch.full_like(d["x"], float("nan"))
        dw = torch.full(d["w"].shape, float("nan"), dtype=dw_type, device="cuda")
        db = torch.full((n_out,), float("nan"), device="cuda")
        ws = space(d["x"], d["w"], name, dw_type)
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, ws, act=name)
        check_backward(d, name, dx, dw, db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [32, 33, 48, 64, 65])
@pytest.mark.parametrize("n_in,n_out", [(64, 48), (33, 17), (520, 264), (1031, 300), (4096, 200)])
def test_few_rows_and_more(rows, n_in, n_out, dtype):
    # on both sides of the form for few rows, with W's rows aligned and not
    d = make(rows, n_in, n_out, dtype, rows + n_in)
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, space(d["x"], d["w"], "tanh", None), act="tanh", residual=d["r"], z=z)
    check_forward(d, "tanh", y, z)
    dx = torch.full_like(d["x"], float("nan"))
    dw = torch.full(d["w"].shape, float("nan"), device="cuda")
    db = torch.full((n_out,), float("nan"), device="cuda")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], "silu"), act="silu")
    check_backward(d, "silu", dx, dw, db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 16, 31])
@pytest.mark.parametrize("n_in", [7, 31, 256, 1027, 2304, 4099])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (2, 1), (8, 1)])
def test_few_rows_at_any_address(rows, n_in, pad, offset, dtype):
    # rows of x and W at even and odd addresses, sums that end anywhere in a vector or a step; what lies between is NaN
    d = make(rows, n_in, 37, dtype, n_in)
    x, w = strided(d["x"], pad, offset), strided(d["w"], pad, offset)
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    gs.gs_linear_fwd(x, w, d["bias"], y, space(x, w, "sigmoid", None), act="sigmoid", residual=d["r"], z=z)
    check_forward(d, "sigmoid", y, z)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(1000, 2064, 968), (70, 1032, 2048), (2100, 1000, 960), (1025, 136, 520)])
def test_sums_shared_within_a_workgroup(rows, n_in, n_out, dtype):
    # products of about one tile for each compute unit, with long sums: parts of unequal length, ends inside a tile
    d = make(rows, n_in, n_out, dtype, 23)
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, space(d["x"], d["w"], "gelu", None), act="gelu", residual=d["r"], z=z)
    check_forward(d, "gelu", y, z)
    for name, dw_type in (("relu", dtype), ("silu", torch.float32)):
        dx = torch.full_like(d["x"], float("nan"))
        dw = torch.full(d["w"].shape, float("nan"), dtype=dw_type, device="cuda")
        db = torch.full((n_out,), float("nan"), device="cuda")
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], name, dw_type), act=name)
        check_backward(d, name, dx, dw, db)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 63, 64, 65, 40_000])
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (65, 64), (64, 65), (128, 128), (129, 128), (128, 129), (17, 3), (3, 128)])
def test_backward_on_both_sides_of_the_narrow_form(rows, n_in, n_out, dtype):
    # one pass up to 128 inputs and outputs, separate products beyond; whole and part tiles of rows, fewer tiles than
    # workgroups and more
    d = make(rows, n_in, n_out, dtype, rows + n_in)
    for name, dw_type in (("relu", torch.float32), ("silu", torch.float32), ("sigmoid", dtype)):
        dx = torch.full_like(d["x"], float("nan"))
        dw = torch.full(d["w"].shape, float("nan"), dtype=dw_type, device="cuda")
        db = torch.full((n_out,), float("nan"), device="cuda")
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], name, dw_type), act=name)
        check_backward(d, name, dx, dw, db)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [65, 79, 80, 20_011])
@pytest.mark.parametrize("n_in,n_out", [(32, 32), (33, 31), (64, 128), (128, 64), (128, 128), (127, 125), (128, 129), (8, 3)])
def test_forward_on_both_sides_of_the_narrow_form(rows, n_in, n_out, dtype):
    d = make(rows, n_in, n_out, dtype, rows + n_in)
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    ws = space(d["x"], d["w"], "gelu", None)
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, ws, act="gelu", residual=d["r"], z=z)
    check_forward(d, "gelu", y, z)
    wide, s = strided(torch.zeros_like(d["r"]), 3), {k: strided(v, 5, 1) if v.dim() == 2 else v for k, v in d.items()}
    gs.gs_linear_fwd(s["x"], s["w"], d["bias"], wide, ws, act="tanh", residual=s["r"])
    check_forward(d, "tanh", wide)


def test_forward_of_more_than_the_cache_holds():
    # the widening layer that goes through tiles where it keeps z (rows compared in a few places)
    d = make(1_100_003, 32, 64, torch.float16, 3)
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    ws = space(d["x"], d["w"], "relu", None)
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, ws, act="relu", residual=d["r"], z=z)
    plain = torch.full_like(y, float("nan"))
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], plain, ws, act="relu", residual=d["r"])
    for rows in (slice(0, 2000), slice(550_000, 552_000), slice(-2000, None)):
        part = {k: v[rows] if v.shape[0] == 1_100_003 else v for k, v in d.items()}
        check_forward(part, "relu", y[rows], z[rows])
        check_forward(part, "relu", plain[rows])
    assert torch.isfinite(y).all() and torch.isfinite(plain).all()
