"""Layer norm forward and backward (gs_layer_norm_*) against float64, at widths on both sides of every change of the
rows' spread over lanes, odd and unaligned ones, one row and many; the backward also against differences of the
forward. Bounds: the fp32 error of a row's sums (at most 64 additions deep) relative to the largest magnitude in the
row, then one rounding to the type."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from rows_reference import U32, assert_close, strided, sum_bound

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = 1e-5
DEPTH = 64   # additions that one value of a row's sum goes through, at most (32 in a lane, then lanes and waves)


def make(rows, dim, dtype, seed, shift=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, dim, generator=g, device="cuda") * 1.5 + shift).to(dtype)
    dy = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    w = torch.randn(dim, generator=g, device="cuda") * 0.3 + 1
    b = torch.randn(dim, generator=g, device="cuda") * 0.1
    add = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    return x, dy, w, b, add


def statistics(x):
    x = x.double()
    mean = x.mean(1)
    return mean, ((x - mean[:, None]).square().mean(1) + EPS).rsqrt()


def check_forward(x, w, b, y, mean, rstd, dtype):
    rm, rr = statistics(x)
    big = x.double().abs().amax(1) if x.numel() else rm
    assert_close("mean", mean, rm, DEPTH * U32 * big, torch.float32)
    # rstd: half the relative error of the variance, whose deviations carry the mean's error
    dev = DEPTH * U32 * big * rr
    assert_close("rstd", rstd, rr, rr * (DEPTH * U32 + 2 * dev), torch.float32)
    xh = (x.double() - rm[:, None]) * rr[:, None]
    wd = w.double() if w is not None else torch.ones_like(xh[0])
    bd = b.double() if b is not None else torch.zeros_like(xh[0])
    err = (dev[:, None] + xh.abs() * (DEPTH * U32 + 2 * dev[:, None])) * wd.abs() + 4 * U32 * (xh * wd).abs() \
        + 4 * U32 * bd.abs()
    assert_close("y", y, xh * wd + bd, err, dtype)


SHAPES = [(1, 1), (3, 2), (5, 3), (7, 8), (300, 9), (1, 17), (64, 31), (33, 64), (257, 100), (20, 255), (5, 256),
          (9, 257), (3, 511), (4, 512), (3, 513), (2, 1000), (6, 1024), (3, 1025), (2, 2048), (5, 2049), (3, 4096),
          (2, 4097), (2, 8192), (3, 8193), (2, 16384), (2, 16391), (1, 40000), (70000, 4), (20011, 24)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_forward(rows, dim, dtype):
    x, _, w, b, _ = make(rows, dim, dtype, rows + dim)
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    gs.gs_layer_norm_fwd(x, w, b, EPS, y, mean, rstd)
    check_forward(x, w, b, y, mean, rstd, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (8, 0), (16, 5)])
def test_strides_and_no_parameters(dtype, pad, offset):
    rows, dim = 37, 203
    x, dy, w, b, add = make(rows, dim, dtype, 7)
    xs, ys = strided(x, pad, offset), strided(torch.zeros_like(x), pad + 2, offset + 1)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    gs.gs_layer_norm_fwd(xs, None, None, EPS, ys, mean, rstd)
    check_forward(x, None, None, ys, mean, rstd, dtype)
    gs.gs_layer_norm_fwd(xs, w, None, EPS, ys)          # statistics not wanted
    check_forward(x, w, None, ys, mean, rstd, dtype)
    dx = strided(torch.zeros_like(x), pad + 1, offset)
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    backward(strided(dy, pad + 4, offset), xs, w, mean, rstd, dx, dw, db, strided(add, pad, offset))
    check_backward(x, dy, w, mean, rstd, add, dx, dw, db, dtype)


def backward(dy, x, w, mean, rstd, dx, dw, db, add=None):
    ws = torch.empty(max(gs.gs_layer_norm_workspace_size(x), 1), dtype=torch.uint8, device="cuda")
    gs.gs_layer_norm_bwd(dy, x, w, mean, rstd, dx, dw, db, ws, add=add)


def check_backward(x, dy, w, mean, rstd, add, dx, dw, db, dtype):
    rows, dim = x.shape
    mu, rs = mean.double()[:, None], rstd.double()[:, None]
    xh = (x.double() - mu) * rs
    wd = w.double() if w is not None else torch.ones(dim, dtype=torch.float64, device="cuda")
    g = dy.double() * wd
    ref = rs * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    exh = 4 * U32 * (xh.abs() + rs * mu.abs())                       # xh's own error
    err = rs * DEPTH * U32 * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)) \
        + rs * (exh * (g * xh).abs().mean(1, keepdim=True) + xh.abs() * (g.abs() * exh).mean(1, keepdim=True))
    if add is not None:
        ref = ref + add.double()
        err = err + 2 * U32 * (add.double().abs() + ref.abs())
    assert_close("dx", dx, ref, err, dtype)
    k = sum_bound(rows)
    if dw is not None:
        assert_close("dw", dw, (dy.double() * xh).sum(0),
                     k * (dy.double() * xh).abs().sum(0) + (dy.double().abs() * exh).sum(0), torch.float32)
    if db is not None:
        assert_close("db", db, dy.double().sum(0), k * dy.double().abs().sum(0), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_backward(rows, dim, dtype):
    x, dy, w, _, add = make(rows, dim, dtype, 2 * rows + dim)
    mean, rstd = (v.float() for v in statistics(x))
    for use_add in (False, True):
        dx = torch.full_like(x, float("nan"))
        dw, db = (torch.full((dim,), float("nan"), device="cuda") for _ in range(2))
        backward(dy, x, w, mean, rstd, dx, dw, db, add if use_add else None)
        check_backward(x, dy, w, mean, rstd, add if use_add else None, dx, dw, db, dtype)
    again = [torch.empty_like(v) for v in (dx, dw, db)]
    backward(dy, x, w, mean, rstd, *again, add)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))   # the same bits


def test_backward_of_some_outputs():
    x, dy, w, _, _ = make(50, 40, torch.float32, 3)
    mean, rstd = (v.float() for v in statistics(x))
    dx, dw, db = torch.empty_like(x), torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    backward(dy, x, w, mean, rstd, dx, dw, None)
    check_backward(x, dy, w, mean, rstd, None, dx, dw, None, torch.float32)
    backward(dy, x, w, mean, rstd, dx, None, db)
    check_backward(x, dy, w, mean, rstd, None, dx, None, db, torch.float32)
    dx.fill_(float("nan"))
    backward(dy, x, None, mean, rstd, dx, None, None)
    check_backward(x, dy, None, mean, rstd, None, dx, None, None, torch.float32)


@pytest.mark.parametrize("dim", [12, 300, 9000])
def test_no_rows(dim):
    x = torch.empty(0, dim, device="cuda")
    dw, db = (torch.full((dim,), 7.0, device="cuda") for _ in range(2))
    none = torch.empty(0, device="cuda")
    gs.gs_layer_norm_fwd(x, None, None, EPS, torch.empty_like(x), none, none)
    backward(torch.empty_like(x), x, None, none, none, torch.empty_like(x), dw, db)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_are_hard(dtype):
    # a constant row (variance 0), one far from zero, and rows with an infinity or an undefined value, which stay
    # alone: each row is its own
    rows, dim = 6, 130
    x, _, w, b, _ = make(rows, dim, dtype, 11)
    x[0] = 3.0
    x[1] = x[1] * 0.25 + 1000
    x[2, 5] = float("inf")
    x[3, 129] = float("nan")
    y = torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    gs.gs_layer_norm_fwd(x, w, b, EPS, y, mean, rstd)
    assert torch.isnan(y[3]).all() and torch.isnan(y[2]).any()
    keep = [0, 1, 4, 5]
    check_forward(x[keep], w, b, y[keep], mean[keep], rstd[keep], dtype)


def test_backward_against_differences():
    rows, dim = 9, 37
    x, dy, w, b, _ = make(rows, dim, torch.float32, 21)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    y = torch.empty_like(x)
    gs.gs_layer_norm_fwd(x, w, b, EPS, y, mean, rstd)
    backward(dy, x, w, mean, rstd, dx, dw, db)

    def loss(x_, w_, b_):
        gs.gs_layer_norm_fwd(x_, w_, b_, EPS, y)
        return float((y.double() * dy.double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(5)
    h = 2.0 ** -7
    for k, (t, grad) in enumerate(((x, dx), (w, dw), (b, db))):
        d = torch.randn(t.shape, generator=gen, device="cuda")
        args = [x, w, b]
        plus, minus = list(args), list(args)
        plus[k], minus[k] = t + h * d, t - h * d
        slope = (loss(*plus) - loss(*minus)) / (2 * h)
        want = float((grad.double() * d.double()).sum())
        # the third derivative's h^2 / 6, and the fp32 rounding of some 300 values of y over 2 h
        assert abs(slope - want) <= 2e-3 * float((grad.double() * d.double()).abs().sum()) + 300 ** 0.5 * U32 * 8 / h, \
            (k, slope, want)


def test_another_stream():
    x, _, w, b, _ = make(2000, 777, torch.float16, 13)
    side = torch.cuda.Stream()
    y = torch.zeros_like(x)
    mean, rstd = torch.empty(2000, device="cuda"), torch.empty(2000, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    gs.gs_layer_norm_fwd(x, w, b, EPS, y, mean, rstd, stream=side)
    side.synchronize()
    check_forward(x, w, b, y, mean, rstd, torch.float16)
