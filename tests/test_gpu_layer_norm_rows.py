"""Layer norm at row values and row counts beyond those of test_gpu_layer_norm.py, against float64 with its bounds."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from rows_reference import U32, assert_close, sum_bound
from test_gpu_layer_norm import DEPTH, EPS, backward, check_backward, check_forward, make, statistics

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [1, 2, 5, 17, 203, 333, 1001, 5003, 16391])
def test_backward_of_constant_rows_far_from_zero(dim, dtype):
    # x is its row's mean, so xh is 0; the mean times rstd lies beyond fp32, which no place beyond the row may meet
    rows = 9
    x, dy, w, _, _ = make(rows, dim, dtype, dim)
    x[:] = 2.0 ** 122
    mean = torch.full((rows,), 2.0 ** 122, device="cuda")
    rstd = torch.full((rows,), EPS ** -0.5, device="cuda")
    assert torch.isinf(mean * rstd).all()
    dx, dw, db = torch.full_like(x, float("nan")), torch.full((dim,), 1.0, device="cuda"), torch.empty(dim, device="cuda")
    backward(dy, x, w, mean, rstd, dx, dw, db)
    g = dy.double() * w.double()
    rs = rstd.double()[:, None]
    err = rs * DEPTH * U32 * (g.abs() + g.abs().mean(1, keepdim=True))
    assert_close("dx", dx, rs * (g - g.mean(1, keepdim=True)), err, dtype)
    assert not dw.any()
    assert_close("db", db, dy.double().sum(0), sum_bound(rows) * dy.double().abs().sum(0), torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [1, 2])
def test_forward_and_backward_of_constant_rows_far_from_zero(dim, dtype):
    # the same with the forward's own statistics
    x, dy, w, b, _ = make(5, dim, dtype, 3)
    x[:] = 2.0 ** 122
    y, mean, rstd = torch.empty_like(x), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    gs.gs_layer_norm_fwd(x, w, b, EPS, y, mean, rstd)
    assert torch.equal(y, b.to(dtype).expand(5, dim))
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    backward(dy, x, w, mean, rstd, dx, dw, db)
    assert torch.isfinite(dx).all() and not dw.any()


# more rows than the grid has groups of lanes, at every spread of a row over lanes, waves and workgroups: a group takes
# several rows in turn, with the next one's values on their way
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,dim", [(300_000, 3), (150_000, 30), (20_000, 200), (9_001, 333), (9_000, 700), (6_000, 1000),
                                      (5_001, 1500), (4_100, 2048), (4_100, 3000), (2_001, 4096), (1_300, 6001),
                                      (1_200, 8192), (1_100, 16384), (1_050, 20_000)])
def test_many_rows(rows, dim, dtype):
    x, dy, w, b, add = make(rows, dim, dtype, rows)
    bad = [1, rows // 2, rows - 2]   # rows of their own: an infinity or an undefined value reaches no other
    x[bad[0], 0], x[bad[1], dim - 1], x[bad[2], dim // 2] = float("inf"), float("nan"), float("-inf")
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    gs.gs_layer_norm_fwd(x, w, b, EPS, y, mean, rstd)
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[bad] = False
    check_forward(x[good], w, b, y[good], mean[good], rstd[good], dtype)
    assert torch.isnan(y[bad]).any(1).all()
    x[bad] = 1.0
    rm, rr = (v.float() for v in statistics(x))
    dx = torch.full_like(x, float("nan"))
    dw, db = (torch.full((dim,), float("nan"), device="cuda") for _ in range(2))
    backward(dy, x, w, rm, rr, dx, dw, db, add)
    check_backward(x, dy, w, rm, rr, add, dx, dw, db, dtype)
