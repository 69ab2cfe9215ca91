"""The linear backward's fp32 weight gradient where dz is kept in planes of a 16-bit type (an activation with a smooth
slope): operands far from size 1, on both sides of the narrow form. Bounds as in test_gpu_linear.py; with few rows the
sum's own share of them lies well below the 2^-12 that a lost plane would leave."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from rows_reference import assert_close, slope, sum_bound
from test_gpu_linear import ACT_ERROR, check_backward, make, space

pytestmark = pytest.mark.gpu

HALF_TYPES = [torch.float16, torch.bfloat16]
# (rows, inputs, outputs): the narrow form's widths with whole and part tiles of rows, then tiles
LAYERS = [(64, 128, 128), (65, 64, 64), (40, 17, 40), (33, 127, 31), (300, 32, 128), (64, 129, 128), (64, 256, 200),
          (300, 72, 400), (48, 1032, 520)]


def backward(d, name):
    n_out, n_in = d["w"].shape
    dx = torch.full_like(d["x"], float("nan"))
    dw = torch.full((n_out, n_in), float("nan"), device="cuda")
    db = torch.full((n_out,), float("nan"), device="cuda")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], name), act=name)
    return dx, dw, db


@pytest.mark.parametrize("dtype", HALF_TYPES)
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4, 100.0])
@pytest.mark.parametrize("rows,n_in,n_out", LAYERS)
def test_weight_gradient_of_inputs_of_any_size(rows, n_in, n_out, size, dtype):
    d = make(rows, n_in, n_out, dtype, rows + n_in)
    d["x"] = (d["x"].float() * size).to(dtype)
    for name in ("gelu", "silu"):
        check_backward(d, name, *backward(d, name))


@pytest.mark.parametrize("dtype", HALF_TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(300, 48, 40), (500, 256, 200), (333, 203, 150), (20, 300, 72)])
def test_outputs_left_out_with_workspaces_for_either_type(rows, n_in, n_out, dtype):
    d = make(rows, n_in, n_out, dtype, rows)
    for dw_type in (torch.float32, dtype):
        ws = space(d["x"], d["w"], "gelu", dw_type)
        dx, db = torch.empty_like(d["x"]), torch.empty(n_out, device="cuda")
        dw = torch.empty(n_out, n_in, dtype=dw_type, device="cuda")
        for keep in range(8):
            outs = [t if keep >> k & 1 else None for k, t in enumerate((dx, dw, db))]
            for t in (dx, dw, db):
                t.fill_(float("nan"))
            gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], *outs, ws, act="gelu")
            check_backward(d, "gelu", *outs)


@pytest.mark.parametrize("dtype", HALF_TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", LAYERS + [(70, 1032, 2048), (2100, 1000, 960), (4100, 264, 1040)])
def test_infinite_and_undefined_inputs(rows, n_in, n_out, dtype):
    # an x that is not finite meets its column of dw alone, and that with the sign of its products with dz: what it makes
    # of the lower planes' zeros and signs must not show
    d = make(rows, n_in, n_out, dtype, 3 * rows + n_in)
    d["dy"] = (d["dy"].sign() * (0.02 + d["dy"].abs().float())).to(dtype)
    d["z"] = (d["z"].abs().float() + 0.5).to(dtype)   # slopes between 0.7 and 1.2
    d["dy"][5, 3] = 0.0
    up, down, none = 7, n_in - 1, n_in // 2
    d["x"][5, up] = float("inf")
    d["x"][rows - 1, down] = float("-inf")
    d["x"][11, none] = float("nan")
    for name in ("gelu", "silu"):
        dx, dw, db = backward(d, name)
        sign = d["dy"].float().sign()
        want = sign[5] * float("inf")   # (0 times infinity is undefined)
        assert torch.equal(dw[:, up].isnan(), want.isnan()) and bool(want.isnan()[3])
        assert torch.equal(dw[:, up].nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
        assert torch.equal(dw[:, down], -sign[rows - 1] * float("inf"))
        assert torch.isnan(dw[:, none]).all()
        keep = [c for c in range(n_in) if c not in (up, down, none)]
        check_backward({**d, "x": d["x"][:, keep], "w": d["w"][:, keep]}, name, dx[:, keep], dw[:, keep], db)


@pytest.mark.parametrize("dtype", HALF_TYPES)
@pytest.mark.parametrize("size", [1e-4, 1e-6, 1e-7])
@pytest.mark.parametrize("rows,n_in,n_out", LAYERS)
def test_weight_gradient_of_small_gradients(rows, n_in, n_out, size, dtype):
    # dz is kept to 22 bits, in binary16 to within 2^-36 where it is small (2^-14 and less)
    d = make(rows, n_in, n_out, dtype, 5 * rows + n_in)
    d["dy"] = (d["dy"].float() * (10 * size)).to(dtype)
    x, dy, z = (d[k].double() for k in ("x", "dy", "z"))
    dz = dy * slope("gelu", z)
    lost = 2.0 ** -22 * dz.abs() + (2.0 ** -36 if dtype == torch.float16 else 0.0) + dy.abs() * ACT_ERROR * (1 + z.abs())
    dw = backward(d, "gelu")[1]
    assert_close("dw", dw, dz.t() @ x, sum_bound(rows) * (dz.abs().t() @ x.abs()) + lost.t() @ x.abs(), torch.float32)
