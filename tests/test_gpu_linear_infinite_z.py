"""The linear backward where a stored pre-activation is infinite: in binary16 a z beyond 65,504 is, although the layer's
own sum and its output are not. Its slope is the activation's limit."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from test_gpu_linear import TYPES, check_backward, make, space

pytestmark = pytest.mark.gpu

ACTS = ["relu", "gelu", "silu", "tanh", "sigmoid"]


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(20, 40, 24), (300, 128, 100), (300, 200, 150)])
def test_slope_at_infinity(rows, n_in, n_out, dtype, name):
    d = make(rows, n_in, n_out, dtype, 11)
    z = d["z"].clone()
    d["z"][3::7, 1::3], z[3::7, 1::3] = 300.0, float("inf")     # at 300 every slope is its limit in fp32
    d["z"][5::7, ::4], z[5::7, ::4] = -300.0, float("-inf")
    dx = torch.full_like(d["x"], float("nan"))
    dw, db = torch.full((n_out, n_in), float("nan"), device="cuda"), torch.full((n_out,), float("nan"), device="cuda")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], z, dx, dw, db, space(d["x"], d["w"], name), act=name)
    check_backward(d, name, dx, dw, db)


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_undefined_stays_undefined(name):
    d = make(64, 48, 40, torch.float32, 12)
    d["z"][7, 5] = float("nan")
    dx, dw, db = torch.empty_like(d["x"]), torch.empty_like(d["w"]), torch.empty(40, device="cuda")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], name), act=name)
    assert torch.isnan(dx[7]).all() and torch.isnan(dw[5]).all() and torch.isnan(db[5])
    assert torch.isfinite(db[:5]).all() and torch.isfinite(dx[:7]).all()


@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("n_in,n_out", [(64, 48), (160, 136)])
def test_large_negative_pre_activations(name, n_in, n_out):
    # z = -80,000 in one column: y is 0 there, z is stored as -infinity, and nothing comes back from it
    d = make(100, n_in, n_out, torch.float16, 13)
    d["x"][:, 0], d["w"][2] = 40.0, 0.0
    d["w"][2, 0] = -2000.0
    d["bias"][2] = 0.0
    y, z = torch.empty_like(d["r"]), torch.empty_like(d["r"])
    ws = space(d["x"], d["w"], name)
    gs.gs_linear_fwd(d["x"], d["w"], d["bias"], y, ws, act=name, z=z)
    assert torch.isneginf(z[:, 2]).all() and not y[:, 2].any()
    dx, dw, db = torch.empty_like(d["x"]), torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
    gs.gs_linear_bwd(d["dy"], d["x"], d["w"], z, dx, dw, db, ws, act=name)
    assert not dw[2].any() and db[2] == 0
    check_backward({**d, "z": z.clamp(-300, 300)}, name, dx, dw, db)
