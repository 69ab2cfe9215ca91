"""The linear operators' larger tiles, and the ones whose groups of waves share a sum, on matrices with rows further apart
than their columns, and the tiles with dz in planes where the gradient is infinite."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from rows_reference import strided
from test_gpu_linear import TYPES, check_backward, check_forward, make, space

pytestmark = pytest.mark.gpu


# 256 x 256 tiles (the first two), groups that share a sum, 128 x 128 tiles, split sums; rows at aligned strides (what
# lies between is NaN) and off the vectors' alignment
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(4166, 520, 4104), (300, 4096, 4608), (1000, 2064, 968), (70, 1032, 2048),
                                             (20_000, 128, 256), (256, 1536, 264)])
@pytest.mark.parametrize("pad,offset", [(8, 0), (24, 8), (7, 1)])
def test_strides(rows, n_in, n_out, dtype, pad, offset):
    d = make(rows, n_in, n_out, dtype, 19)
    s = {k: strided(v, pad, offset) if v.dim() == 2 else v for k, v in d.items()}
    y, z = (strided(torch.zeros_like(d["r"]), pad, offset) for _ in range(2))
    gs.gs_linear_fwd(s["x"], s["w"], d["bias"], y, space(d["x"], d["w"], "gelu", None), act="gelu", residual=s["r"], z=z)
    check_forward(d, "gelu", y, z)
    for name, dw_type in (("silu", torch.float32), ("relu", dtype), ("none", torch.float32)):
        dx = strided(torch.zeros_like(d["x"]), pad, offset)
        dw = strided(torch.zeros(n_out, n_in, dtype=dw_type, device="cuda"), pad, offset)
        db = torch.full((n_out,), float("nan"), device="cuda")
        gs.gs_linear_bwd(s["dy"], s["x"], s["w"], s["z"], dx, dw, db, space(d["x"], d["w"], name, dw_type), act=name)
        check_backward(d, name, dx, dw, db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(300, 200, 160), (4100, 264, 1040), (70, 1032, 2048), (2100, 1000, 960)])
def test_infinite_gradient(rows, n_in, n_out, dtype):
    # an infinite dy makes its row of dx and its column's dw and db infinite or undefined; the rest is as without it
    d = make(rows, n_in, n_out, dtype, 6)
    d["z"][7, 3], d["z"][rows - 1, n_out - 1] = 1.0, -0.25
    d["dy"][7, 3], d["dy"][rows - 1, n_out - 1] = float("inf"), float("-inf")
    for name in ("silu", "gelu", "relu"):
        dx = torch.full_like(d["x"], float("nan"))
        dw = torch.full((n_out, n_in), float("nan"), device="cuda")
        db = torch.full((n_out,), float("nan"), device="cuda")
        gs.gs_linear_bwd(d["dy"], d["x"], d["w"], d["z"], dx, dw, db, space(d["x"], d["w"], name), act=name)
        assert db[3] == float("inf") and torch.equal(dw[3], d["x"][7].float().sign() * float("inf"))
        assert not torch.isfinite(dx[7]).any()
        cols, keep = list(range(n_out)), list(range(rows))
        cols.remove(3)
        keep.remove(7)
        if name != "relu":   # (whose slope at -0.25 is 0)
            assert db[n_out - 1] != 0 and not torch.isfinite(db[n_out - 1]) and not torch.isfinite(dw[n_out - 1]).any()
            assert not torch.isfinite(dx[rows - 1]).any()
            cols.remove(n_out - 1)
            keep.remove(rows - 1)
        clean = dict(d)
        clean["dy"] = d["dy"].clone()
        clean["dy"][7, 3] = clean["dy"][rows - 1, n_out - 1] = 0.0
        check_backward({**clean, "dy": clean["dy"][keep], "z": d["z"][keep], "x": d["x"][keep]}, name, dx[keep], None, None)
        check_backward({**clean, "dy": clean["dy"][:, cols], "z": d["z"][:, cols], "w": d["w"][cols]}, name, None,
                       dw[cols], db[cols])


# more z and y than the cache holds, in the narrow form and in tiles: by the activation, the inputs' width and x's alignment
@pytest.mark.parametrize("rows,n_in,n_out,name,pad", [(1_100_003, 32, 64, "gelu", 0), (1_100_003, 32, 64, "relu", 4),
                                                      (1_100_003, 32, 64, "none", 8), (600_001, 72, 120, "relu", 0),
                                                      (1_500_001, 17, 45, "relu", 0)])
def test_forward_of_more_than_the_cache_holds(rows, n_in, n_out, name, pad):
    d = make(rows, n_in, n_out, torch.float16, 3)
    x = strided(d["x"], pad) if pad else d["x"]
    y, z = (torch.full_like(d["r"], float("nan")) for _ in range(2))
    gs.gs_linear_fwd(x, d["w"], d["bias"], y, space(d["x"], d["w"], name, None), act=name, residual=d["r"], z=z)
    for part in (slice(0, 2000), slice(rows // 2, rows // 2 + 2000), slice(rows - 2000, rows)):
        check_forward({k: v[part] if v.shape[0] == rows else v for k, v in d.items()}, name, y[part], z[part])
    assert torch.isfinite(y).all() and torch.isfinite(z).all()
