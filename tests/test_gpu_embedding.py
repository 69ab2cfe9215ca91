"""Embedding lookup and its gradient (gs_embedding_*) against 64 bits, at widths on both sides of every change of the
rows' spread over lanes, with frequent entries that many workgroups share, entries of a single row, and rows without an
entry. A lookup's value is one fp32 product and one rounding; a gradient an fp32 sum over the entry's rows."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from mixture_reference import embedding_grad
from rows_reference import U32, assert_close, strided, sum_bound

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def make_index(rows, entries, seed, spread):
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
    v = ((u ** 6 if spread == "skewed" else u) * entries).long().clamp(max=entries - 1)
    if spread == "one":
        v.fill_(entries // 2)
    if rows > 1:
        v = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.05, -1, v)
        v[0] = entries   # beyond the table
    return v.int()


def sort(index, entries):
    o = gs.RowOrder(index.numel(), entries, place=False)
    gs.gs_sort_rows(index, o, torch.empty(max(gs.gs_sort_rows_workspace_size(o), 1), dtype=torch.uint8, device="cuda"))
    return o


def normal(seed, *shape, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


SHAPES = [(1, 1, 1), (1, 256, 4096), (7, 3, 5), (100, 8, 3), (1000, 9, 50), (333, 17, 700), (513, 33, 20), (200, 64, 9),
          (1025, 65, 1000), (64, 255, 30), (100, 333, 77), (40, 512, 6), (33, 513, 8), (50, 1000, 20), (9, 2049, 4),
          (5, 5000, 3), (20_011, 24, 500), (70_000, 4, 100), (100_003, 64, 9000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,entries", SHAPES)
def test_lookup(rows, dim, entries, dtype):
    table, index = normal(1, entries, dim, dtype=dtype), make_index(rows, entries, rows, "even")
    y = torch.full((rows, dim), float("nan"), dtype=dtype, device="cuda")
    gs.gs_embedding_fwd(table, index, 1.7, y)
    i = index.long()
    keep = (i >= 0) & (i < entries)
    scale = float(torch.tensor(1.7))
    ref = torch.where(keep[:, None], table.double()[i.clamp(0, entries - 1)] * scale, 0.0)
    assert_close("y", y, ref, U32 * ref.abs(), dtype)
    assert torch.equal(y[~keep], torch.zeros_like(y[~keep]))


@pytest.mark.parametrize("spread", ["even", "skewed", "one"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,entries", SHAPES)
def test_gradient(rows, dim, entries, dtype, spread):
    index, dy = make_index(rows, entries, rows, spread), normal(2, rows, dim, dtype=dtype)
    order = sort(index, entries)
    ws = torch.full((gs.gs_embedding_workspace_size(dy),), 0xFF, dtype=torch.uint8, device="cuda")
    scale = float(torch.tensor(0.3))
    ref, size, count = embedding_grad(dy, index, entries, scale)
    bound = (sum_bound(1) + 4 * U32 * count.double().sqrt())[:, None] * size
    for out in {torch.float32, dtype}:
        dt = torch.full((entries, dim), float("nan"), dtype=out, device="cuda")
        gs.gs_embedding_bwd(dy, order, 0.3, dt, ws)
        assert_close("dtable", dt, ref, bound, out)
        assert torch.equal(dt[(count == 0).cuda()], torch.zeros_like(dt[(count == 0).cuda()]))
        again = torch.empty_like(dt)
        ws.zero_()
        gs.gs_embedding_bwd(dy, order, 0.3, again, ws)
        assert torch.equal(again, dt)   # the same bits


def test_many_rows_of_few_entries():
    """More positions than the groups of lanes take at once, entries of hundreds of thousands of rows."""
    rows, dim, entries = 1_500_007, 16, 11
    index, dy = make_index(rows, entries, 3, "skewed"), normal(4, rows, dim, dtype=torch.float16)
    ref, size, count = embedding_grad(dy, index, entries, 1.0)
    dt = torch.empty(entries, dim, device="cuda")
    gs.gs_embedding_bwd(dy, sort(index, entries), 1.0, dt,
                        torch.empty(gs.gs_embedding_workspace_size(dy), dtype=torch.uint8, device="cuda"))
    assert_close("dtable", dt, ref, (sum_bound(1) + 4 * U32 * count.double().sqrt())[:, None] * size, torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (5, 3), (8, 8)])
def test_strides(dtype, pad, offset):
    rows, dim, entries = 301, 45, 60
    index = make_index(rows, entries, 1, "even")
    table, dy = normal(5, entries, dim, dtype=dtype), normal(6, rows, dim, dtype=dtype)
    y, ys = (torch.empty(rows, dim, dtype=dtype, device="cuda") for _ in range(2))
    gs.gs_embedding_fwd(table, index, 2.0, y)
    ys = strided(ys, pad, offset)
    gs.gs_embedding_fwd(strided(table, pad, offset), index, 2.0, ys)
    assert torch.equal(y, ys)
    order = sort(index, entries)
    ws = torch.empty(gs.gs_embedding_workspace_size(dy), dtype=torch.uint8, device="cuda")
    dt = torch.empty(entries, dim, device="cuda")
    gs.gs_embedding_bwd(dy, order, 2.0, dt, ws)
    dts = strided(torch.zeros_like(dt), pad, offset)
    store = dts._base.clone() if dts._base is not None else None
    gs.gs_embedding_bwd(strided(dy, pad, offset), order, 2.0, dts, ws)
    assert torch.equal(dt, dts)
    if pad and store is not None:   # what lies between the rows is left alone
        between = torch.ones_like(store, dtype=torch.bool)
        between[offset:].view(entries, dim + pad)[:, :dim] = False
        assert torch.isnan(dts._base[between]).all()


def test_no_rows():
    dt = torch.full((5, 7), float("nan"), device="cuda")
    index = torch.empty(0, dtype=torch.int32, device="cuda")
    gs.gs_embedding_bwd(torch.empty(0, 7, device="cuda"), sort(index, 5), 1.0, dt, None)
    assert torch.equal(dt, torch.zeros_like(dt))
    gs.gs_embedding_fwd(dt, index, 1.0, torch.empty(0, 7, device="cuda"))


def test_special_values_stay_in_their_entries():
    index = torch.tensor([0, 1, 1, 3, 0, 4], dtype=torch.int32, device="cuda")
    dy = torch.ones(6, 20, device="cuda")
    dy[1, 3], dy[3, 5] = float("inf"), float("nan")
    dt = torch.empty(6, 20, device="cuda")
    gs.gs_embedding_bwd(dy, sort(index, 6), 1.0, dt,
                        torch.empty(gs.gs_embedding_workspace_size(dy), dtype=torch.uint8, device="cuda"))
    want = torch.tensor([2.0, 2.0, 0.0, 1.0, 1.0, 0.0], device="cuda")[:, None].repeat(1, 20)
    want[1, 3], want[3, 5] = float("inf"), float("nan")
    assert torch.equal(dt.nan_to_num(nan=-5.0), want.nan_to_num(nan=-5.0))


def test_gradient_against_differences():
    """sum(y c) moves by dtable as the table moves: exact for a function that is linear in the table."""
    rows, dim, entries = 50, 6, 9
    index, table = make_index(rows, entries, 8, "even"), normal(7, entries, dim)
    c = normal(8, rows, dim)
    dt = torch.empty_like(table)
    gs.gs_embedding_bwd(c, sort(index, entries), 3.0, dt,
                        torch.empty(gs.gs_embedding_workspace_size(c), dtype=torch.uint8, device="cuda"))

    def value(t):
        y = torch.empty(rows, dim, device="cuda")
        gs.gs_embedding_fwd(t, index, 3.0, y)
        return float((y.double() * c.double()).sum())

    for v, j in ((0, 0), (4, 3), (8, 5)):
        up, down = table.clone(), table.clone()
        up[v, j] += 1.0
        down[v, j] -= 1.0
        # (the moved values and the products are rounded to fp32: 4 roundings of at most 5 * 3 |c| each over the rows)
        size = 15 * float(c.abs().double().sum()) * 4 * U32
        assert abs((value(up) - value(down)) / 2 - float(dt[v, j])) <= size + 1e-6


def test_a_long_table():
    """Offsets beyond 32 bits: an entry more than 2^31 values behind the first."""
    entries, dim = 2 ** 22 + 8, 516
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("8.7 GB of table and gradient each")
    table = torch.zeros(entries, dim, dtype=torch.bfloat16, device="cuda")
    table[-1] = 3.0
    table[0] = 1.0
    index = torch.tensor([entries - 1, 0, entries - 1], dtype=torch.int32, device="cuda")
    y = torch.empty(3, dim, dtype=torch.bfloat16, device="cuda")
    gs.gs_embedding_fwd(table, index, 2.0, y)
    assert torch.equal(y[:, 0].cpu().float(), torch.tensor([6.0, 2.0, 6.0])) and torch.equal(y[0], y[2])
    table.fill_(float("nan"))
    gs.gs_embedding_bwd(y, sort(index, entries), 0.5, table,
                        torch.empty(gs.gs_embedding_workspace_size(y), dtype=torch.uint8, device="cuda"))
    assert torch.equal(table[-1].float(), torch.full((dim,), 6.0, device="cuda"))
    assert torch.equal(table[0].float(), torch.full((dim,), 1.0, device="cuda"))
    assert int(torch.count_nonzero(table)) == 2 * dim
