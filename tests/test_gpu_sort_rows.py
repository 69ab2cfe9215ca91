"""Rows sorted by key (gs_sort_rows): whole numbers, equal to a stable sort's, for few and many positions on both sides
of every change of form, from one group to millions, with frequent, rare and absent groups and positions without one."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from mixture_reference import sort_rows

pytestmark = pytest.mark.gpu


def run(group_of, groups, sorted=True, place=True, workspace_fill=0xAB):
    o = gs.RowOrder(group_of.numel(), groups, sorted=sorted, place=place)
    for t in (o.order, o.sorted, o.place, o.offsets):
        if t is not None:
            t.fill_(-7)
    ws = torch.full((max(gs.gs_sort_rows_workspace_size(o), 1),), workspace_fill, dtype=torch.uint8, device="cuda")
    gs.gs_sort_rows(group_of, o, ws)
    return o


def check(group_of, groups, **kw):
    o = run(group_of, groups, **kw)
    order, key, place, offsets = sort_rows(group_of, groups)
    assert torch.equal(o.offsets.cpu().long(), offsets)
    assert torch.equal(o.order.cpu().long(), order)
    if o.sorted is not None:
        assert torch.equal(o.sorted.cpu().long(), key)
    if o.place is not None:
        assert torch.equal(o.place.cpu().long(), place)


def draw(count, groups, seed, spread="even"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(count, generator=g, device="cuda", dtype=torch.float64)
    if spread == "skewed":
        u = u ** 8
    v = (u * groups).long().clamp(max=groups - 1)
    if spread != "full":
        v = torch.where(torch.rand(count, generator=g, device="cuda") < 0.1, -1, v)
    return v.int()


COUNTS = [1, 2, 63, 64, 65, 1000, 4096, 8191, 8192, 8193, 12_289, 100_003, 1_000_003]
GROUPS = [1, 2, 16, 255, 256, 257, 16_384, 16_385, 65_535, 65_536, 1_000_000]


@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("count", COUNTS)
def test_sort(count, groups):
    check(draw(count, groups, count + groups), groups)


@pytest.mark.parametrize("spread", ["skewed", "full"])
@pytest.mark.parametrize("count,groups", [(5000, 7), (300_001, 255), (300_001, 5000), (200_000, 20_000_000)])
def test_spreads(count, groups, spread):
    check(draw(count, groups, 5, spread), groups)


@pytest.mark.parametrize("count", [5, 8192, 50_000])
@pytest.mark.parametrize("value", [0, 3, 99, 100, -1, -2147483648, 2147483647])
def test_one_value(count, value):
    """Every position in one group, or in none."""
    check(torch.full((count,), value, dtype=torch.int32, device="cuda"), 100)


@pytest.mark.parametrize("count", [100, 20_000])
@pytest.mark.parametrize("sorted", [True, False])
@pytest.mark.parametrize("place", [True, False])
@pytest.mark.parametrize("groups", [50, 30_000, 2 ** 31 - 2])
def test_left_out_arrays(count, sorted, place, groups):
    if groups > 10 ** 9:
        pytest.skip("offsets of 8 GiB") if torch.cuda.mem_get_info()[0] < 40 << 30 else None
        v = draw(count, groups, 9)
        o = run(v, groups, sorted=sorted, place=place)
        order, key, at, _ = sort_rows(v, groups)
        assert torch.equal(o.order.cpu().long(), order)
        some = torch.unique(key[key < groups])
        want = torch.searchsorted(key, some)
        assert torch.equal(o.offsets[some.cuda()].cpu().long(), want)
        assert int(o.offsets[-1]) == int((key < groups).sum())
        return
    check(draw(count, groups, 9), groups, sorted=sorted, place=place)


def test_no_positions():
    o = run(torch.empty(0, dtype=torch.int32, device="cuda"), 300)
    assert torch.equal(o.offsets.cpu(), torch.zeros(301, dtype=torch.int32))


def test_same_bits_and_matrix_input():
    v = draw(60_000, 40, 3).view(20_000, 3)
    check(v, 40)
    a, b = run(v, 40), run(v, 40, workspace_fill=0)
    assert torch.equal(a.order, b.order) and torch.equal(a.place, b.place)


def test_other_stream():
    s = torch.cuda.Stream()
    v = draw(100_000, 1000, 4)
    torch.cuda.synchronize()
    o = gs.RowOrder(v.numel(), 1000)
    ws = torch.empty(gs.gs_sort_rows_workspace_size(o), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    gs.gs_sort_rows(v, o, ws, stream=s)
    s.synchronize()
    assert torch.equal(o.order.cpu().long(), sort_rows(v, 1000)[0])


@pytest.mark.parametrize("groups", [16, 1_000_000])
def test_many_positions(groups):
    """300 million positions: more than the rest of the tests has in all, checked on the GPU."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("15 GB")
    count = 300_000_007
    v = torch.randint(-1, groups, (count,), dtype=torch.int32, device="cuda")
    o = run(v, groups, place=False)
    key = torch.where(v < 0, groups, v)
    assert torch.equal(key[o.order.long()], o.sorted)
    rising = o.sorted[1:] > o.sorted[:-1]
    assert ((o.order[1:] > o.order[:-1]) & (o.sorted[1:] == o.sorted[:-1]) | rising).all()
    counts = torch.bincount(key, minlength=groups + 1)
    assert torch.equal(o.offsets[1:].long(), counts[:-1].cumsum(0)) and int(o.offsets[0]) == 0
