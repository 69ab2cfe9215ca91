"""The router (gs_route_*) against one choice after the other in 64 bits: experts on both sides of every change of the
rows' spread over lanes, ties, masked experts and rows, undefined and infinite logits, one row and many; the gradient
against automatic differentiation. Weights: the fp32 errors of exp, whose argument x carries 3 |x| roundings (difference,
product, constant) and whose result 4, of the sum (up to 24 additions deep) and of the division."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from mixture_reference import route, route_grad
from rows_reference import U32, assert_close, strided

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
INF = float("inf")


def make(rows, experts, dtype, seed, masked=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    l = torch.randn(rows, experts, generator=g, device="cuda") * 2
    if masked:
        l[torch.rand(rows, experts, generator=g, device="cuda") < 0.4] = -INF
        l[::5] = -INF
    return l.to(dtype)


def forward(l, k, normalise):
    expert = torch.full((l.shape[0], k), -9, dtype=torch.int32, device="cuda")
    weight = torch.full((l.shape[0], k), float("nan"), device="cuda")
    gs.gs_route_fwd(l, expert, weight, normalise=normalise)
    return expert, weight


def spread(l):
    """Sum over a row of p |x|, x the distance from the largest logit."""
    l = l.double().cpu()
    x = torch.where(torch.isneginf(l), 0.0, l - l.amax(1, keepdim=True).clamp(min=-1e300))
    p = torch.softmax(l, 1).nan_to_num(nan=0.0)
    return (p * x.abs()).sum(1, keepdim=True), x


def check(l, k, normalise):
    expert, weight = forward(l, k, normalise)
    re, rw = route(l, k, normalise)
    assert torch.equal(expert.cpu().long(), re)
    mean, x = spread(l)
    far = x.gather(1, re.clamp(min=0)).abs()
    # (among the chosen the mean distance is smaller than over all)
    assert_close("weight", weight, rw, rw * U32 * (3 * far + 3 * mean + 4 + 4 + 24 + 2) * 1.01, torch.float32)
    return expert, weight


SHAPES = [(1, 1, 1), (1, 8, 2), (5, 2, 2), (9, 3, 1), (70, 4, 4), (33, 5, 3), (64, 8, 8), (17, 9, 2), (100, 16, 16),
          (20, 17, 5), (50, 37, 3), (40, 64, 2), (21, 65, 6), (12, 128, 8), (10, 200, 16), (8, 256, 4), (7, 257, 3),
          (6, 500, 16), (5, 513, 2), (4, 1000, 7), (3, 1024, 16)]


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,k", SHAPES)
def test_forward(rows, experts, k, dtype, masked, normalise):
    check(make(rows, experts, dtype, rows * experts, masked), k, normalise)


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,k", SHAPES)
def test_backward(rows, experts, k, dtype, masked, normalise):
    l = make(rows, experts, dtype, rows + experts, masked)
    g = torch.Generator(device="cuda").manual_seed(3)
    dw = torch.randn(rows, k, generator=g, device="cuda")
    expert, weight = check(l, k, normalise)
    dl = torch.full_like(l, float("nan"))
    gs.gs_route_bwd(dw, None if normalise else l, expert, weight, dl, normalise=normalise)
    ref = route_grad(dw, l, expert.cpu(), normalise)
    # p (dw - inner): p and inner carry the weights' relative errors, inner k more, the difference one
    mean, x = spread(l)
    w = weight.double().cpu()
    size = (w * dw.double().cpu().abs()).sum(1, keepdim=True)
    err = U32 * (3 * x.abs().clamp(max=60) + 3 * mean + 3 * x.gather(1, expert.cpu().long().clamp(min=0)).abs().amax(1, keepdim=True) + 60 + k)
    p = torch.softmax(l.double().cpu(), 1).nan_to_num(nan=0.0)
    at = torch.zeros_like(p)
    for j in range(k):
        e = expert[:, j].cpu().long()
        r = (e >= 0).nonzero().view(-1)
        at[r, e[r]] = dw[r.cuda(), j].double().cpu().abs()
        if normalise:
            p[r, e[r]] = w[r, j]
    assert_close("dlogits", dl, ref, p * (at + size) * err * 1.01, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_go_to_the_lowest(dtype):
    l = torch.zeros(4, 40, dtype=dtype, device="cuda")
    l[1, 7::3] = 1.0
    l[2] = torch.finfo(dtype).min   # finite: ordinary logits
    l[3, ::2] = -0.0                # the two zeros are equal
    expert, weight = check(l, 3, True)
    assert expert.tolist() == [[0, 1, 2], [7, 10, 13], [0, 1, 2], [0, 1, 2]]


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
def test_masks(dtype, normalise):
    """Rows with fewer experts than choices, the last of them with none."""
    l = make(5, 12, dtype, 1)
    l[0, 1:] = -INF
    l[1, :10] = -INF
    l[2, 3:] = torch.finfo(dtype).min
    l[4] = -INF
    expert, weight = check(l, 4, normalise)
    assert expert[0].tolist() == [0, -1, -1, -1] and weight[0].tolist() == [1.0, 0.0, 0.0, 0.0]
    assert expert[4].tolist() == [-1] * 4 and weight[4].tolist() == [0.0] * 4
    dw = torch.ones(5, 4, device="cuda")
    dw[4], dw[0, 1:] = float("nan"), float("nan")   # of no expert: not read
    dl = torch.full_like(l, float("nan"))
    gs.gs_route_bwd(dw, l, expert, weight, dl, normalise=normalise)
    assert torch.isfinite(dl).all() and not dl[4].any() and not dl[0].any()


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts", [24, 27, 64, 300])
def test_undefined_and_infinite(dtype, normalise, experts):
    """Experts are valid whatever the logits, undefined ones first whatever their sign; other rows keep their weights."""
    l = make(40, experts, dtype, 2)
    clean = l.clone()
    l[3, 5], l[17, 20], l[17, 2] = float("nan"), INF, INF
    l[30, experts - 1] = -torch.tensor(float("nan"), dtype=dtype, device="cuda")
    expert, weight = forward(l, 3, normalise)
    e0, w0 = forward(clean, 3, normalise)
    others = [r for r in range(40) if r not in (3, 17, 30)]
    assert expert[30, 0] == experts - 1 and torch.isnan(weight[30]).all()
    assert torch.equal(expert[others], e0[others]) and torch.equal(weight[others], w0[others])
    assert expert[3, 0] == 5 and expert[17, :2].tolist() == [2, 20]
    assert ((expert >= 0) & (expert < experts)).all()
    assert torch.isnan(weight[3]).all()
    assert all(len(set(r)) == 3 for r in expert.tolist())


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_many_rows(dtype):
    l = make(30_001, 33, dtype, 4)
    expert, weight = forward(l, 2, False)
    s = strided(l, 3, 1)
    e2, w2 = forward(s, 2, False)
    assert torch.equal(expert, e2) and torch.equal(weight, w2)
    top = torch.sort(l.float(), dim=1, descending=True, stable=True).indices[:, :2]
    assert torch.equal(expert.long(), top)
    dw = torch.randn(30_001, 2, device="cuda")
    dl = torch.empty_like(l)
    gs.gs_route_bwd(dw, l, expert, weight, dl, normalise=False)
    dls = strided(torch.zeros_like(l), 3, 1)
    gs.gs_route_bwd(dw, s, expert, weight, dls, normalise=False)
    assert torch.equal(dl, dls)


def test_gradient_against_differences():
    l = make(6, 10, torch.float32, 6)
    dw = torch.randn(6, 3, device="cuda")
    for normalise in (True, False):
        expert, weight = forward(l, 3, normalise)
        dl = torch.empty_like(l)
        gs.gs_route_bwd(dw, l, expert, weight, dl, normalise=normalise)
        h = 2.0 ** -7
        for e in range(10):
            up, down = l.clone(), l.clone()
            up[:, e] += h
            down[:, e] -= h
            (eu, wu), (ed, wd) = forward(up, 3, normalise), forward(down, 3, normalise)
            same = (eu == expert).all(1) & (ed == expert).all(1)
            diff = ((wu - wd).double() * dw.double()).sum(1) / (2 * h)
            # third derivatives of a softmax are at most 1; the weights' own errors are divided by h
            bound = (dw.double().abs().sum(1)) * (h * h / 6 + 100 * U32 / h)
            assert (((diff - dl[:, e].double()).abs() <= bound) | ~same).all()
        assert same.any()


def test_no_rows():
    forward(torch.empty(0, 8, device="cuda"), 2, True)
    gs.gs_route_bwd(torch.empty(0, 2, device="cuda"), None, torch.empty(0, 2, dtype=torch.int32, device="cuda"),
                    torch.empty(0, 2, device="cuda"), torch.empty(0, 8, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts", [1, 5, 37, 64, 600])
def test_gradient_in_the_place_of_the_logits(experts, dtype):
    l = make(203, experts, dtype, 8)
    k = min(experts, 6)
    expert, weight = forward(l, k, False)
    dw, dl = torch.randn(203, k, device="cuda"), torch.empty_like(l)
    gs.gs_route_bwd(dw, l, expert, weight, dl, normalise=False)
    gs.gs_route_bwd(dw, l, expert, weight, l, normalise=False)
    assert torch.equal(l, dl)


def test_a_long_matrix_of_logits():
    """Rows that begin more than 2^31 values behind the first."""
    rows, experts = 2 ** 25 + 3, 72
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("4.8 GB of logits")
    l = torch.zeros(rows, experts, dtype=torch.float16, device="cuda")
    l[-1, 70], l[-1, 3] = 2.0, 1.0
    expert, weight = forward(l, 2, True)
    assert expert[-1].tolist() == [70, 3] and expert[0].tolist() == [0, 1] and expert[-2].tolist() == [0, 1]
    last = forward(l[-1:], 2, True)[1]
    dw = torch.zeros(rows, 2, device="cuda")
    dw[-1, 0] = 1.0
    gs.gs_route_bwd(dw, None, expert, weight, l)
    assert torch.equal(weight[-1:], last) and int(torch.count_nonzero(l)) == 2
    assert float(l[-1, 70]) > 0 > float(l[-1, 3])
