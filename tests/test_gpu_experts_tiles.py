"""The experts' products in their largest tiles, and tiles that are split along the sum: 256 x 256 ones whole, with a split
tail (of dx too) and with parts of dW, 128 x 128 ones with a split tail, a split that is left without a share of the sum,
beside experts without rows and rows that are no expert's. Against float64 with the bounds of the other experts' tests;
compared on the GPU, as the matrices have tens of millions of values. Which tiles these sizes take follows from the plan's
rates: 256 x 256 in all three products at 2,048 -> 2,048, in the forward at 1,032 -> 2,056, in dW at 7,000 rows."""
import pytest
import torch

import test_gpu_experts as experts_tests
from paper_2609_05255_amd import gsraster as gs
from rows_reference import TINY, U32, UNIT, sum_bound
from test_gpu_experts import ACT_ERROR, NAN, backward, check_backward, check_forward, forward

pytestmark = pytest.mark.gpu

HALVES = [torch.float16, torch.bfloat16]


def assert_close_here(name, got, ref, bound, dtype):
    got = got.double()
    limit = bound * (1 + UNIT[dtype]) + UNIT[dtype] * ref.abs() + TINY[dtype]
    bad = ~((got - ref).abs() <= limit)
    if bad.any():
        k = int(torch.argmax(((got - ref).abs() / limit).nan_to_num(nan=float("inf")).reshape(-1)))
        raise AssertionError("%s: %d of %d values off; worst at %d: %r, %r expected, limit %.3g" % (
            name, int(bad.sum()), bad.numel(), k, got.reshape(-1)[k].item(), ref.reshape(-1)[k].item(),
            limit.reshape(-1)[k].item()))


@pytest.fixture(autouse=True)
def compare_on_the_gpu(monkeypatch):
    monkeypatch.setattr(experts_tests, "assert_close", assert_close_here)


def make(lengths, spare, n_in, n_out, dtype, seed):
    """As the other tests' inputs, with the rows that each expert has; `spare` more are nobody's."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    experts, rows = len(lengths), sum(lengths) + spare
    ends = [sum(lengths[:e]) for e in range(experts + 1)]
    d = dict(x=rand(rows, n_in).to(dtype), w=(rand(experts, n_out, n_in) * n_in ** -0.5).to(dtype),
             b=rand(experts, n_out) * 0.3, dy=(rand(rows, n_out) * 0.1).to(dtype), z=(rand(rows, n_out) * 1.5).to(dtype))
    for name in ("x", "dy", "z"):
        d[name][ends[-1]:] = NAN
    for e in range(experts):
        if lengths[e] == 0:
            d["w"][e] = NAN
    d.update(ends=ends, offsets=torch.tensor(ends, dtype=torch.int32, device="cuda"))
    return d


# (rows of the experts, spare rows, in, out)
SIZES = [
    # 68 units of 256 rows: 544 tiles of 256 x 256, the last 32 split into four; an expert's dW in two parts
    ([9000, 0, 3000, 1500, 1284, 300, 1000, 300], 0, 2048, 2048),
    # one expert has all: 512 tiles, none left to split, and two parts of its dW
    ([0, 0, 0, 16_300, 0, 0, 0, 0], 84, 2048, 2048),
    # 65 units: the last 8 of 520 tiles, sums of 33 steps, in eight splits of five steps: the last split has none
    ([8200, 0, 5100, 3000], 84, 2056, 2048),
    # 256 x 256 in the forward, whole, edges in both directions
    ([3700, 0, 5000, 1, 2900], 399, 1032, 2056),
    # dx in 128 x 128, the last 24 of 1,048 tiles split into four
    ([9000, 0, 4500, 3000], 0, 1024, 1032),
    # dW in 256 x 256 with parts
    ([4500, 0, 2300], 200, 1032, 2056),
]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("lengths,spare,n_in,n_out", SIZES)
def test_forward(lengths, spare, n_in, n_out, dtype):
    d = make(lengths, spare, n_in, n_out, dtype, 31)
    check_forward(d, "gelu", *forward(d, "gelu"))
    check_forward(d, "none", *forward(d, "none", keep=False, bias=False), bias=False)


@pytest.mark.parametrize("name,same", [("silu", False), ("relu", False), ("tanh", True)])
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("lengths,spare,n_in,n_out", SIZES)
def test_backward(lengths, spare, n_in, n_out, dtype, name, same):
    d = make(lengths, spare, n_in, n_out, dtype, 32)
    check_backward(d, name, *backward(d, name, dtype if same else torch.float32))


# 63 units of 128 rows: 2,079 tiles of 128 x 128, the last 31 split into eight, of which the last has no share
@pytest.mark.parametrize("lengths,spare,n_in,n_out", [([3840, 0, 4160], 0, 1032, 4104), ([4096, 1280, 2048], 576, 2048, 2048)])
def test_fp32(lengths, spare, n_in, n_out):
    d = make(lengths, spare, n_in, n_out, torch.float32, 33)
    check_forward(d, "silu", *forward(d, "silu"))
    check_backward(d, "gelu", *backward(d, "gelu", torch.float32))


@pytest.mark.parametrize("dtype", [torch.float32] + HALVES)
def test_same_bits(dtype):
    """Twice the same, whatever the workspace holds, and each gradient alone."""
    d = make(*SIZES[0][:2], 2048, 2048, dtype, 34)
    for a, b in zip(forward(d, "gelu"), forward(d, "gelu")):
        assert torch.equal(a, b)
    whole = backward(d, "silu", torch.float32)
    for k, name in enumerate(("dx", "dw", "db")):
        assert torch.equal(backward(d, "silu", torch.float32, want=(name,))[k], whole[k])
        assert torch.equal(backward(d, "silu", torch.float32)[k], whole[k])


@pytest.mark.parametrize("dtype", HALVES)
def test_captured(dtype):
    """Shares that change between replays: tiles, their split tail and the parts of dW are found on the GPU."""
    lengths, spare, n_in, n_out = SIZES[0]
    d = make(lengths, spare, n_in, n_out, dtype, 35)
    d["w"].nan_to_num_(nan=0.25)
    rows, s = d["x"].shape[0], torch.cuda.Stream()
    y, z, dx = (torch.empty(rows, n, dtype=dtype, device="cuda") for n in (n_out, n_out, n_in))
    dw, db = torch.empty(d["w"].shape, device="cuda"), torch.empty(d["w"].shape[:2], device="cuda")
    ws = torch.empty(gs.gs_experts_workspace_size(d["x"], d["w"], "silu"), dtype=torch.uint8, device="cuda")

    def run():
        gs.gs_experts_fwd(d["x"], d["offsets"], d["w"], d["b"], y, ws, act="silu", z=z)
        gs.gs_experts_bwd(d["dy"], d["x"], d["offsets"], d["w"], z, dx, dw, db, ws, act="silu")

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run()
    for shares in (lengths, [0, 0, 0, rows, 0, 0, 0, 0], [rows // 8] * 8, [rows - 7, 1, 1, 1, 1, 1, 1, 1], lengths[::-1]):
        ends = torch.tensor([sum(shares[:e]) for e in range(9)], dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            d["offsets"].copy_(ends)
            graph.replay()
            replayed = [t.clone() for t in (y, z, dx, dw, db)]
            torch.randn(1000, device="cuda").sum().item()
            run()
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (y, z, dx, dw, db))), shares


def test_gradients_against_differences():
    """Each place's own outputs only, so that the bound is far below the gradient: central differences of sum(c y) err by
    h^2 / 6 times its third derivative (silu's is below 0.4: 3 s'' + z s''' with s the sigmoid, |s''| < 0.1, |s'''| <= 1 / 8
    and |z s'''| < 0.1) and by the rounding of the outputs over h."""
    experts, n_in, n_out = 3, 9, 7
    lengths = [20, 9, 6]
    d = make(lengths, 5, n_in, n_out, torch.float32, 36)
    used = sum(lengths)
    c = torch.randn(used + 5, n_out, generator=torch.Generator(device="cuda").manual_seed(37), device="cuda")
    _, z = forward(d, "silu")
    d.update(z=z, dy=c)
    dx, dw, db = backward(d, "silu", torch.float32)
    h = 2.0 ** -5
    owner = [e for e in range(experts) for _ in range(lengths[e])]

    def rounding(r, o):
        """of output (r, o), at most, with the moved operand"""
        x, w = d["x"][r].double().abs() + h, d["w"][owner[r], o].double().abs() + h
        size = float((x * w).sum())
        b = float(d["b"][owner[r], o].abs()) + h
        return sum_bound(n_in) * size + 2 * U32 * (b + size) + ACT_ERROR * (1 + size + b) + U32 * (size + b)

    places = [("x", (r, j)) for r in (0, 19, 20, 28, used - 1) for j in (0, 8)]
    places += [("w", (e, o, j)) for e in range(experts) for o, j in ((0, 0), (3, 5), (6, 8))]
    places += [("b", (e, o)) for e in range(experts) for o in (0, 6)]
    for name, at in places:
        if name == "x":
            outputs = [(at[0], o, float(d["w"][owner[at[0]], o, at[1]])) for o in range(n_out)]
        else:
            outputs = [(r, at[1], float(d["x"][r, at[2]]) if name == "w" else 1.0) for r in range(used) if owner[r] == at[0]]
        moved = []
        for step in (h, -h):
            t = {k: d[k].clone() for k in ("x", "w", "b")}
            t[name][at] += step
            y, _ = forward(dict(d, **t), "silu")
            moved.append(sum(float(c[r, o]) * float(y[r, o]) for r, o, _ in outputs))
        weights = [abs(float(c[r, o])) for r, o, _ in outputs]
        bound = sum(v * (0.4 * abs(a) ** 3 * h * h / 6 + rounding(r, o) / h) for v, (r, o, a) in zip(weights, outputs))
        # the gradient's own error, and the step's (an operand plus or minus h is rounded to fp32)
        own = sum(v * abs(a) * 1.1 * (sum_bound(len(outputs)) + 2 * ACT_ERROR + 8 * U32 / h) for v, (_, _, a) in zip(weights, outputs))
        grad = {"x": dx, "w": dw, "b": db}[name]
        assert bound + own <= 0.02 * sum(v * abs(a) for v, (_, _, a) in zip(weights, outputs)) + 1e-3, (name, at)
        assert abs((moved[0] - moved[1]) / (2 * h) - float(grad[at])) <= bound + own, (name, at)
