"""The row operators in float64 with torch, and the error bounds that their tests hold the kernels to."""
import math

import torch

U32 = 2.0 ** -24
# half the spacing of a type's values at 1: the relative error of rounding to it
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}
# half the spacing of the smallest values: what rounding to the type may lose beside a relative error
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}


def act(name, z):
    return {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * torch.special.ndtr(v),
            "silu": lambda v: v * torch.sigmoid(v), "tanh": torch.tanh, "sigmoid": torch.sigmoid}[name](z)


def slope(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "tanh":
        return 1 - torch.tanh(z) ** 2
    s = torch.sigmoid(z)
    return s * (1 - s) if name == "sigmoid" else s * (1 + z * (1 - s))


def sum_bound(length):
    """Relative (to the sum of magnitudes) error of an fp32 sum of `length` products, added up in some order: the
    errors of sqrt(length) steps beyond a few, as of a random walk, with a factor of four."""
    return 4 * U32 * (4 + math.sqrt(length))


def assert_close(name, got, ref, bound, dtype):
    """|got - ref| <= bound (an fp32 error, per element) plus one rounding to dtype."""
    got, ref = got.double().cpu(), ref.cpu()
    bound = torch.as_tensor(bound, dtype=torch.float64).cpu()
    limit = bound * (1 + UNIT[dtype]) + UNIT[dtype] * ref.abs() + TINY[dtype]
    off = (got - ref).abs()
    bad = ~(off <= limit)
    if bad.any():
        k = int(torch.argmax((off / limit).nan_to_num(nan=float("inf")).reshape(-1)))
        raise AssertionError("%s: %d of %d values off; worst at %d: %r, %r expected, limit %.3g" % (
            name, int(bad.sum()), bad.numel(), k, got.reshape(-1)[k].item(), ref.reshape(-1)[k].item(),
            limit.expand_as(off).reshape(-1)[k].item()))


def strided(t, pad, offset=0):
    """The same matrix with rows `pad` elements further apart, `offset` elements into its storage; what lies between
    the rows is not a number."""
    rows, cols = t.shape
    store = torch.full((rows * (cols + pad) + offset,), float("nan"), dtype=t.dtype, device=t.device)
    view = store[offset:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view
