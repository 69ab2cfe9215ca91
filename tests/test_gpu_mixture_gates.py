"""The router's gradient in every block of a mixture decoder against float64 autograd.

A gate's gradient is the sum over rows of dl a, dl_j = p_j (dw_j - sum of p dw), dw_j = dy . ys_j. Each factor carries the
roundings to binary16 along its path, a relative `limit` in norm; those of different rows and columns are independent, so
they add in squares: dw_j is off by limit (|dw_j| + |dy| |ys_j| / sqrt(dim)), dl_j by p_j times that and its mean over the
choices, the sum by the root of the rows' squares."""
import pytest
import torch

from paper_2609_05255_amd.decoder import NORM_EPS, MixtureDecoder
from rows_reference import act

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,dim,hidden,blocks,experts,k", [(500, 32, 48, 2, 4, 2), (3000, 40, 200, 3, 16, 3),
                                                         (800, 64, 128, 4, 8, 2), (40, 24, 16, 2, 70, 4)])
def test_gates_of_every_block(n, dim, hidden, blocks, experts, k):
    g = torch.Generator(device="cuda").manual_seed(41)
    x = (torch.randn(n, dim, generator=g, device="cuda") * 0.7).half()
    dc0 = torch.randn(n, 3, generator=g, device="cuda").half()
    dec = MixtureDecoder(n, dim, hidden, blocks, experts, k, seed=42)
    dec.forward(x)
    dx = dec.backward(dc0)
    params = {p: (dec._half(*p) if p[1].startswith("w") or p[1] == "gate" else dec.weight(*p)).double().clone()
              .requires_grad_() for p in dec.names}
    start = x.double().requires_grad_()
    v, kept = start, []
    for b in range(blocks):
        mu = v.mean(1, keepdim=True)
        xh = (v - mu) / torch.sqrt((v - mu).square().mean(1, keepdim=True) + NORM_EPS)
        a = xh * params[(b, "norm_w")] + params[(b, "norm_b")]
        chosen = dec.saved[b]["expert"].long()   # (experts as the router chose them)
        p = torch.softmax((a @ params[(b, "gate")].t()).gather(1, chosen), 1)
        ys = torch.zeros(n, k, dim, dtype=torch.float64, device="cuda")
        for e in range(experts):
            r, j = (chosen == e).nonzero(as_tuple=True)
            if r.numel():
                h = act("gelu", a[r] @ params[(b, "w1")][e].t() + params[(b, "b1")][e])
                ys = ys.index_put((r, j), h @ params[(b, "w2")][e].t() + params[(b, "b2")][e])
        v = v + (p.unsqueeze(2) * ys).sum(1)
        p.retain_grad()
        v.retain_grad()
        kept.append((a, p, ys, v))
    out = v @ params[("head", "w")].t() + params[("head", "b")]
    out.backward(dc0.double())
    # binary16 values (2^-11 each): a dozen roundings per block along each path; the weights move by the logits' own
    # rounding, 2^-11 of values up to about 4
    limit = 2.0 ** -11 * (6 + 16 * blocks)
    assert float((dx.double() - start.grad).norm()) < limit * float(start.grad.norm())
    for b, (a, p, ys, v) in enumerate(kept):
        a, q, dw = a.detach(), p.detach(), p.grad
        off = dw.abs() + v.grad.norm(dim=1)[:, None] * ys.detach().norm(dim=2) / dim ** 0.5
        off = q * (off + (q * off).sum(1, keepdim=True))
        bound = limit * float((a.norm(dim=1, keepdim=True) * off).norm())
        grad, want = dec.grad(b, "gate").double(), params[(b, "gate")].grad
        assert float((grad - want).norm()) < bound, b
        # (half of a gradient, one that is left out, or another block's is further off than that)
        assert float(want.norm()) > 4 * bound, b
