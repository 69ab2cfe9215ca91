"""The codebook and the mixture decoder: the operators together, as they are used, against float64 autograd from the same
binary16 weights (experts as the router chose them), captured in a HIP graph and replayed, on a stream of their own, and
in the training example."""
import os
import sys

import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from paper_2609_05255_amd.decoder import NORM_EPS, Codebook, MixtureDecoder
from rows_reference import act

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def setup(n, dim, hidden, blocks, experts, k, entries, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(-1, entries, (n,), generator=g, device="cuda").int()
    book = Codebook(codes, entries, dim, scale=1.5, seed=seed)
    dec = MixtureDecoder(n, dim, hidden, blocks, experts, k, seed=seed)
    dc0 = torch.randn(n, 3, generator=g, device="cuda").half()
    return book, dec, dc0


SIZES = [(500, 32, 48, 2, 4, 2, 40), (1, 64, 128, 1, 8, 2, 3), (3000, 40, 200, 2, 16, 3, 500), (77, 17, 9, 1, 3, 1, 20),
         (40, 24, 16, 1, 70, 4, 10)]


@pytest.mark.parametrize("n,dim,hidden,blocks,experts,k,entries", SIZES)
def test_against_autograd(n, dim, hidden, blocks, experts, k, entries):
    book, dec, dc0 = setup(n, dim, hidden, blocks, experts, k, entries)
    c0 = dec.forward(book.forward()).clone()
    dtable = book.backward(dec.backward(dc0)).clone()
    params = {p: (dec._half(*p) if p[1].startswith("w") or p[1] == "gate" else dec.weight(*p)).double().clone()
              .requires_grad_() for p in dec.names}
    table = book.half.double().requires_grad_()
    i = book.codes.long()
    v = torch.where((i >= 0)[:, None], table[i.clamp(min=0)] * book.scale, 0.0)
    for b in range(blocks):
        mu = v.mean(1, keepdim=True)
        xh = (v - mu) / torch.sqrt((v - mu).square().mean(1, keepdim=True) + NORM_EPS)
        a = xh * params[(b, "norm_w")] + params[(b, "norm_b")]
        chosen = dec.saved[b]["expert"].long()
        # nothing beyond the choices is larger than the last of them, but for the logits' rounding
        logits = a @ params[(b, "gate")].t()
        assert (logits.gather(1, chosen).amin(1) >= logits.topk(k, dim=1).values[:, -1] - 0.02 * logits.abs().amax()).all()
        p = torch.softmax(logits.gather(1, chosen), 1)
        out = torch.zeros_like(v)
        for e in range(experts):
            r, j = (chosen == e).nonzero(as_tuple=True)
            if r.numel():
                h = act("gelu", a[r] @ params[(b, "w1")][e].t() + params[(b, "b1")][e])
                out = out.index_add(0, r, p[r, j][:, None] * (h @ params[(b, "w2")][e].t() + params[(b, "b2")][e]))
        v = v + out
    out = v @ params[("head", "w")].t() + params[("head", "b")]
    out.backward(dc0.double())
    # binary16 values (2^-11 each): a dozen roundings per block along each path, in norm; the router's weights move by the
    # logits' own rounding, 2^-11 of values up to about 4
    limit = 2.0 ** -11 * (6 + 16 * blocks)
    rel = lambda p, q: float((p.double() - q).norm() / q.norm().clamp(min=1e-30))  # noqa: E731
    assert rel(c0, out.detach()) < limit
    if int((i >= 0).sum()):
        assert rel(dtable, table.grad) < limit
    for name, p in params.items():
        if name[1] == "gate":
            # its rows' gradients are differences of the choices' contributions, which nearly cancel where the experts
            # are alike: against the size of what is subtracted (with one choice they are exactly 0)
            if k == 1:
                assert not dec.grad(*name).any()
            else:
                s = dec.saved[name[0]]
                size = float((s["a"].double().abs().t() @ (dec.dweight.double().abs() * s["weight"].double()).sum(1)).norm())
                if name[0] == 0:   # (dweight is the first block's, the last one of the backward)
                    assert float((dec.grad(*name).double() - p.grad).norm()) < limit * (size + float(p.grad.norm()))
            continue
        want = p.grad if p.grad is not None else torch.zeros_like(p)
        assert rel(dec.grad(*name), want) < limit, name


def test_graph():
    """One captured step of both, replayed on changing inputs with eager work between: the eager bits."""
    n, dim, hidden, experts, k, entries = 20_000, 48, 72, 12, 2, 300
    book, dec, dc0 = setup(n, dim, hidden, 2, experts, k, entries)
    s = torch.cuda.Stream()

    def step():
        gs.gs_sort_rows(book.codes, book.order, book.workspace)
        c0 = dec.forward(book.forward())
        book.backward(dec.backward(dc0))
        return c0

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        book.codes.copy_(torch.randint(-1, entries, (n,), generator=g, device="cuda"))
        book.half.copy_(torch.randn(entries, dim, generator=g, device="cuda") * 0.5)
        dc0.copy_(torch.randn(n, 3, generator=g, device="cuda"))

    def outputs():
        return [dec.c0.clone(), book.grad.clone(), dec.grads.clone(), dec.saved[1]["order"].offsets.clone()]

    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for seed in (1, 2, 3, 4):
        with torch.cuda.stream(s):
            fill(seed)
            graph.replay()
            replayed = outputs()
            torch.randn(1000, device="cuda").sum().item()
            fill(seed)
            step()
            eager = outputs()
        s.synchronize()
        assert all(torch.isfinite(t.float()).all() for t in eager)
        assert all(torch.equal(a, b) for a, b in zip(replayed, eager)), seed


@pytest.mark.parametrize("n,dim,hidden,blocks,experts,k,entries", SIZES[:3])
def test_same_bits_on_another_stream(n, dim, hidden, blocks, experts, k, entries):
    book, dec, dc0 = setup(n, dim, hidden, blocks, experts, k, entries)
    out = []
    for stream in (None, torch.cuda.Stream()):
        torch.cuda.synchronize()
        dec.forward(book.forward(stream), stream)
        book.backward(dec.backward(dc0, stream), stream)
        torch.cuda.synchronize()
        out.append([dec.c0.clone(), book.grad.clone(), dec.grads.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_two_mixtures_at_once():
    """Two decoders with workspaces of their own, on two streams at the same time."""
    pairs = [setup(5000, 32, 64, 2, 8, 2, 100, seed=s) for s in (1, 2)]
    alone = []
    for book, dec, dc0 in pairs:
        dec.forward(book.forward())
        book.backward(dec.backward(dc0))
        torch.cuda.synchronize()
        alone.append([dec.c0.clone(), book.grad.clone(), dec.grads.clone()])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for (book, dec, dc0), s in zip(pairs, streams):
            dec.forward(book.forward(s), s)
            book.backward(dec.backward(dc0, s), s)
    torch.cuda.synchronize()
    for (book, dec, _), want in zip(pairs, alone):
        assert all(torch.equal(a, b) for a, b in zip([dec.c0, book.grad, dec.grads], want))


def test_refusals():
    x = torch.zeros(6, 8, device="cuda")
    o = gs.RowOrder(12, 4)
    with pytest.raises(ValueError):
        gs.gs_sort_rows(torch.zeros(11, dtype=torch.int32, device="cuda"), o)
    with pytest.raises(ValueError):
        gs.gs_sort_rows(torch.zeros(12, dtype=torch.int64, device="cuda"), o)
    with pytest.raises(ValueError):
        gs.gs_sort_rows(torch.zeros(12, dtype=torch.int32), o)
    gs.gs_sort_rows(torch.zeros(12, dtype=torch.int32, device="cuda"), o)
    with pytest.raises(ValueError):
        gs.gs_dispatch_fwd(x, o, torch.zeros(12, 7, device="cuda"))
    with pytest.raises(ValueError):
        gs.gs_dispatch_fwd(x, o, torch.zeros(12, 8, device="cuda", dtype=torch.float16))
    with pytest.raises(gs.GsError):   # 12 places for 5 rows
        gs.gs_dispatch_fwd(x[:5], o, torch.zeros(12, 8, device="cuda"))
    with pytest.raises(ValueError):
        gs.gs_combine_fwd(torch.zeros(12, 8, device="cuda"), o, torch.zeros(6, 3, device="cuda"), x)
    with pytest.raises(gs.GsError):   # no places
        gs.gs_combine_fwd(torch.zeros(12, 8, device="cuda"), _without(o, "place"), torch.zeros(6, 2, device="cuda"), x)
    with pytest.raises(gs.GsError):   # no sorted keys
        gs.gs_embedding_bwd(torch.zeros(12, 8, device="cuda"), _without(o, "sorted"), 1.0, torch.zeros(4, 8, device="cuda"),
                            torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        gs.gs_embedding_bwd(x, o, 1.0, torch.zeros(4, 8, device="cuda"), None)
    with pytest.raises(gs.GsError):   # more choices than experts
        gs.gs_route_fwd(x, torch.zeros(6, 9, dtype=torch.int32, device="cuda"), torch.zeros(6, 9, device="cuda"))
    w = torch.zeros(4, 5, 8, device="cuda")
    with pytest.raises(ValueError):
        gs.gs_experts_fwd(x, o.offsets[:4], w, None, torch.zeros(6, 5, device="cuda"))
    with pytest.raises(ValueError):
        gs.gs_experts_fwd(x, o.offsets, w, torch.zeros(5, device="cuda"), torch.zeros(6, 5, device="cuda"))
    with pytest.raises(ValueError):
        gs.gs_experts_fwd(x, o.offsets, w.transpose(1, 2), None, torch.zeros(6, 8, device="cuda"))


def _without(o, name):
    other = gs.RowOrder(o.count, o.groups, **{name: False})
    other.order, other.offsets = o.order, o.offsets
    return other


@pytest.mark.parametrize("codes,experts", [(64, 0), (0, 4), (200, 6)])
def test_training_example(codes, experts):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_decoder
    log = train_decoder.train(gaussians=3000, size=96, steps=12, dim=32, hidden=64, blocks=1, codes=codes,
                              experts=experts).cpu()
    assert torch.isfinite(log).all() and (log[:, 1] > 0).all()
