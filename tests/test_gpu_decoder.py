"""The residual decoder on the row operators against float64 autograd, FusedAdam with clipping against the same steps
on clipped gradients, and the training example."""
import os
import sys

import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from paper_2609_05255_amd import inputs
from paper_2609_05255_amd.decoder import NORM_EPS, ResidualDecoder
from paper_2609_05255_amd.optim import FusedAdam
from parity import tiny_camera
from rows_reference import act

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("n,dim,hidden,blocks", [(500, 32, 48, 2), (1, 64, 128, 1), (3000, 40, 200, 3), (77, 17, 9, 1)])
def test_decoder_against_autograd(n, dim, hidden, blocks):
    dec = ResidualDecoder(n, dim, hidden, blocks, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(n, dim, generator=gen, device="cuda").half()
    dc0 = torch.randn(n, 3, generator=gen, device="cuda").half()
    c0 = dec.forward(x).clone()
    dx = dec.backward(dc0).clone()
    # the same in float64 from the same binary16 weights (norm parameters and biases from the fp32 ones)
    params = {k: (dec._half(*k) if k[1].startswith("w") else dec.weight(*k)).double().clone().requires_grad_()
              for k in dec.names}
    xd = x.double().requires_grad_()
    v = xd
    for b in range(blocks):
        mu = v.mean(1, keepdim=True)
        xh = (v - mu) / torch.sqrt((v - mu).square().mean(1, keepdim=True) + NORM_EPS)
        a = xh * params[(b, "norm_w")] + params[(b, "norm_b")]
        h = act("gelu", a @ params[(b, "w1")].t() + params[(b, "b1")])
        v = v + h @ params[(b, "w2")].t() + params[(b, "b2")]
    out = v @ params[("head", "w")].t() + params[("head", "b")]
    out.backward(dc0.double())
    # binary16 activations (2^-11 each): a handful of roundings per block along each path, in norm
    limit = 2.0 ** -11 * (4 + 6 * blocks)
    rel = lambda p, q: float((p.double() - q).norm() / q.norm())  # noqa: E731
    assert rel(c0, out.detach()) < limit
    assert rel(dx, xd.grad) < limit
    for k, p in params.items():
        assert rel(dec.grad(*k), p.grad) < limit, k


@pytest.mark.parametrize("hit", [False, True])
def test_fused_adam_clips(hit):
    sc = inputs.make_scene("tiny", appearance=("neural",))
    cam = tiny_camera()
    cs = gs.camera_struct(cam)
    up = torch.from_numpy(inputs.make_upstream_grad(cam.width, cam.height, 0)).cuda()
    results = []
    for clip in (True, False):
        st = gs.SceneTensors(sc)
        fr = gs.Frame(sc.n, cam.width, cam.height, gs.GS_APP_NEURAL, 1 << 16)
        fr.forward(cs, st)
        fr.backward(cs, st, up)
        plain = FusedAdam(st, fr, gs.GS_APP_NEURAL)
        if not results:   # the same gradients for both (the backward's atomics vary in the last bits)
            grads = [g["grad"].clone() for g in plain.groups]
        for g, t in zip(plain.groups, grads):
            g["grad"].copy_(t)
        norm = float(torch.stack([t.double().square().sum() for t in grads]).sum().sqrt())
        bound = norm * (0.125 if hit else 8.0)
        if clip:
            opt = FusedAdam(st, fr, gs.GS_APP_NEURAL, max_grad_norm=bound)
            opt.step()
            assert abs(float(opt.clip[0]) - norm) <= 1e-6 * norm
            c = float(opt.clip[1])
            assert (c < 1.0) == hit
            assert all(torch.equal(g["grad"], t) for g, t in zip(opt.groups, grads))
        else:
            opt = plain
            for g in opt.groups:
                g["grad"] *= c
            opt.step()
        results.append([(g["param"].clone(), g["exp_avg"].clone(), g["exp_avg_sq"].clone()) for g in opt.groups])
    for a, b in zip(*results):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_clipping_and_the_step_inside_the_backward_exclude_each_other():
    sc = inputs.make_scene("tiny")
    st = gs.SceneTensors(sc)
    fr = gs.Frame(sc.n, 64, 64, gs.GS_APP_SH3, 1 << 14)
    opt = FusedAdam(st, fr, gs.GS_APP_SH3, max_grad_norm=1.0)
    with pytest.raises(ValueError, match="clipping"):
        opt.backward_step(fr, None, st, None)


def test_training_example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_decoder
    log = train_decoder.train(gaussians=3000, size=96, steps=60, dim=32, hidden=64, blocks=1).cpu()
    assert torch.isfinite(log).all() and (log[:, 1] > 0).all()
    # four cameras take turns: the last round against the first
    assert float(log[-4:, 0].mean()) < 0.5 * float(log[:4, 0].mean()), log[:, 0]
