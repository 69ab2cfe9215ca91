"""FusedAdam with clipping takes the norm of the gradients that its groups name when step() is called, as the step
itself does: tensors that a caller replaces or adds between steps count."""
import math

import pytest
import torch

from paper_2609_05255_amd import gsraster as gs
from paper_2609_05255_amd import inputs
from paper_2609_05255_amd.optim import FusedAdam

pytestmark = pytest.mark.gpu


def optimiser(**kw):
    scene = gs.SceneTensors(inputs.make_scene("tiny"))
    frame = gs.Frame(scene.n, 64, 64, gs.GS_APP_SH3, 1 << 14)
    opt = FusedAdam(scene, frame, gs.GS_APP_SH3, **kw)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for g in opt.groups:
        g["grad"].normal_(0.0, 1e-3, generator=gen)
    return opt


def norm(opt):
    return math.sqrt(sum(float(g["grad"].double().square().sum()) for g in opt.groups))


def results(opt):
    return [g[k].clone() for g in opt.groups for k in ("param", "exp_avg", "exp_avg_sq")]


def check_step(opt, plain):
    """One step of opt, and of an optimiser without clipping on the clipped gradients."""
    opt.step()
    want = norm(opt)
    assert abs(float(opt.clip[0]) - want) <= 1e-6 * want
    c = opt.clip[1]
    assert abs(float(c) - min(1.0, opt.max_grad_norm / want)) <= 1e-5
    for g, h in zip(plain.groups, opt.groups):
        g["grad"] = h["grad"] * c
    plain.step()
    assert all(torch.equal(a, b) for a, b in zip(results(opt), results(plain)))


def test_replaced_gradients_count():
    opt, plain = optimiser(max_grad_norm=0.05), optimiser()
    check_step(opt, plain)
    old = opt.groups[0]["grad"]
    opt.groups[0]["grad"] = old * 300.0
    old.zero_()
    check_step(opt, plain)


def test_a_larger_group_counts():
    # more gradients than the optimiser was made with: its workspace grows
    opt, plain = optimiser(max_grad_norm=0.05), optimiser()
    n = 30_000_000
    gen = torch.Generator(device="cuda").manual_seed(3)
    param, grad = (torch.randn(1, n, generator=gen, device="cuda") * s for s in (1.0, 1e-3))
    for o in (opt, plain):
        o.groups.append(dict(param=param.clone(), grad=grad.clone(), exp_avg=torch.zeros_like(param),
                             exp_avg_sq=torch.zeros_like(param), param_half=None, rows=1, n=n, beta2=0.999, lr=[1e-3]))
    check_step(opt, plain)
    check_step(opt, plain)
