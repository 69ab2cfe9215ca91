"""Trains a scene whose base colours come from a residual decoder over per-Gaussian embeddings.

    python examples/train_decoder.py --gaussians 100000 --steps 50

Each step decodes the base colour of every Gaussian (ResidualDecoder: layer norm, linear layers with activation and
skip connection), renders one camera, takes the squared error against that camera's image of a reference scene, goes
back through the rasterizer and the decoder, clips the gradients by their global norm and applies Adam to the geometry,
the embeddings and the decoder's weights. The embeddings' gradient is binary16; clipping writes it into the fp32 array
that the Adam step reads. Losses and norms stay on the GPU until the end.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_05255_amd import gsraster as gs  # noqa: E402
from paper_2609_05255_amd import inputs, optim  # noqa: E402
from paper_2609_05255_amd.decoder import ResidualDecoder  # noqa: E402

# the gradients are kept this many times larger than the loss's, so that binary16 holds the embeddings' (Adam's step
# does not depend on their scale)
LOSS_SCALE = 4096.0


def group(param, grad, lr, half=None, beta2=0.999):
    rows = len(lr)
    return dict(param=param.view(rows, -1), grad=grad, exp_avg=torch.zeros_like(param),
                exp_avg_sq=torch.zeros_like(param), param_half=half, rows=rows, n=param.numel() // rows, beta2=beta2,
                lr=lr)


def train(gaussians: int, size: int, steps: int, dim: int = 64, hidden: int = 128, blocks: int = 2, cameras: int = 4,
          max_norm: float = 1.0, device="cuda"):
    """Losses and gradient norms of the steps, as a [steps][2] tensor on the GPU."""
    kind = gs.GS_APP_NASG   # at degree 0 the lobe is off and a Gaussian's colour is max(0, c0 + 0.5)
    scene = gs.SceneTensors(inputs.make_scene("medium", n=gaussians, appearance=("nasg",)), device)
    views = [inputs.look_at_camera([3.0 * c, 0.4, 3.0 * s], size, size)
             for c, s in ((torch.cos(a).item(), torch.sin(a).item()) for a in torch.arange(cameras) * 6.28318 / cameras)]
    views = [gs.camera_struct(v) for v in views]
    probe = gs.Frame(gaussians, size, size, kind, 1, device=device)
    pairs = max(gs.gs_preprocess(v, scene.gaussians(), scene.appearance(kind, 0), probe.pre, probe.workspace,
                                 probe.ws_bytes) for v in views)
    del probe
    frame = gs.Frame(gaussians, size, size, kind, 2 * pairs + 4096, device=device)
    targets = []
    for v in views:
        frame.forward(v, scene, sh_degree=0)
        targets.append(frame.image.clone())

    gen = torch.Generator(device=device).manual_seed(1)
    embedding = torch.randn(gaussians, dim, generator=gen, device=device) * 0.5   # fp32, with a binary16 copy
    half = embedding.half()
    d_embedding = torch.empty_like(embedding)
    decoder = ResidualDecoder(gaussians, dim, hidden, blocks, device=device)
    groups = [group(scene.means, frame.dmeans, [optim.LR_MEANS] * 3),
              group(scene.log_scales, frame.dlog_scales, [optim.LR_SCALES] * 3),
              group(scene.quats, frame.dquats, [optim.LR_QUATS] * 4),
              group(scene.opacity_logits, frame.dopacity_logits, [optim.LR_OPACITY]),
              group(embedding, d_embedding, [optim.LR_FEATURES], half.view(torch.int16)),
              decoder.adam_group(optim.LR_MLP, optim.BETA2_MLP)]
    clip = torch.empty(2, device=device)
    log = torch.empty(steps, 2, device=device)
    dc0 = torch.empty(gaussians, 3, dtype=torch.float16, device=device)
    grad_set = workspace = None
    for step in range(1, steps + 1):
        view, target = views[step % cameras], targets[step % cameras]
        scene.base_color.copy_(decoder.forward(half).t())
        frame.forward(view, scene, sh_degree=0, sync_pairs=False)
        error = frame.image - target
        frame.backward(view, scene, error * (2.0 * LOSS_SCALE / error.numel()), sh_degree=0)
        dc0.copy_(frame.dbase_color.t())
        d_half = decoder.backward(dc0)
        if grad_set is None:   # the buffers stay the same from here on
            grad_set = gs.GradSet([g["grad"] for g in groups[:4]] + [d_half, decoder.grads],
                                  out=[None] * 4 + [d_embedding, None])
            workspace = torch.empty(gs.gs_grad_workspace_size(grad_set), dtype=torch.uint8, device=device)
        gs.gs_grad_clip(grad_set, max_norm * LOSS_SCALE, clip, workspace)
        gs.gs_adam_step(groups, 0.9, 1e-15, step)
        log[step - 1, 0] = error.square().mean()
        log[step - 1, 1] = clip[0] / LOSS_SCALE
    if frame.pairs_overflowed():
        raise RuntimeError("more (tile, Gaussian) pairs than the buffers hold")
    return log


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--gaussians", type=int, default=100_000)
    p.add_argument("--size", type=int, default=400)
    p.add_argument("--steps", type=int, default=50)
    p.add_argument("--dim", type=int, default=64)
    p.add_argument("--hidden", type=int, default=128)
    p.add_argument("--blocks", type=int, default=2)
    p.add_argument("--max-norm", type=float, default=1.0)
    a = p.parse_args()
    log = train(a.gaussians, a.size, a.steps, a.dim, a.hidden, a.blocks, max_norm=a.max_norm).cpu()
    for k in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d  loss %.6f  gradient norm %.3e" % (k + 1, log[k, 0], log[k, 1]))
    print("step %4d  loss %.6f  gradient norm %.3e" % (a.steps, log[-1, 0], log[-1, 1]))


if __name__ == "__main__":
    main()
