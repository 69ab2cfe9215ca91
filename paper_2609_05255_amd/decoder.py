"""A residual decoder over per-Gaussian embeddings, wider than the decoders fused into the preprocess: layer norm, a
hidden layer and its projection back with a skip connection, a few times, then a head with three outputs, the
Gaussian's base colour c0. Forward and backward run on the row operators (gs_layer_norm_*, gs_linear_*), a row per
Gaussian.

    a = norm(x), h = act(a W1^T + b1), x <- x + h W2^T + b2    (per block)
    c0 = x Wh^T + bh

The weights are one flat fp32 array with a binary16 copy that the products read, as FusedAdam keeps the decoders'
weights: one tensor of an Adam step, which writes the copy. Norm parameters and biases are read from the fp32 array
itself. Every tensor starts at a multiple of 8 values, so that its rows can be read as aligned vectors.
"""
from __future__ import annotations

import torch

from . import gsraster as gs

NORM_EPS = 1e-5


class ResidualDecoder:
    def __init__(self, n: int, dim: int, hidden: int, blocks: int, act: str = "gelu", seed: int = 0, device="cuda"):
        self.n, self.dim, self.hidden, self.act = n, dim, hidden, act
        self.names, at = {}, 0
        for b in range(blocks):
            for name, shape in (("norm_w", (dim,)), ("norm_b", (dim,)), ("w1", (hidden, dim)), ("b1", (hidden,)),
                                ("w2", (dim, hidden)), ("b2", (dim,))):
                self.names[(b, name)] = (at, shape)
                at += -(-torch.Size(shape).numel() // 8) * 8
        for name, shape in (("w", (3, dim)), ("b", (3,))):
            self.names[("head", name)] = (at, shape)
            at += -(-torch.Size(shape).numel() // 8) * 8
        self.blocks = blocks
        self.weights = torch.zeros(at, device=device)
        self.half = torch.zeros(at, dtype=torch.float16, device=device)
        self.grads = torch.zeros(at, device=device)
        g = torch.Generator(device=device).manual_seed(seed)
        for (b, name), (_, shape) in self.names.items():
            w = self.weight(b, name)
            if name == "norm_w":
                w.fill_(1.0)
            elif len(shape) == 2:
                # the skip connections start as near to the identity as the projections are small
                w.normal_(0.0, shape[1] ** -0.5 * (0.1 if name == "w2" else 1.0), generator=g)
        self.half.copy_(self.weights)
        rows = lambda k: torch.empty(n, k, dtype=torch.float16, device=device)  # noqa: E731
        # per block: the norm's output and statistics, z and h of the hidden layer, the block's output
        self.saved = [dict(a=rows(dim), mean=torch.empty(n, device=device), rstd=torch.empty(n, device=device),
                           z=rows(hidden), h=rows(hidden), x=rows(dim)) for _ in range(blocks)]
        self.c0 = rows(3)
        self.dx, self.dh, self.da = [rows(dim), rows(dim)], rows(hidden), rows(dim)
        size = max(gs.gs_linear_workspace_size(self.dx[0], self._half(0, "w1"), act) if blocks else 0,
                   gs.gs_linear_workspace_size(self.dh, self._half(0, "w2")) if blocks else 0,
                   gs.gs_linear_workspace_size(self.dx[0], self._half("head", "w")),
                   gs.gs_layer_norm_workspace_size(self.dx[0]), 1)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device)

    def _view(self, flat, b, name):
        at, shape = self.names[(b, name)]
        return flat[at:at + torch.Size(shape).numel()].view(shape)

    def weight(self, b, name):
        """The fp32 values of a tensor: block b (or "head"), norm_w, norm_b, w1, b1, w2, b2 (w, b)."""
        return self._view(self.weights, b, name)

    def grad(self, b, name):
        return self._view(self.grads, b, name)

    def _half(self, b, name):
        return self._view(self.half, b, name)

    def forward(self, x, stream=None):
        """c0 [n][3] of the embeddings x [n][dim] (binary16). Keeps what the backward needs, x among it."""
        self.x = x
        for b, s in enumerate(self.saved):
            gs.gs_layer_norm_fwd(x, self.weight(b, "norm_w"), self.weight(b, "norm_b"), NORM_EPS, s["a"], s["mean"],
                                 s["rstd"], stream)
            gs.gs_linear_fwd(s["a"], self._half(b, "w1"), self.weight(b, "b1"), s["h"], self.workspace, self.act,
                             z=s["z"], stream=stream)
            gs.gs_linear_fwd(s["h"], self._half(b, "w2"), self.weight(b, "b2"), s["x"], self.workspace, residual=x,
                             stream=stream)
            x = s["x"]
        gs.gs_linear_fwd(x, self._half("head", "w"), self.weight("head", "b"), self.c0, self.workspace, stream=stream)
        return self.c0

    def backward(self, dc0, stream=None):
        """The embeddings' gradient (binary16 [n][dim]); the weights' is in self.grads (fp32), overwritten."""
        ws, (dx, other) = self.workspace, self.dx
        x = self.saved[-1]["x"] if self.blocks else self.x
        gs.gs_linear_bwd(dc0, x, self._half("head", "w"), None, dx, self.grad("head", "w"), self.grad("head", "b"), ws,
                         stream=stream)
        for b in reversed(range(self.blocks)):
            s = self.saved[b]
            x = self.saved[b - 1]["x"] if b else self.x
            gs.gs_linear_bwd(dx, s["h"], self._half(b, "w2"), None, self.dh, self.grad(b, "w2"), self.grad(b, "b2"), ws,
                             stream=stream)
            gs.gs_linear_bwd(self.dh, s["a"], self._half(b, "w1"), s["z"], self.da, self.grad(b, "w1"),
                             self.grad(b, "b1"), ws, self.act, stream)
            # the skip connection's gradient joins the norm's
            gs.gs_layer_norm_bwd(self.da, x, self.weight(b, "norm_w"), s["mean"], s["rstd"], other,
                                 self.grad(b, "norm_w"), self.grad(b, "norm_b"), ws, add=dx, stream=stream)
            dx, other = other, dx
        return dx

    def adam_group(self, lr: float, beta2: float) -> dict:
        """The weights as one tensor of an Adam step (the gs_adam_step dict), which also writes the binary16 copy."""
        n = self.weights.numel()
        return dict(param=self.weights.view(1, n), grad=self.grads, exp_avg=torch.zeros_like(self.weights),
                    exp_avg_sq=torch.zeros_like(self.weights), param_half=self.half.view(torch.int16), rows=1, n=n,
                    beta2=beta2, lr=[lr])
