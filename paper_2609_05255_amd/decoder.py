"""A residual decoder over per-Gaussian embeddings, wider than the decoders fused into the preprocess: layer norm, a
hidden layer and its projection back with a skip connection, a few times, then a head with three outputs, the
Gaussian's base colour c0. Forward and backward run on the row operators (gs_layer_norm_*, gs_linear_*), a row per
Gaussian.

    a = norm(x), h = act(a W1^T + b1), x <- x + h W2^T + b2    (per block)
    c0 = x Wh^T + bh

The weights are one flat fp32 array with a binary16 copy that the products read, as FusedAdam keeps the decoders'
weights: one tensor of an Adam step, which writes the copy. Norm parameters and biases are read from the fp32 array
itself. Every tensor starts at a multiple of 8 values, so that its rows can be read as aligned vectors.

MixtureDecoder has a mixture of experts in place of the hidden layer (gs_route_*, gs_sort_rows, gs_dispatch_*,
gs_experts_*, gs_combine_*), and Codebook gives either its embeddings by an index into a table that the Gaussians share
(gs_embedding_*).
"""
from __future__ import annotations

import torch

from . import gsraster as gs

NORM_EPS = 1e-5


class _FlatWeights:
    """Weights in one flat fp32 array with a binary16 copy and an array of gradients. names: (block, name) to shape, in
    order; shapes of three sizes are those of experts."""

    def __init__(self, shapes: dict, seed: int, device):
        self.names, at = {}, 0
        for key, shape in shapes.items():
            self.names[key] = (at, shape)
            at += -(-torch.Size(shape).numel() // 8) * 8
        self.weights = torch.zeros(at, device=device)
        self.half = torch.zeros(at, dtype=torch.float16, device=device)
        self.grads = torch.zeros(at, device=device)
        g = torch.Generator(device=device).manual_seed(seed)
        for (b, name), (_, shape) in self.names.items():
            w = self.weight(b, name)
            if name == "norm_w":
                w.fill_(1.0)
            elif name.startswith("w") or name == "gate":
                # the skip connections start as near to the identity as the projections are small
                w.normal_(0.0, shape[-1] ** -0.5 * (0.1 if name == "w2" else 1.0), generator=g)
        self.half.copy_(self.weights)

    def _view(self, flat, b, name):
        at, shape = self.names[(b, name)]
        return flat[at:at + torch.Size(shape).numel()].view(shape)

    def weight(self, b, name):
        """The fp32 values of a tensor: block b (or "head"), and its name as in the class's shapes."""
        return self._view(self.weights, b, name)

    def grad(self, b, name):
        return self._view(self.grads, b, name)

    def _half(self, b, name):
        return self._view(self.half, b, name)

    def adam_group(self, lr: float, beta2: float) -> dict:
        """The weights as one tensor of an Adam step (the gs_adam_step dict), which also writes the binary16 copy."""
        n = self.weights.numel()
        return dict(param=self.weights.view(1, n), grad=self.grads, exp_avg=torch.zeros_like(self.weights),
                    exp_avg_sq=torch.zeros_like(self.weights), param_half=self.half.view(torch.int16), rows=1, n=n,
                    beta2=beta2, lr=[lr])


class ResidualDecoder(_FlatWeights):
    def __init__(self, n: int, dim: int, hidden: int, blocks: int, act: str = "gelu", seed: int = 0, device="cuda"):
        self.n, self.dim, self.hidden, self.blocks, self.act = n, dim, hidden, blocks, act
        shapes = {}
        for b in range(blocks):
            for name, shape in (("norm_w", (dim,)), ("norm_b", (dim,)), ("w1", (hidden, dim)), ("b1", (hidden,)),
                                ("w2", (dim, hidden)), ("b2", (dim,))):
                shapes[(b, name)] = shape
        for name, shape in (("w", (3, dim)), ("b", (3,))):
            shapes[("head", name)] = shape
        super().__init__(shapes, seed, device)
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


class Codebook:
    """Embeddings that Gaussians share: row i of the decoder's input is scale * table[codes[i]] (codes int32, n values of
    any shape; a Gaussian whose code is none of the table's has an embedding of zeros). The table is kept in fp32 with a
    binary16 copy that the lookups read. The book keeps a copy of the codes, sorted once for the table's gradient, and
    again when set_codes changes them or a forward finds that torch has written them; what becomes of the caller's tensor
    does not matter. (Neither a captured forward's replay nor a write by address is found: where codes change like that,
    set_codes is captured with the forward, or called with the book's own codes.)"""

    def __init__(self, codes, entries: int, dim: int, scale: float = 1.0, seed: int = 0):
        device = codes.device
        self.scale, self.entries, self.dim = scale, entries, dim
        g = torch.Generator(device=device).manual_seed(seed)
        self.table = torch.randn(entries, dim, generator=g, device=device) * 0.5
        self.half, self.grad = self.table.half(), torch.zeros_like(self.table)
        self.x = torch.empty(codes.numel(), dim, dtype=torch.float16, device=device)
        self.order = gs.RowOrder(codes.numel(), entries, device=device, place=False)
        size = max(gs.gs_sort_rows_workspace_size(self.order), gs.gs_embedding_workspace_size(self.x), 1)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device)
        with torch.inference_mode(False):   # (a tensor whose version tells of writes)
            self._codes = torch.empty(codes.numel(), dtype=torch.int32, device=device)
        self._sorted = None   # the version of the codes that the order is of
        self.set_codes(codes)

    @property
    def codes(self):
        """The book's own codes, int32 [n]."""
        return self._codes

    def set_codes(self, codes, stream=None):
        """Other codes, as many: copied and sorted. Codes that are refused change nothing."""
        n = self._codes.numel()
        if (codes.numel() != n or codes.dtype != torch.int32 or codes.device != self._codes.device
                or not codes.is_contiguous()):
            raise ValueError("codes: %s of %s on %s, a contiguous int32 tensor of %d values on %s expected" % (
                tuple(codes.shape), codes.dtype, codes.device, n, self._codes.device))
        gs._one_device(codes)
        if codes is not self._codes:
            if isinstance(stream, int):
                stream = torch.cuda.ExternalStream(stream, device=codes.device)
            with torch.cuda.stream(stream):   # (None: the current one)
                self._codes.copy_(codes.view(-1))
            if stream is not None:
                codes.record_stream(stream)   # (the caller may let go of them before they are read)
        gs.gs_sort_rows(self._codes, self.order, self.workspace, stream)
        if not torch.cuda.is_current_stream_capturing():   # (else nothing is sorted before the graph runs)
            self._sorted = self._codes._version

    def forward(self, stream=None):
        """The embeddings [n][dim] (binary16)."""
        if self._codes._version != self._sorted:
            self.set_codes(self._codes, stream)
        gs.gs_embedding_fwd(self.half, self._codes, self.scale, self.x, stream)
        return self.x

    def backward(self, dx, stream=None):
        """The table's gradient (fp32, overwritten) from that of the embeddings (binary16 [n][dim])."""
        gs.gs_embedding_bwd(dx, self.order, self.scale, self.grad, self.workspace, stream)
        return self.grad

    def adam_group(self, lr: float, beta2: float = 0.999) -> dict:
        """The table as one tensor of an Adam step, which also writes the binary16 copy."""
        n = self.table.numel()
        return dict(param=self.table.view(1, n), grad=self.grad, exp_avg=torch.zeros_like(self.table),
                    exp_avg_sq=torch.zeros_like(self.table), param_half=self.half.view(torch.int16), rows=1, n=n,
                    beta2=beta2, lr=[lr])


class MixtureDecoder(_FlatWeights):
    """The residual decoder with a mixture of experts in each block: a router sends each Gaussian's row to k of them.

        a = norm(x), l = a G^T, (e_j, p_j) = the k largest logits and their softmax
        x <- x + sum over j of p_j (act(a W1_e_j^T + b1_e_j) W2_e_j^T + b2_e_j)     (per block)
        c0 = x Wh^T + bh

    Forward and backward read nothing back: where each expert's rows begin stays on the GPU."""

    def __init__(self, n: int, dim: int, hidden: int, blocks: int, experts: int, k: int = 2, act: str = "gelu",
                 seed: int = 0, device="cuda"):
        self.n, self.dim, self.hidden, self.blocks, self.experts, self.k, self.act = (n, dim, hidden, blocks, experts, k,
                                                                                      act)
        shapes = {}
        for b in range(blocks):
            for name, shape in (("norm_w", (dim,)), ("norm_b", (dim,)), ("gate", (experts, dim)),
                                ("w1", (experts, hidden, dim)), ("b1", (experts, hidden)),
                                ("w2", (experts, dim, hidden)), ("b2", (experts, dim))):
                shapes[(b, name)] = shape
        for name, shape in (("w", (3, dim)), ("b", (3,))):
            shapes[("head", name)] = shape
        super().__init__(shapes, seed, device)
        rows = lambda m, c: torch.empty(m, c, dtype=torch.float16, device=device)  # noqa: E731
        floats = lambda *shape: torch.empty(shape, device=device)  # noqa: E731
        nk = n * k
        # per block: the norm's output and statistics, the logits, choices and their order, the experts' inputs, hidden
        # layer and results, the block's output
        self.saved = [dict(a=rows(n, dim), mean=floats(n), rstd=floats(n), logits=rows(n, experts),
                           expert=torch.empty(n, k, dtype=torch.int32, device=device), weight=floats(n, k),
                           order=gs.RowOrder(nk, experts, device=device, sorted=False), xs=rows(nk, dim),
                           z=rows(nk, hidden), h=rows(nk, hidden), ys=rows(nk, dim), x=rows(n, dim))
                      for _ in range(blocks)]
        self.c0 = rows(n, 3)
        self.dx, self.da = [rows(n, dim), rows(n, dim)], [rows(n, dim), rows(n, dim)]
        self.dys, self.dh, self.dxs = rows(nk, dim), rows(nk, hidden), rows(nk, dim)
        self.dweight, self.dlogits = floats(n, k), rows(n, experts)
        size = max(gs.gs_linear_workspace_size(self.dx[0], self._half("head", "w")),
                   gs.gs_layer_norm_workspace_size(self.dx[0]), 1)
        if blocks:
            size = max(size, gs.gs_linear_workspace_size(self.dx[0], self._half(0, "gate")),
                       gs.gs_sort_rows_workspace_size(self.saved[0]["order"]),
                       gs.gs_experts_workspace_size(self.dxs, self._half(0, "w1"), act),
                       gs.gs_experts_workspace_size(self.dh, self._half(0, "w2")))
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device)

    def forward(self, x, stream=None):
        """c0 [n][3] of the embeddings x [n][dim] (binary16). Keeps what the backward needs, x among it."""
        self.x, ws = x, self.workspace
        for b, s in enumerate(self.saved):
            order = s["order"]
            gs.gs_layer_norm_fwd(x, self.weight(b, "norm_w"), self.weight(b, "norm_b"), NORM_EPS, s["a"], s["mean"],
                                 s["rstd"], stream)
            gs.gs_linear_fwd(s["a"], self._half(b, "gate"), None, s["logits"], ws, stream=stream)
            gs.gs_route_fwd(s["logits"], s["expert"], s["weight"], stream=stream)
            gs.gs_sort_rows(s["expert"], order, ws, stream)
            gs.gs_dispatch_fwd(s["a"], order, s["xs"], stream)
            gs.gs_experts_fwd(s["xs"], order.offsets, self._half(b, "w1"), self.weight(b, "b1"), s["h"], ws, self.act,
                              z=s["z"], stream=stream)
            gs.gs_experts_fwd(s["h"], order.offsets, self._half(b, "w2"), self.weight(b, "b2"), s["ys"], ws,
                              stream=stream)
            gs.gs_combine_fwd(s["ys"], order, s["weight"], s["x"], residual=x, stream=stream)
            x = s["x"]
        gs.gs_linear_fwd(x, self._half("head", "w"), self.weight("head", "b"), self.c0, ws, stream=stream)
        return self.c0

    def backward(self, dc0, stream=None):
        """The embeddings' gradient (binary16 [n][dim]); the weights' is in self.grads (fp32), overwritten."""
        ws, (dx, other) = self.workspace, self.dx
        x = self.saved[-1]["x"] if self.blocks else self.x
        gs.gs_linear_bwd(dc0, x, self._half("head", "w"), None, dx, self.grad("head", "w"), self.grad("head", "b"), ws,
                         stream=stream)
        for b in reversed(range(self.blocks)):
            s = self.saved[b]
            order = s["order"]
            x = self.saved[b - 1]["x"] if b else self.x
            gs.gs_combine_bwd(dx, s["ys"], order, s["weight"], self.dys, self.dweight, stream)
            gs.gs_experts_bwd(self.dys, s["h"], order.offsets, self._half(b, "w2"), None, self.dh, self.grad(b, "w2"),
                              self.grad(b, "b2"), ws, stream=stream)
            gs.gs_experts_bwd(self.dh, s["xs"], order.offsets, self._half(b, "w1"), s["z"], self.dxs, self.grad(b, "w1"),
                              self.grad(b, "b1"), ws, self.act, stream)
            gs.gs_route_bwd(self.dweight, None, s["expert"], s["weight"], self.dlogits, stream=stream)
            gs.gs_linear_bwd(self.dlogits, s["a"], self._half(b, "gate"), None, self.da[0], self.grad(b, "gate"), None, ws,
                             stream=stream)
            gs.gs_dispatch_bwd(self.dxs, order, self.da[1], add=self.da[0], stream=stream)
            # the skip connection's gradient joins the norm's
            gs.gs_layer_norm_bwd(self.da[1], x, self.weight(b, "norm_w"), s["mean"], s["rstd"], other,
                                 self.grad(b, "norm_w"), self.grad(b, "norm_b"), ws, add=dx, stream=stream)
            dx, other = other, dx
        return dx
