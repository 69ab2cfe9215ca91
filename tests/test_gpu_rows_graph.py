"""The row operators captured in a HIP graph on a stream of their own and replayed on changing inputs, with eager work and
synchronisations between the replays. They allocate nothing, wait for nothing and add in fixed orders, so every replay
must give the bits of the eager calls on the same inputs."""
import pytest
import torch

from paper_2609_05255_amd import gsraster as gs

pytestmark = pytest.mark.gpu


def space(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")


class Chain:
    """x -> layer norm -> linear with residual -> back, its gradients' norm, and their clipping into fp32."""

    def __init__(self, rows, dim, out, dtype):
        t = {"dtype": dtype, "device": "cuda"}
        f = {"device": "cuda"}
        self.x, self.dy = torch.zeros(rows, dim, **t), torch.zeros(rows, out, **t)
        self.w, self.r = torch.zeros(out, dim, **t), torch.zeros(rows, out, **t)
        self.nw, self.nb, self.b = torch.zeros(dim, **f), torch.zeros(dim, **f), torch.zeros(out, **f)
        self.a, self.da, self.dx = (torch.zeros(rows, dim, **t) for _ in range(3))
        self.y, self.z = torch.zeros(rows, out, **t), torch.zeros(rows, out, **t)
        self.mean, self.rstd = torch.zeros(rows, **f), torch.zeros(rows, **f)
        self.dw, self.db = torch.zeros(out, dim, **f), torch.zeros(out, **f)
        self.dnw, self.dnb = torch.zeros(dim, **f), torch.zeros(dim, **f)
        self.clipped = torch.zeros(rows, dim, **f)
        self.result = torch.zeros(2, **f)
        self.grads = gs.GradSet([self.dx], [self.clipped])
        self.ws_norm = space(gs.gs_layer_norm_workspace_size(self.x))
        self.ws = space(gs.gs_linear_workspace_size(self.x, self.w, "gelu"))
        self.ws_grad = space(gs.gs_grad_workspace_size(self.grads))

    def fill(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t, scale in ((self.x, 1.0), (self.dy, 1.0), (self.w, 0.1), (self.r, 1.0), (self.nw, 1.0), (self.nb, 1.0),
                         (self.b, 1.0)):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda") * scale)

    def run(self):
        gs.gs_layer_norm_fwd(self.x, self.nw, self.nb, 1e-5, self.a, self.mean, self.rstd)
        gs.gs_linear_fwd(self.a, self.w, self.b, self.y, self.ws, act="gelu", residual=self.r, z=self.z)
        gs.gs_linear_bwd(self.dy, self.a, self.w, self.z, self.da, self.dw, self.db, self.ws, act="gelu")
        gs.gs_layer_norm_bwd(self.da, self.x, self.nw, self.mean, self.rstd, self.dx, self.dnw, self.dnb, self.ws_norm)
        gs.gs_grad_clip(self.grads, 1.0, self.result, self.ws_grad)

    def outputs(self):
        return {k: getattr(self, k).clone() for k in ("a", "y", "z", "da", "dw", "db", "dx", "dnw", "dnb", "clipped", "result")}


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,dim,out", [(3, 64, 40), (500, 96, 72), (300, 1040, 200), (2001, 333, 129)])
def test_rows_in_a_graph(rows, dim, out, dtype):
    c = Chain(rows, dim, out, dtype)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.fill(0)
        c.run()   # the first launches of a kernel are not captured
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.run()
    for seed in (1, 2, 3, 4):
        with torch.cuda.stream(s):
            c.fill(seed)
            g.replay()
            replayed = c.outputs()
            torch.randn(1000, device="cuda").sum().item()
            c.fill(seed)
            c.run()
            eager = c.outputs()
        s.synchronize()
        assert torch.isfinite(eager["result"]).all() and float(eager["result"][0]) > 1.0
        for k in eager:
            assert torch.equal(replayed[k], eager[k]), (k, seed)
