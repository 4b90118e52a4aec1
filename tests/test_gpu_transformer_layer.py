"""A layer norm and the linear layer behind it, trained as a program would: forward with the 8-bit checkpoint, backward through the
linear layer's gradient and statistic and the norm's backward pass into the slices of the flat buffers, then the compressor and the
decoder on those.  Nothing waits between the calls; also captured and replayed.

Reference: the same step in 64 bits from the same inputs, its checkpoint rounded from the norm's output as the library stored it.
Bounds: of the calls, see their own tests (gradient 2e-6 of the products' magnitudes, statistic 1e-5, column sums (rows / 64 + 67) u); the
norm's backward pass is given the library's dy, mean and rstd."""
import numpy as np
import pytest
import torch

import oracle
import paper_1802_06058_b200 as vgc
from activations import U, activations, errors, quantised, workspace

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Layer:
    """Parameters [out x in weights | gain | bias] in one flat buffer; g and s like it."""

    def __init__(self, rows, n_in, n_out, dtype, seed):
        gen = torch.Generator("cuda").manual_seed(seed)
        new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.rows, self.n_in, self.n_out, self.dtype = rows, n_in, n_out, dtype
        n_w = n_in * n_out
        self.offsets = np.array([0, n_w, n_w + n_in, n_w + 2 * n_in], np.uint32)
        self.n = n = int(self.offsets[-1])
        self.flat = torch.randn(n, device="cuda", generator=gen) * 0.1
        self.flat[n_w:n_w + n_in] += 1
        self.g, self.s = new(n), new(n)
        part = lambda t: (t[:n_w].view(n_out, n_in), t[n_w:n_w + n_in], t[n_w + n_in:])  # noqa: E731
        self.W, self.gamma, self.beta = part(self.flat)
        self.gW, self.g_gamma, self.g_beta = part(self.g)
        self.sW, self.s_gamma, self.s_beta = part(self.s)
        self.x, self.delta = activations(rows, n_in, dtype, seed), errors(rows, n_out, dtype, seed + 1)
        self.y, self.dx, self.dy = new(rows, n_in, dtype=dtype), new(rows, n_in, dtype=dtype), new(rows, n_in, dtype=dtype)
        self.mean, self.rstd = new(rows), new(rows)
        self.checkpoint = new(vgc.vgc_checkpoint_bytes(rows, n_in), dtype=torch.uint8)
        self.ws_norm = workspace(vgc.vgc_layernorm_backward_workspace_bytes(rows, n_in)).t
        self.ws_w = workspace(vgc.vgc_wgrad_checkpoint_workspace_bytes(rows, n_in, n_out, dtype)).t
        self.ws_c = torch.empty(vgc.vgc_compress_workspace_bytes(n, 3), dtype=torch.uint8, device="cuda")
        self.r, self.v, self.u = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), new(n)
        self.offs = vgc.offsets_tensor(self.offsets)
        self.out, self.status = vgc.MessageBuffers(n, 3, n), torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(self):
        scale = dict(scale_g=1.0 / self.rows, scale_s=1.0 / self.rows ** 2)
        vgc.vgc_layernorm(self.x, self.gamma, self.beta, EPS, self.y, self.mean, self.rstd, checkpoint=self.checkpoint)
        torch.matmul(self.delta, self.W.to(self.dtype), out=self.dy)
        vgc.vgc_wgrad_checkpoint(self.checkpoint, self.delta, self.gW, self.sW, ws=self.ws_w, **scale)
        vgc.vgc_layernorm_backward(self.x, self.dy, self.gamma, self.mean, self.rstd, self.dx, self.g_gamma, self.g_beta, self.s_gamma,
                                   self.s_beta, ws=self.ws_norm, **scale)
        vgc.vgc_compress(self.g, self.s, self.r, self.v, self.offs, 1.0, 0.999, self.out, self.ws_c)
        vgc.vgc_decode_sum([self.out], self.offs, 1.0, self.u, self.status)

    def check(self, r, v):
        """r, v: the oracle's state, which goes on"""
        rows = self.rows
        d, q = self.delta.double(), quantised(self.y)
        assert bool(((self.gW.double() - d.t() @ q / rows).abs() <= 2e-6 / rows * (d.abs().t() @ q.abs())).all())
        want = d.square().t() @ q.square() / rows ** 2
        assert bool(((self.sW.double() - want).abs() <= 1e-5 * want).all())
        xh, dy = (self.x.double() - self.mean.double()[:, None]) * self.rstd.double()[:, None], self.dy.double()
        chain = (rows / 64 + 70) * U
        for term, g, s in ((dy * xh, self.g_gamma, self.s_gamma), (dy, self.g_beta, self.s_beta)):
            assert bool(((g.double() - term.sum(0) / rows).abs() <= chain / rows * term.abs().sum(0)).all())
            want = term.square().sum(0) / rows ** 2
            assert bool(((s.double() - want).abs() <= chain * want).all())
        message = oracle.compress(self.g.cpu().numpy(), self.s.cpu().numpy(), r, v, self.offsets, 1.0, 0.999)
        got = self.out.read()
        assert got["dev_status"] == 0 and got["nnz"] == message.nnz and np.array_equal(got["words"], message.words)
        assert message.nnz > 0
        u = np.zeros(self.n, np.float32)
        oracle.decode_accumulate([(message.words, message.group_exp)], self.offsets, 1.0, u)
        assert np.array_equal(self.u.cpu().numpy(), u)
        for ws in (self.ws_w,):
            assert int(ws[:4].view(torch.int32).item()) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n_in,n_out", [(512, 256, 384), (1000, 132, 260), (64, 1024, 512)])
def test_steps(rows, n_in, n_out, dtype):
    layer = Layer(rows, n_in, n_out, dtype, rows)
    r, v = np.zeros(layer.n, np.float32), np.zeros(layer.n, np.float32)
    for step in range(3):
        layer.x.copy_(activations(rows, n_in, dtype, 10 + step))
        layer.delta.copy_(errors(rows, n_out, dtype, 20 + step))
        layer.out.counters.zero_()
        layer.step()
        layer.check(r, v)


def test_captured_step():
    layer = Layer(512, 256, 384, torch.bfloat16, 1)
    layer.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.out.counters.zero_()
        layer.step()
    layer.r.zero_(), layer.v.zero_()
    r, v = np.zeros(layer.n, np.float32), np.zeros(layer.n, np.float32)
    for step in range(2):
        layer.x.copy_(activations(512, 256, torch.bfloat16, 30 + step))
        layer.delta.copy_(errors(512, 384, torch.bfloat16, 40 + step))
        graph.replay()
        layer.check(r, v)


def test_gradient_accumulated_over_micro_batches():
    """Two micro-batches added into g, their statistics into v, as a program without room for the whole batch does."""
    a, b = Layer(300, 132, 260, torch.bfloat16, 5), Layer(300, 132, 260, torch.bfloat16, 6)
    a.step(), b.step()
    total_g, total_s = torch.zeros(a.n, device="cuda"), torch.zeros(a.n, device="cuda")
    n_w = a.n_in * a.n_out
    for layer in (a, b):
        scale = dict(scale_g=1.0 / 300, scale_s=1.0 / 300 ** 2, accumulate_g=True, accumulate_s=True)
        vgc.vgc_wgrad_checkpoint(layer.checkpoint, layer.delta, total_g[:n_w].view(a.n_out, a.n_in), total_s[:n_w].view(a.n_out, a.n_in), ws=layer.ws_w,
                                 **scale)
        vgc.vgc_layernorm_backward(layer.x, layer.dy, layer.gamma, layer.mean, layer.rstd, layer.dx, total_g[n_w:n_w + a.n_in], total_g[n_w + a.n_in:],
                                   total_s[n_w:n_w + a.n_in], total_s[n_w + a.n_in:], ws=layer.ws_norm, **scale)
    assert torch.equal(total_g, a.g + b.g) and torch.equal(total_s, a.s + b.s)
