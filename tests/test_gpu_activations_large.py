"""Activations of more than 2^31 elements (4.9 GB in bf16): offsets beyond 32 bits in every call; and calls side by side on two
streams, results that begin on 4 bytes."""
import pytest
import torch

import paper_1802_06058_b200 as vgc
from activations import U, activations, checkpoint_of, errors, half_ulp, quantised, workspace
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
ROWS, C, EPS = 150_000, 16_384, 1e-5


def test_offsets_beyond_32_bits():
    gen = torch.Generator("cuda").manual_seed(1)
    x = torch.empty(ROWS, C, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    assert x.numel() > 2 ** 31
    c = torch.empty(vgc.vgc_checkpoint_bytes(ROWS, C), dtype=torch.uint8, device="cuda")
    back, y = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(ROWS, device="cuda"), torch.empty(ROWS, device="cuda")
    vgc.vgc_layernorm(x, None, None, EPS, y, mean, rstd, checkpoint=c)
    vgc.vgc_checkpoint_load(c, back)
    places = [slice(0, 3), slice(131_070, 131_075), slice(ROWS - 3, ROWS)]            # 2^31 elements lie in row 131072
    for at in places:
        wide = x[at].double()
        d = wide - wide.mean(1, keepdim=True)
        want = d * (d.square().mean(1, keepdim=True) + EPS).rsqrt()
        # the tolerance of layer norm's own tests with |x| < 8, deviations near 1: 32 + 27 + 1 u of the values, half an ulp
        assert bool(((y[at].double() - want).abs() <= 64 * U * (1 + want.abs()) + half_ulp(torch.bfloat16) * want.abs()).all())
        assert torch.equal(back[at].double(), quantised(y[at]))
    stored = torch.empty_like(c)
    vgc.vgc_checkpoint_store(y, stored)
    assert torch.equal(stored, c)
    # a linear layer's pair over all rows: errors that are zero but in a few rows on either side of the border
    delta = torch.zeros(ROWS, 8, dtype=torch.bfloat16, device="cuda")
    for at in places:
        delta[at] = torch.randn(delta[at].shape, device="cuda", generator=gen).bfloat16()
    g, S = torch.empty(8, C, device="cuda"), torch.empty(8, C, device="cuda")
    ws = workspace(vgc.vgc_wgrad_checkpoint_workspace_bytes(ROWS, C, 8)).t
    vgc.vgc_wgrad_checkpoint(c, delta, g, S, ws=ws)
    d, q = torch.cat([delta[at] for at in places]).double(), torch.cat([back[at] for at in places]).double()
    assert bool(((g.double() - d.t() @ q).abs() <= 2e-6 * (d.abs().t() @ q.abs())).all())
    want = d.square().t() @ q.square()
    assert bool(((S.double() - want).abs() <= 1e-5 * want).all()) and int(ws[:4].view(torch.int32).item()) == 0
    # backward, dx over y (its dy): rows checked, and sums of rows that are zero elsewhere
    y.zero_()
    for at in places:
        y[at] = torch.randn(y[at].shape, device="cuda", generator=gen).bfloat16()
    dy = torch.cat([y[at] for at in places]).double()
    sums = [torch.empty(C, device="cuda") for _ in range(4)]
    ws = workspace(vgc.vgc_layernorm_backward_workspace_bytes(ROWS, C)).t
    vgc.vgc_layernorm_backward(x, y, None, mean, rstd, y, *sums, ws=ws)
    m, r = (torch.cat([t[at] for at in places]).double()[:, None] for t in (mean, rstd))
    xh = (torch.cat([x[at] for at in places]).double() - m) * r
    want = r * (dy - dy.mean(1, keepdim=True) - xh * (dy * xh).mean(1, keepdim=True))
    got = torch.cat([y[at] for at in places]).double()
    assert bool(((got - want).abs() <= 128 * U * r * (1 + dy.abs() + xh.abs()) + half_ulp(torch.bfloat16) * want.abs() * 1.01).all())
    for s, term in zip(sums, (dy * xh, dy, (dy * xh).square(), dy.square())):
        assert bool(((s.double() - term.sum(0)).abs() <= 16 * U * term.abs().sum(0)).all())      # eleven rows: at most 11 + 3 roundings


def test_two_streams_and_results_on_4_bytes():
    """Calls side by side, each with its workspace; g and S begin one element into a buffer."""
    rows, n_in, n_out = 2000, 300, 260
    streams = [torch.cuda.Stream() for _ in range(2)]
    jobs = []
    for k in range(2):
        x, delta = activations(rows, n_in, torch.bfloat16, k), errors(rows, n_out, torch.bfloat16, 10 + k)
        n = n_in * n_out
        g, S = Guarded(n + 1, fill=3.0), Guarded(n + 1, fill=3.0)
        jobs.append((x, delta, checkpoint_of(x), g, S, workspace(vgc.vgc_wgrad_checkpoint_workspace_bytes(rows, n_in, n_out))))
    torch.cuda.synchronize()
    for _ in range(5):
        for (x, delta, c, g, S, ws), stream in zip(jobs, streams):
            vgc.vgc_wgrad_checkpoint(c.t, delta, g.t[1:].view(n_out, n_in), S.t[1:].view(n_out, n_in), ws=ws.t, stream=stream)
    torch.cuda.synchronize()
    for x, delta, c, g, S, ws in jobs:
        d, q = delta.double(), quantised(x)
        assert float(g.t[0]) == 3 and float(S.t[0]) == 3 and int(ws.t[:4].view(torch.int32).item()) == 0
        for b in (g, S, ws):
            b.check()
        assert bool(((g.t[1:].view(n_out, n_in).double() - d.t() @ q).abs() <= 2e-6 * (d.abs().t() @ q.abs())).all())
        want = d.square().t() @ q.square()
        assert bool(((S.t[1:].view(n_out, n_in).double() - want).abs() <= 1e-5 * want).all())
