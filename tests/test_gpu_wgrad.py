"""A linear layer's gradient and statistic from its input's 8-bit checkpoint, against fp64 products of what the checkpoint stands
for.  Bounds, the library's own: the gradient within 2e-6 of the sum of the products' magnitudes, the statistic within 1e-5."""
import pytest
import torch

import paper_1802_06058_b200 as vgc
from activations import activations, checkpoint_of, errors, quantised, workspace
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]
SHAPES = [(1, 1, 1), (1, 16, 10), (3, 33, 5), (16, 128, 128), (17, 129, 127), (63, 64, 256), (64, 100, 130), (65, 784, 1024), (128, 784, 1024), (129, 257, 8),
          (200, 1000, 2051), (255, 512, 64), (256, 256, 256), (257, 130, 515), (500, 40, 4000), (1000, 2048, 136), (2049, 260, 264), (3001, 1000, 300),
          (5000, 128, 128), (10000, 20, 30), (16384, 64, 200), (700, 1536, 1544)]


def call(c, delta, n_in, scale_g=1.0, scale_s=1.0, acc_g=False, acc_s=False, old=None, want=(True, True)):
    rows, n_out = delta.shape
    g, S = (Guarded(n_in * n_out, fill=float("nan")) if w else None for w in want)
    if old is not None:
        for o, v in zip((g, S), old):
            if o is not None:
                o.t.copy_(v.reshape(-1))
    ws = workspace(vgc.vgc_wgrad_checkpoint_workspace_bytes(rows, n_in, n_out, delta.dtype))
    vgc.vgc_wgrad_checkpoint(c, delta, *(None if o is None else o.t.view(n_out, n_in) for o in (g, S)), scale_g=scale_g, scale_s=scale_s,
                             accumulate_g=acc_g, accumulate_s=acc_s, ws=ws.t)
    assert int(ws.t[:4].view(torch.int32).item()) == 0
    for b in (g, S, ws):
        if b is not None:
            b.check()
    return tuple(None if o is None else o.t.view(n_out, n_in) for o in (g, S))


def check(x, delta, scale_g, scale_s, g, S):
    d, q = delta.double(), quantised(x)
    if g is not None:
        assert bool(((g.double() - scale_g * (d.t() @ q)).abs() <= 2e-6 * scale_g * (d.abs().t() @ q.abs())).all())
    if S is not None:
        want = scale_s * (d.square().t() @ q.square())
        # The first part of a square is its nearest bf16, up to 2^-9 above it; so is the sum of first parts, before the later parts
        # are added: within 2^-8 of fp32's largest number the sum may be infinite, and beyond it has to be.
        most = torch.finfo(torch.float32).max
        assert bool(torch.isinf(S[want > most * (1 + 2.0 ** -24)]).all())
        near = (want > most * (1 - 2.0 ** -8)) & torch.isinf(S)
        assert bool((((S.double() - want).abs() <= 1e-5 * want) | near).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_gradient_and_statistic(rows, n_in, n_out, dtype):
    x, delta = activations(rows, n_in, torch.bfloat16, rows), errors(rows, n_out, dtype, rows + 1)
    c = checkpoint_of(x)
    g, S = call(c.t, delta, n_in, 1.0 / rows, 1.0 / rows ** 2)
    check(x, delta, 1.0 / rows, 1.0 / rows ** 2, g, S)
    g2, S2 = call(c.t, delta, n_in, 1.0 / rows, 1.0 / rows ** 2)
    assert torch.equal(g, g2) and torch.equal(S, S2)                                 # the same bits


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(64, 100, 130), (300, 784, 1024), (2000, 130, 515), (5000, 128, 128)])
def test_one_of_the_two_and_added(rows, n_in, n_out, dtype):
    x, delta = activations(rows, n_in, torch.float32, rows), errors(rows, n_out, dtype, rows + 1)
    c = checkpoint_of(x)
    g, S = call(c.t, delta, n_in, 0.5, 0.25)
    check(x, delta, 0.5, 0.25, g, S)
    only_g, only_S = call(c.t, delta, n_in, 0.5, 0.25, want=(True, False))[0], call(c.t, delta, n_in, 0.5, 0.25, want=(False, True))[1]
    assert torch.equal(only_g, g) and torch.equal(only_S, S)
    old = [torch.randn(n_out, n_in, device="cuda"), torch.rand(n_out, n_in, device="cuda")]
    for acc in ((True, True), (True, False), (False, True)):
        got = call(c.t, delta, n_in, 0.5, 0.25, *acc, old=old)
        for a, o, v, added in zip(got, old, (g, S), acc):
            assert torch.equal(a, o + v if added else v)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [12, 5, 0])
def test_sizes_of_the_values(dtype, top):
    """Errors from 1e-12 to 1e12 (1e5, 1) beside one another, activations likewise (a row's block of 32 shares its scale), zero rows and
    columns, the last row alone not zero."""
    rows, n_in, n_out = 600, 320, 200
    x, delta = activations(rows, n_in, torch.float32, 1), errors(rows, n_out, torch.float32, 2)
    torch.manual_seed(top)
    x *= torch.logspace(-12, top, rows, device="cuda")[torch.randperm(rows, device="cuda")][:, None]
    delta *= torch.logspace(-9, top, rows, device="cuda")[torch.randperm(rows, device="cuda")][:, None]
    x[:, 64:96] = 0
    delta[:, 7] = 0
    delta[:-1, 9] = 0
    delta[-1, 9] = 1
    delta = delta.to(dtype)
    c = checkpoint_of(x)
    g, S = call(c.t, delta, n_in)
    check(x, delta, 1.0, 1.0, g, S)
    assert bool((S[:, 64:96] == 0).all()) and bool((g[7] == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(40, 100, 60), (400, 256, 384)])
def test_not_finite_values_stay_in_their_row_and_column(rows, n_in, n_out, dtype):
    x, delta = activations(rows, n_in, torch.float32, 1), errors(rows, n_out, dtype, 2)
    x[3, 50], x[rows - 1, 51] = float("nan"), float("inf")
    delta[5, 11], delta[6, 12] = float("inf"), float("nan")
    c = checkpoint_of(x)
    for got in call(c.t, delta, n_in):
        odd = ~torch.isfinite(got)
        assert bool(odd[:, 50].all()) and bool(odd[:, 51].all()) and bool(odd[11].all()) and bool(odd[12].all())
        odd[:, 50:52] = False
        odd[11:13] = False
        assert not bool(odd.any())


def test_no_rows_and_refusals():
    g, S = torch.ones(4, 8, device="cuda"), torch.ones(4, 8, device="cuda")
    empty = torch.zeros(0, dtype=torch.uint8, device="cuda")
    vgc.vgc_wgrad_checkpoint(empty, torch.zeros(0, 4, device="cuda"), g, S, accumulate_s=True)
    assert bool((g == 0).all()) and bool((S == 1).all())
    d = torch.zeros(3, 4, device="cuda")
    c = torch.zeros(vgc.vgc_checkpoint_bytes(3, 8), dtype=torch.uint8, device="cuda")
    with pytest.raises(vgc.VgcError) as err:
        vgc.vgc_wgrad_checkpoint(c, d, g, S)                                         # no workspace
    assert err.value.status == 3
    ws = workspace(vgc.vgc_wgrad_checkpoint_workspace_bytes(3, 8, 4, torch.float32)).t
    for bad in ((c[:-1], d, g, S), (c, d[:, :3].contiguous(), g, S), (c, d, g, S.view(8, 4)), (c, d, None, None), (c, d.t(), g, S)):
        with pytest.raises(ValueError):
            vgc.vgc_wgrad_checkpoint(*bad, ws=ws)
    for bad in ((c, d.half(), g, S), (c, d, g.double(), S), (c.to(torch.int8), d, g, S)):
        with pytest.raises(TypeError):
            vgc.vgc_wgrad_checkpoint(*bad, ws=ws)
    with pytest.raises(TypeError):
        vgc.vgc_wgrad_checkpoint_workspace_bytes(3, 8, 4, torch.float16)


def test_streams_and_replay():
    """Two captured calls that share a workspace, replayed in turn on other values; a call on a side stream."""
    rows, n_in, n_out = 3000, 256, 264
    delta = errors(rows, n_out, torch.bfloat16, 1)
    c = torch.zeros(vgc.vgc_checkpoint_bytes(rows, n_in), dtype=torch.uint8, device="cuda")
    ws = workspace(vgc.vgc_wgrad_checkpoint_workspace_bytes(rows, n_in, n_out)).t
    g, S = ([torch.empty(n_out, n_in, device="cuda") for _ in range(2)] for _ in range(2))
    vgc.vgc_wgrad_checkpoint(c, delta, g[0], S[0], ws=ws)
    graphs = []
    for k in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            vgc.vgc_wgrad_checkpoint(c, delta, g[k], S[k], ws=ws)
    for seed in (3, 4, 5):
        x = activations(rows, n_in, torch.bfloat16, seed)
        vgc.vgc_checkpoint_store(x, c)
        delta.copy_(errors(rows, n_out, torch.bfloat16, seed))
        graphs[seed % 2].replay()
        check(x, delta, 1.0, 1.0, g[seed % 2], S[seed % 2])
    side = torch.cuda.Stream()
    g[0].zero_()
    side.wait_stream(torch.cuda.current_stream())
    vgc.vgc_wgrad_checkpoint(c, delta, g[0], S[0], ws=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check(x, delta, 1.0, 1.0, g[0], S[0])
