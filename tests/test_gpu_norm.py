"""Layer norm, its backward pass and the sums of gain and bias against the definitions in 64 bits.

Tolerances, with u = 2^-24.  A sum over a row passes at most 8 (16 beyond 8192 features) additions in a lane, 5 between lanes, 5
between warps: fewer than 32 roundings, so it is off by at most 32 u of the sum of magnitudes.
  forward   mean: 32 u mean|x|, and u of itself.  rstd: the squares' sum has 32 u, twice the relative error of d = x - mean (rounding u; the
            mean's own error enters squared), its division and eps 2 u; half of that in the root, and u each for root and
            division: 24 u.  y = d * rstd * gamma + beta: d's error (mean's + u |d|) times rstd |gamma|, (24 + 3) u |xh gamma|, u |y|.
  backward  mean and rstd are inputs.  xh: 2 u.  w: u.  Their means: 36 u of the mean magnitudes (products included).
  sums      a column's chain of additions is at most rows / 64 in a block and 64 behind it (tests of few rows stay far below)
Every result in bf16 is rounded once more: half an ulp."""
import pytest
import torch

import paper_1802_06058_b200 as vgc
from activations import U, activations, checkpoint_of, errors, half_ulp, workspace
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
EPS = 1e-5
DTYPES = [torch.float32, torch.bfloat16]
SHAPES = [(1, 1), (3, 7), (2, 32), (5, 255), (4, 256), (300, 257), (16, 784), (1000, 1000), (257, 1001), (2, 1032), (700, 2048), (35, 2056), (40, 3001),
          (9, 4096), (5, 4100), (20, 5001), (7, 8192), (3, 8200), (5, 12289), (2, 16384), (5000, 64), (3000, 520), (40000, 24)]


def vectors(features, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    return 1 + 0.3 * torch.randn(features, device="cuda", generator=gen), 0.2 * torch.randn(features, device="cuda", generator=gen)


def forward(x, gamma, beta, checkpoint=False, eps=EPS, y=None):
    rows, C = x.shape
    y = Guarded(rows * C, x.dtype) if y is None else y
    mean, rstd = Guarded(rows), Guarded(rows)
    c = Guarded(vgc.vgc_checkpoint_bytes(rows, C), torch.uint8) if checkpoint else None
    vgc.vgc_layernorm(x, gamma, beta, eps, y.t.view(rows, C), mean.t, rstd.t, checkpoint=c.t if c else None)
    for b in (y, mean, rstd, c):
        if b is not None:
            b.check()
    return y.t.view(rows, C), mean.t, rstd.t, c


def check_forward(x, gamma, beta, y, mean, rstd, eps=EPS):
    wide, C = x.double(), x.shape[1]
    g = torch.ones(C, device="cuda", dtype=torch.float64) if gamma is None else gamma.double()
    b = torch.zeros(C, device="cuda", dtype=torch.float64) if beta is None else beta.double()
    m = wide.mean(1, keepdim=True)
    d = wide - m
    r = 1 / (d.square().mean(1, keepdim=True) + eps).sqrt()
    off = U * (32 * wide.abs().mean(1, keepdim=True) + m.abs())
    assert bool(((mean.double()[:, None] - m).abs() <= off).all())
    # the mean's error moves the squares' mean by its square
    off_r = r * (24 * U + (off * r).square())
    assert bool(((rstd.double()[:, None] - r).abs() <= off_r).all())
    want = d * r * g + b
    tol = (off + U * d.abs()) * r * g.abs() + (d * r * g).abs() * (27 * U + (off * r).square()) + U * want.abs()
    tol = tol + half_ulp(x.dtype) * (want.abs() + tol) * (x.dtype != torch.float32)
    assert bool(((y.double() - want).abs() <= tol * 1.01 + 1e-45).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,features", SHAPES)
def test_forward(rows, features, dtype):
    x = activations(rows, features, dtype, rows * features)
    gamma, beta = vectors(features, rows)
    y, mean, rstd, c = forward(x, gamma, beta, checkpoint=True)
    check_forward(x, gamma, beta, y, mean, rstd)
    again = checkpoint_of(y)                                      # the same bits as a checkpoint of what was stored
    assert torch.equal(c.t, again.t)
    alone, mean2, rstd2, _ = forward(x, gamma, beta)
    assert torch.equal(alone, y) and torch.equal(mean2, mean) and torch.equal(rstd2, rstd)


@pytest.mark.parametrize("features", [40, 1001, 9000])
def test_forward_without_gain_or_bias_and_in_place(features):
    x = activations(11, features, torch.float32, 1)
    gamma, beta = vectors(features, 2)
    for g, b in ((None, None), (gamma, None), (None, beta)):
        y, mean, rstd, _ = forward(x, g, b)
        check_forward(x, g, b, y, mean, rstd)
    want = forward(x, gamma, beta)[0].clone()
    z = x.clone()
    mean, rstd = torch.empty(11, device="cuda"), torch.empty(11, device="cuda")
    vgc.vgc_layernorm(z, gamma, beta, EPS, z, mean, rstd)
    assert torch.equal(z, want)


def test_forward_far_from_zero_and_constant_rows():
    """A mean of 1000 deviations: a variance from the sum of squares would have no bit left.  A constant row: deviations are the
    mean's own rounding."""
    x = activations(64, 2048, torch.float32, 9) * 1e-3 + 1000
    x[5] = 3.0
    gamma, beta = vectors(2048, 3)
    y, mean, rstd, _ = forward(x, gamma, beta)
    check_forward(x, gamma, beta, y, mean, rstd)


def test_forward_not_finite():
    """Infinities and NaN stay in their row; the checkpoint of such a row is NaN."""
    x = activations(9, 300, torch.bfloat16, 4)
    x[2, 7], x[6, 200] = float("inf"), float("nan")
    gamma, beta = vectors(300, 4)
    y, mean, rstd, c = forward(x, gamma, beta, checkpoint=True)
    assert bool(torch.isnan(y[[2, 6]]).all())
    rest = [0, 1, 3, 4, 5, 7, 8]
    check_forward(x[rest], gamma, beta, y[rest], mean[rest], rstd[rest])
    back = torch.empty(9, 300, device="cuda")
    vgc.vgc_checkpoint_load(c.t, back)
    assert torch.equal(torch.isnan(back).all(1), torch.isnan(y).all(1)) and not bool(torch.isnan(back[rest]).any())


def backward(x, dy, gamma, mean, rstd, per=1, scale_g=1.0, scale_s=1.0, acc_g=False, acc_s=False, old=None, dx=None):
    rows, C = x.shape
    dx = Guarded(rows * C, x.dtype) if dx is None else dx
    out = [Guarded(C, fill=float("nan")) for _ in range(4)]
    if old is not None:
        for o, v in zip(out, old):
            o.t.copy_(v)
    ws = workspace(vgc.vgc_layernorm_backward_workspace_bytes(rows, C, per))
    vgc.vgc_layernorm_backward(x, dy, gamma, mean, rstd, dx.t.view(rows, C), *[o.t for o in out], scale_g=scale_g, scale_s=scale_s,
                               accumulate_g=acc_g, accumulate_s=acc_s, rows_per_example=per, ws=ws.t)
    for b in [dx, ws] + out:
        b.check()
    return dx.t.view(rows, C), [o.t for o in out]


def statistics(x):
    m = x.double().mean(1)
    return m.float(), (x.double().var(1, unbiased=False) + EPS).rsqrt().float()


def check_backward(x, dy, gamma, mean, rstd, per, scale_g, scale_s, dx, out):
    rows, C = x.shape
    g = torch.ones(C, device="cuda", dtype=torch.float64) if gamma is None else gamma.double()
    r, d = rstd.double()[:, None], dy.double()
    xh = (x.double() - mean.double()[:, None]) * r
    w = d * g
    first, second = w.mean(1, keepdim=True), (w * xh).mean(1, keepdim=True)
    want = r * (w - first - xh * second)
    tol = U * r * (6 * w.abs() + 40 * w.abs().mean(1, keepdim=True) + xh.abs() * (6 * second.abs() + 40 * (w * xh).abs().mean(1, keepdim=True)))
    tol = tol + half_ulp(x.dtype) * (want.abs() + tol) * (x.dtype != torch.float32)
    assert bool(((dx.double() - want).abs() <= tol * 1.01 + 1e-45).all())
    chain = -(-rows // 64) + 64
    n = rows // per
    for q, term in ((0, d * xh), (1, d)):
        part = term.view(n, per, C)
        sample, size = part.sum(1), part.abs().sum(1)
        off = (chain + 3) * U * size                               # of a sample's sum
        got = out[q].double()
        assert bool(((got - scale_g * sample.sum(0)).abs() <= abs(scale_g) * (off.sum(0) + 2 * U * sample.abs().sum(0)) * 1.01 + 1e-45).all())
        tol_s = scale_s * ((2 * sample.abs() * off + off.square()).sum(0) + (chain + 3) * U * sample.square().sum(0))
        assert bool(((out[2 + q].double() - scale_s * sample.square().sum(0)).abs() <= tol_s * 1.01 + 1e-45).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,features", SHAPES)
def test_backward(rows, features, dtype):
    x, dy = activations(rows, features, dtype, rows + 1), errors(rows, features, dtype, rows + 2)
    gamma, _ = vectors(features, rows)
    mean, rstd = statistics(x)
    dx, out = backward(x, dy, gamma, mean, rstd, scale_g=1.0 / rows, scale_s=1.0 / rows ** 2)
    check_backward(x, dy, gamma, mean, rstd, 1, 1.0 / rows, 1.0 / rows ** 2, dx, out)
    dx2, out2 = backward(x, dy, gamma, mean, rstd, scale_g=1.0 / rows, scale_s=1.0 / rows ** 2)
    assert torch.equal(dx, dx2) and all(torch.equal(a, b) for a, b in zip(out, out2))            # the same bits


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("samples,per,features", [(1, 2, 7), (1, 5000, 260), (3, 197, 1280), (64, 197, 384), (2000, 2, 128), (5000, 3, 36), (2500, 4, 1001),
                                                  (700, 7, 2048), (7, 300, 4100), (600, 5, 6000), (2, 33, 8192), (3, 65, 9000), (400, 3, 12000), (1, 1, 50)])
def test_samples_of_several_rows(samples, per, features, dtype):
    rows = samples * per
    x, dy = activations(rows, features, dtype, per), errors(rows, features, dtype, per + 2)
    gamma, _ = vectors(features, per)
    mean, rstd = statistics(x)
    dx, out = backward(x, dy, gamma, mean, rstd, per, 1.0 / samples, 1.0 / samples ** 2)
    check_backward(x, dy, gamma, mean, rstd, per, 1.0 / samples, 1.0 / samples ** 2, dx, out)


@pytest.mark.parametrize("rows,per,features", [(300, 1, 257), (300, 100, 257), (2000, 2, 128), (40, 1, 8200)])
def test_added_is_one_fp32_addition(rows, per, features):
    x, dy = activations(rows, features, torch.bfloat16, 1), errors(rows, features, torch.bfloat16, 2)
    mean, rstd = statistics(x)
    old = [torch.rand(features, device="cuda") for _ in range(4)]
    dx, new = backward(x, dy, None, mean, rstd, per, 0.5, 0.25)
    dx2, added = backward(x, dy, None, mean, rstd, per, 0.5, 0.25, acc_g=True, acc_s=True, old=old)
    assert torch.equal(dx, dx2)
    assert all(torch.equal(a, o + v) for a, o, v in zip(added, old, new))
    _, half = backward(x, dy, None, mean, rstd, per, 0.5, 0.25, acc_g=False, acc_s=True, old=old)
    assert all(torch.equal(a, v) for a, v in zip(half, new[:2] + added[2:]))


@pytest.mark.parametrize("features", [512, 1001, 8200])
def test_in_place_missing_outputs_and_slices_of_a_flat_buffer(features):
    """dx over dy and over x; only some sums wanted; vectors that start on 4 bytes."""
    rows = 50
    x, dy = activations(rows, features, torch.float32, 3), errors(rows, features, torch.float32, 4)
    flat = torch.randn(3 * features + 1, device="cuda")
    gamma = flat[1:features + 1]
    mean, rstd = statistics(x)
    want, sums = backward(x, dy, gamma.clone(), mean, rstd)
    ws = workspace(vgc.vgc_layernorm_backward_workspace_bytes(rows, features, 1)).t
    for target in ("dy", "x"):
        a, b = x.clone(), dy.clone()
        g = torch.full((3 * features + 2,), 7.0, device="cuda")
        vgc.vgc_layernorm_backward(a, b, gamma, mean, rstd, b if target == "dy" else a, g_gamma=g[1:features + 1],
                                   s_beta=g[features + 1:2 * features + 1], ws=ws)
        assert torch.equal(b if target == "dy" else a, want)
        assert torch.equal(g[1:features + 1], sums[0]) and torch.equal(g[features + 1:2 * features + 1], sums[3])
        assert bool((g[2 * features + 1:] == 7).all()) and float(g[0]) == 7
    only = torch.empty_like(x)
    vgc.vgc_layernorm_backward(x, dy, gamma, mean, rstd, only, ws=ws)
    assert torch.equal(only, want)


def test_gradients_against_differences():
    """f = sum(y * v): the backward pass against (f(x + h) - f(x - h)) / 2h in 64 bits."""
    rows, C, h = 4, 24, 1e-5
    x, v = activations(rows, C, torch.float32, 8), errors(rows, C, torch.float32, 9)
    gamma, beta = vectors(C, 8)
    mean, rstd = statistics(x)
    dx, out = backward(x, v, gamma, mean, rstd)

    def f(x, gamma, beta):
        d = x - x.mean(1, keepdim=True)
        return float((v.double() * (d * (d.square().mean(1, keepdim=True) + EPS).rsqrt() * gamma + beta)).sum())

    args = [x.double(), gamma.double(), beta.double()]
    for which, got in ((0, dx), (1, out[0]), (2, out[1])):
        got = got.reshape(-1)
        scale = float(got.abs().max())
        for i in range(0, got.numel(), 5):
            values = []
            for sign in (1, -1):
                moved = [a.clone() for a in args]
                moved[which].view(-1)[i] += sign * h
                values.append(f(*moved))
            # the difference's own error is of order h^2; fp32 in the pass: 100 u of the largest gradient
            assert abs((values[0] - values[1]) / (2 * h) - float(got[i])) <= 1e-5 * scale


@pytest.mark.parametrize("features,per", [(1000, 1), (1000, 25), (9000, 1)])
def test_streams_and_replay(features, per):
    """A captured forward and backward pass replayed on other values, and both on a side stream beside work on another."""
    rows = 200
    x, dy = activations(rows, features, torch.bfloat16, 1), errors(rows, features, torch.bfloat16, 2)
    gamma, beta = vectors(features, 1)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    out = [torch.empty(features, device="cuda") for _ in range(4)]
    ws = workspace(vgc.vgc_layernorm_backward_workspace_bytes(rows, features, per)).t
    c = torch.empty(vgc.vgc_checkpoint_bytes(rows, features), dtype=torch.uint8, device="cuda")

    def both(stream=None):
        vgc.vgc_layernorm(x, gamma, beta, EPS, y, mean, rstd, checkpoint=c, stream=stream)
        vgc.vgc_layernorm_backward(x, dy, gamma, mean, rstd, dx, *out, rows_per_example=per, ws=ws, stream=stream)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (3, 4):
        x.copy_(activations(rows, features, torch.bfloat16, seed))
        dy.copy_(errors(rows, features, torch.bfloat16, seed))
        graph.replay()
        check_forward(x, gamma, beta, y, mean, rstd)
        check_backward(x, dy, gamma, mean, rstd, per, 1.0, 1.0, dx, out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in [y, dx, mean, rstd] + out:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    torch.cuda.current_stream().wait_stream(side)
    check_backward(x, dy, gamma, mean, rstd, per, 1.0, 1.0, dx, out)


def test_no_rows_and_refusals():
    x = torch.zeros(0, 8, device="cuda")
    none = torch.zeros(0, device="cuda")
    out = [torch.ones(8, device="cuda") for _ in range(4)]
    vgc.vgc_layernorm(x, None, None, EPS, x, none, none)
    vgc.vgc_layernorm_backward(x, x, None, none, none, x, *out, accumulate_s=True)
    assert all(bool((o == v).all()) for o, v in zip(out, (0, 0, 1, 1)))
    x, m = torch.zeros(6, 8, device="cuda"), torch.zeros(6, device="cuda")
    with pytest.raises(ValueError):
        vgc.vgc_layernorm_backward(x, x, None, m, m, x, rows_per_example=4)
    with pytest.raises(vgc.VgcError):
        vgc.vgc_layernorm_backward(x, x, None, m, m, x)                              # no workspace
    with pytest.raises(ValueError):
        vgc.vgc_layernorm(x, m, None, EPS, x, m, m)
    with pytest.raises(ValueError):
        vgc.vgc_layernorm(x, None, None, EPS, x.bfloat16(), m, m)
    with pytest.raises(TypeError):
        vgc.vgc_layernorm(x.half(), None, None, EPS, x.half(), m, m)
    with pytest.raises(vgc.VgcError):
        vgc.vgc_layernorm(x, None, None, -1.0, x, m, m)
    wide, m = torch.zeros(1, 16388, device="cuda"), torch.zeros(1, device="cuda")
    with pytest.raises(vgc.VgcError) as err:
        vgc.vgc_layernorm(wide, None, None, EPS, wide, m, m)
    assert err.value.status == 2


@pytest.mark.parametrize("rows,features", [(700, 1001), (50, 257), (3, 7), (90, 4099)])
def test_in_place_rows_off_16_bytes(rows, features):
    """bf16 rows that share 16-byte pieces with their neighbours: y over x, dx over dy, dx over x, for many rows in flight."""
    x, dy = activations(rows, features, torch.bfloat16, 1), errors(rows, features, torch.bfloat16, 2)
    gamma, beta = vectors(features, 5)
    want, mean, rstd, _ = forward(x, gamma, beta)
    z, m, r = x.clone(), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    vgc.vgc_layernorm(z, gamma, beta, EPS, z, m, r)
    assert torch.equal(z, want) and torch.equal(m, mean) and torch.equal(r, rstd)
    want, sums = backward(x, dy, gamma, mean, rstd)
    ws = workspace(vgc.vgc_layernorm_backward_workspace_bytes(rows, features, 1)).t
    for over_dy in (True, False):
        a, b, out = x.clone(), dy.clone(), [torch.empty(features, device="cuda") for _ in range(4)]
        vgc.vgc_layernorm_backward(a, b, gamma, mean, rstd, b if over_dy else a, *out, ws=ws)
        assert torch.equal(b if over_dy else a, want) and all(torch.equal(p, q) for p, q in zip(out, sums))
