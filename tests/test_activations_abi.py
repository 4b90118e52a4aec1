"""Layer norm, 8-bit checkpoints and the linear layer's gradient and statistic: sizes and refusals, before anything is enqueued
(no GPU needed)."""
import ctypes

import pytest
import torch

import paper_1802_06058_b200 as vgc

FAKE, ODD, HALF = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), ctypes.c_void_p(0x1002)    # never dereferenced


@pytest.fixture(scope="module")
def lib():
    vgc.build()
    return vgc.load_library()


@pytest.mark.parametrize("rows,features,want", [(1, 1, 128 + 128 * 4), (128, 128, 128 * 128 + 128 * 4), (129, 129, 129 * 256 + 256 * 8), (0, 5, 0), (5, 0, 0), (-1, 5, 0),
                                                (2 ** 31 - 1, 8, 0), (1 << 20, 1 << 14, (1 << 34) + (1 << 29)), (8, (1 << 24) + 1, 0)])
def test_checkpoint_bytes(lib, rows, features, want):
    assert vgc.vgc_checkpoint_bytes(rows, features) == want


def test_checkpoint_refusals(lib):
    store = lambda x=FAKE, t=0, rows=4, features=8, c=FAKE: lib.vgc_checkpoint_store(x, t, rows, features, c, None)  # noqa: E731
    load = lambda x=FAKE, t=0, rows=4, features=8, c=FAKE: lib.vgc_checkpoint_load(c, rows, features, x, t, None)    # noqa: E731
    for call in (store, load):
        assert call(rows=0) == 0 and call(features=0) == 0
        for bad in (dict(x=None), dict(c=None), dict(x=ODD), dict(c=ODD), dict(t=2), dict(rows=-1), dict(features=-1), dict(rows=2 ** 31 - 1)):
            assert call(**bad) == 1, bad


def test_layernorm_refusals(lib):
    def forward(x=FAKE, t=1, gamma=FAKE, beta=FAKE, rows=4, features=8, eps=1e-5, y=FAKE, mean=FAKE, rstd=FAKE, c=None):
        return lib.vgc_layernorm(x, t, gamma, beta, rows, features, eps, y, mean, rstd, c, None)
    assert forward(rows=0, x=None) == 0 and forward(features=0) == 0
    for bad in (dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(x=ODD), dict(y=ODD), dict(c=ODD), dict(gamma=HALF), dict(beta=HALF), dict(t=-1),
                dict(rows=-1), dict(features=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rows=2 ** 31 - 1)):
        assert forward(**bad) == 1, bad
    assert forward(features=16385) == 2

    def backward(x=FAKE, dy=FAKE, t=1, gamma=None, mean=FAKE, rstd=FAKE, rows=4, features=8, per=1, sg=1.0, ss=1.0, dx=FAKE, out=FAKE, ws=FAKE, nbytes=1 << 40):
        return lib.vgc_layernorm_backward(x, dy, t, gamma, mean, rstd, rows, features, per, sg, ss, 0, 0, dx, out, out, out, out, ws, nbytes, None)
    assert backward(features=0) == 0
    for bad in (dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(x=ODD), dict(dy=ODD), dict(dx=ODD), dict(out=HALF), dict(gamma=HALF),
                dict(per=0), dict(per=3), dict(per=-1), dict(t=7), dict(rows=-4), dict(sg=float("nan")), dict(ss=float("nan"))):
        assert backward(**bad) == 1, bad
    assert backward(features=16385) == 2
    for bad in (dict(ws=None), dict(nbytes=16), dict(ws=ODD)):
        assert backward(**bad) == 3, bad


@pytest.mark.parametrize("rows,features,per", [(1, 1, 1), (128, 784, 1), (16384, 4096, 1), (12608, 1280, 197), (1 << 20, 64, 2), (100, 16384, 10), (7, 9000, 7)])
def test_backward_workspace(lib, rows, features, per):
    """Partial sums of the blocks: at most two blocks an SM of four sums a feature, or two sums for each piece of a sample, of which
    there are at most that many and one for each sample."""
    n = vgc.vgc_layernorm_backward_workspace_bytes(rows, features, per)
    most = 8 * rows + 512 + 4 * features * (4 * 296 if per == 1 else max(4 * 296, 2 * (2 * 296 + rows // per)))
    assert 0 < n <= most and n % 256 == 0
    assert vgc.vgc_layernorm_backward_workspace_bytes(rows, features, rows + 1) == 0


def test_wgrad_refusals(lib):
    def call(c=FAKE, d=FAKE, t=1, rows=4, n_in=8, n_out=8, sg=1.0, ss=1.0, g=FAKE, S=FAKE, ws=FAKE, nbytes=1 << 40):
        return lib.vgc_wgrad_checkpoint(c, d, t, rows, n_in, n_out, sg, ss, 0, 1, g, S, ws, nbytes, None)
    assert call(n_in=0) == 0 and call(n_out=0) == 0
    assert call(rows=0, c=None, d=None, g=None) == 0                                  # nothing to add
    for bad in (dict(c=None), dict(d=None), dict(c=ODD), dict(d=ODD), dict(g=None, S=None), dict(g=HALF), dict(S=HALF), dict(t=2), dict(rows=-1), dict(n_in=-1),
                dict(n_out=-1), dict(sg=float("nan")), dict(ss=float("nan")), dict(rows=2 ** 31 - 1)):
        assert call(**bad) == 1, bad
    for bad in (dict(ws=None), dict(nbytes=16), dict(ws=ODD)):
        assert call(**bad) == 3, bad
    assert vgc.vgc_wgrad_checkpoint_workspace_bytes(0, 8, 8) == 0
    assert vgc.vgc_wgrad_checkpoint_workspace_bytes(100, 8, 8, torch.float32) >= 256


def test_binding_refuses_cpu_tensors(lib):
    x, m, c = torch.zeros(2, 8), torch.zeros(2), torch.zeros(640, dtype=torch.uint8)
    for call in (lambda: vgc.vgc_checkpoint_store(x, c), lambda: vgc.vgc_checkpoint_load(c, x), lambda: vgc.vgc_layernorm(x, None, None, 0.0, x, m, m),
                 lambda: vgc.vgc_layernorm_backward(x, x, None, m, m, x), lambda: vgc.vgc_wgrad_checkpoint(c, x, torch.zeros(8, 8), None)):
        with pytest.raises(TypeError):
            call()
