"""8-bit checkpoints: every code bit for bit against the definition in 64 bits, the layout, the values read back, NaN, infinities
and the ends of the range."""
import pytest
import torch

import paper_1802_06058_b200 as vgc
from activations import activations, checkpoint_of, layout, quantised
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
SHAPES = [(1, 1), (1, 32), (3, 31), (2, 33), (5, 127), (129, 128), (7, 130), (64, 256), (33, 257), (128, 264), (17, 1001), (300, 1024),
          (2, 4100), (1, 16384), (1000, 48), (40000, 20), (6000, 1000)]


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=12345.0), torch.nan_to_num(b.double(), nan=12345.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,features", SHAPES)
def test_values(rows, features, dtype):
    x = activations(rows, features, dtype, rows + features)
    x[rows // 2] = 0
    want = quantised(x)
    c = checkpoint_of(x)
    c.check("checkpoint")
    codes, scales = layout(c.t, rows, features)
    assert bool((codes[:, features:] == 0).all()) and bool((scales[:, rows:] == 0).all())
    assert int(scales.max()) < 255 and int(scales[:, :rows].min()) >= 1
    for out in (torch.float32, torch.bfloat16):
        back = Guarded(rows * features, out)
        vgc.vgc_checkpoint_load(c.t, back.t.view(rows, features))
        back.check("restored values")
        assert same(back.t.view(rows, features), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("features", [96, 97])
def test_ends_of_the_range(features, dtype):
    """Largest and smallest numbers, subnormals, zeros of either sign, ties, values next to 448 scale, a block of NaN and
    infinities, one of them beside finite values."""
    big = torch.finfo(dtype).max
    rows = [torch.tensor([big, -big, 1.0, 0.0, -0.0]), torch.tensor([1e-45, 1e-40, -1.2e-38, 0.0]), torch.tensor([float("inf"), float("nan"), -float("inf")]),
            torch.tensor([448.0, 449.0, 447.0, 17.0, 18.0, 19.0, 1.0625, 1.1875, 2.0 ** -6, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 2.0 ** -11]),
            torch.tensor([1.75, 1.7578125, 1.75 * 2.0 ** 100]), torch.tensor([float("inf"), 3.0, -5.0, float("nan"), 0.25])]
    x = torch.zeros(len(rows), features, device="cuda")
    for k, r in enumerate(rows):
        x[k, 3:3 + len(r)] = r.cuda()
        x[k, 40:40 + len(r)] = r.cuda() * 0.5
        x[k, 90] = 1.0
    x = x.to(dtype)
    want = quantised(x)
    assert bool(torch.isnan(want).any())
    c = checkpoint_of(x)
    back = torch.empty(len(rows), features, device="cuda")
    vgc.vgc_checkpoint_load(c.t, back)
    # the largest numbers' codes stand for 2^128, which in fp32 is infinity
    assert bool(torch.isinf(back).any()) and same(back, want.float())


def test_error_of_a_value():
    """2^-4 of a value where |x| >= 2^-6 scale: half a unit of three bits behind the leading one; 2^-10 scale below."""
    x = activations(500, 512, torch.float32, 3)
    c = checkpoint_of(x)
    back = torch.empty_like(x)
    vgc.vgc_checkpoint_load(c.t, back)
    _, scales = layout(c.t, 500, 512)
    scale = (scales[:, :500].permute(1, 0, 2).reshape(500, 16).double() - 127).exp2().repeat_interleave(32, 1)
    assert bool(((back.double() - x.double()).abs() <= torch.maximum(2.0 ** -4 * x.double().abs(), 2.0 ** -10 * scale)).all())


def test_leading_dimensions_streams_and_replay():
    """[batch, tokens, features]; a side stream; a captured pair of calls replayed with other values."""
    x = activations(6 * 50, 200, torch.bfloat16, 5).view(6, 50, 200)
    c, back = torch.empty(vgc.vgc_checkpoint_bytes(300, 200), dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    vgc.vgc_checkpoint_store(x, c, stream=side)
    vgc.vgc_checkpoint_load(c, back, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert same(back.view(300, 200), quantised(x.view(300, 200)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vgc.vgc_checkpoint_store(x, c)
        vgc.vgc_checkpoint_load(c, back)
    for seed in (6, 7):
        x.copy_(activations(300, 200, torch.bfloat16, seed).view(6, 50, 200))
        graph.replay()
        assert same(back.view(300, 200), quantised(x.view(300, 200)))


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    c = torch.zeros(vgc.vgc_checkpoint_bytes(4, 64), dtype=torch.uint8, device="cuda")
    with pytest.raises(TypeError):
        vgc.vgc_checkpoint_store(x.half(), c)
    with pytest.raises(ValueError):
        vgc.vgc_checkpoint_store(x, c[:-1])
    with pytest.raises(ValueError):
        vgc.vgc_checkpoint_store(x.t(), c)
    with pytest.raises(TypeError):
        vgc.vgc_checkpoint_load(c.to(torch.int8), x)
    with pytest.raises(vgc.VgcError):                     # rows that do not start on 16 bytes
        vgc.vgc_checkpoint_store(torch.zeros(257, device="cuda")[1:].view(4, 64), c)
    vgc.vgc_checkpoint_store(x[:0], c[:0])                # no rows: nothing happens
    assert bool((c == 0).all())
