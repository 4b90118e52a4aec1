"""Helpers of the tests of layer norm, 8-bit checkpoints and the linear layer's gradient and statistic: their definitions in
64 bits, and inputs."""
import torch

import paper_1802_06058_b200 as vgc
from gpu_harness import Guarded

U = 2.0 ** -24                       # half an fp32 ulp, relative


def half_ulp(dtype):
    return torch.finfo(dtype).eps / 2


def quantised(x):
    """What the 8-bit checkpoint of x [rows, features] stands for, in 64 bits: x / scale in three bits behind the leading one (steps
    of 2^-9 below 2^-6), scale the smallest power of two, 2^-126 at least, with max |x| <= 448 scale over 32 features."""
    rows, features = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -features % 32)).view(rows, -1, 32)
    odd = ~torch.isfinite(v)
    v = torch.where(odd, 0.0, v)
    exponents = torch.arange(-126, 128, dtype=torch.float64, device=x.device).exp2()
    scale = exponents[torch.searchsorted(448 * exponents, v.abs().amax(2)).clamp(max=len(exponents) - 1)][:, :, None]
    u = v / scale
    step = (torch.frexp(u)[1].double() - 4).clamp(min=-9).exp2()
    q = torch.round(u / step) * step * scale            # torch.round: ties to even
    return torch.where(odd, float("nan"), q).view(rows, -1)[:, :features]


def checkpoint_of(x):
    """A guarded checkpoint of x, written by the library."""
    rows, features = x.shape
    c = Guarded(vgc.vgc_checkpoint_bytes(rows, features), torch.uint8)
    vgc.vgc_checkpoint_store(x, c.t)
    return c


def layout(buffer, rows, features):
    """(codes [rows, Cp] uint8, scale exponents [Cp / 128, Rp, 4] uint8) of a checkpoint"""
    wide, tall = -(-features // 128) * 128, -(-rows // 128) * 128
    codes = buffer[:rows * wide].view(rows, wide)
    return codes, buffer[rows * wide:].view(wide // 128, tall, 4)


def activations(rows, features, dtype, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    size = torch.randn(features, device="cuda", generator=gen).exp()
    return (torch.randn(rows, features, device="cuda", generator=gen) * size + 0.5).to(dtype)


def errors(rows, features, dtype, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    d = torch.randn(rows, features, device="cuda", generator=gen) * torch.randn(rows, 1, device="cuda", generator=gen).exp() * 1e-3
    d[torch.rand(rows, device="cuda", generator=gen) < 0.1] = 0
    return d.to(dtype)


def workspace(nbytes):
    return Guarded(max(nbytes, 256), torch.uint8, fill=0)
