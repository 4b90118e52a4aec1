"""The operators that a transformer's training step asks of this library beside its compressor, as cases that can be timed.

  norm        layer norm's forward pass, on request with the 8-bit checkpoint of its output (the next layer's input)
  norm_back   its backward pass: the input's gradient, gradient and squared-gradient sums of gain and bias
  checkpoint  activations into 8 bits in the forward pass, and back in the backward pass
  wgrad       a linear layer's gradient and squared-gradient sums from its input's 8-bit checkpoint and the error delta

``run`` computes them from their formulas in elementary torch operations, or, where ``own`` is true, through the library.
``exact`` gives the same from the definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # a few tokens of a small model: what a call costs before there is any work
        {"name": "norm_few_rows", "kind": "norm", "rows": 16, "features": 1024, "type": "bf16", "checkpoint": True},
        # one layer of a micro-batch of 8 sequences of 2048 tokens, with the checkpoint that its linear layer is trained from
        {"name": "norm_checkpoint", "kind": "norm", "rows": 16384, "features": 4096, "type": "bf16", "checkpoint": True},
        # a ragged batch of a small network kept in fp32, rows that do not start on 16 bytes
        {"name": "norm_ragged", "kind": "norm", "rows": 5003, "features": 1001, "type": "fp32", "checkpoint": False},
        # a small network's mini-batch, every row a sample
        {"name": "norm_back_small", "kind": "norm_back", "rows": 128, "features": 784, "type": "fp32", "per_example": 1},
        # the micro-batch above on its way back
        {"name": "norm_back_large", "kind": "norm_back", "rows": 16384, "features": 4096, "type": "bf16", "per_example": 1},
        # images as 197 patches each, statistic per image
        {"name": "norm_back_images", "kind": "norm_back", "rows": 64 * 197, "features": 1280, "type": "bf16", "per_example": 197},
        # the hidden layer of a small network
        {"name": "checkpoint_small", "kind": "checkpoint", "rows": 257, "features": 1024, "type": "fp32"},
        # the widest activation of a layer: 8 sequences of 2048 tokens, four times the model's width
        {"name": "checkpoint_large", "kind": "checkpoint", "rows": 16384, "features": 16384, "type": "bf16"},
        # the first layer of the 784-1024-1024-10 network, error in fp32
        {"name": "wgrad_small", "kind": "wgrad", "rows": 128, "in": 784, "out": 1024, "type": "fp32"},
        # an attention projection of a small model
        {"name": "wgrad_square", "kind": "wgrad", "rows": 8192, "in": 1024, "out": 1024, "type": "bf16"},
        # odd sizes: a vocabulary-like output that no vector width divides, error in fp32
        {"name": "wgrad_ragged", "kind": "wgrad", "rows": 3001, "in": 1000, "out": 2051, "type": "fp32"},
        # the first projection of a feed-forward block, 8 sequences of 2048 tokens
        {"name": "wgrad_large", "kind": "wgrad", "rows": 16384, "in": 4096, "out": 16384, "type": "bf16"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of the ranges above: any sizes between the smallest and the largest, odd ones as likely as not."""
    kind = rng.choice(["norm", "norm_back", "checkpoint", "wgrad"])
    type_ = rng.choice(["fp32", "bf16", "bf16"])
    if kind == "wgrad":
        while True:
            rows, n_in, n_out = _log(rng, 1, 16384), _log(rng, 16, 16384), _log(rng, 10, 16384)
            if rng.random() < 0.5:
                n_in, n_out = -(-n_in // 64) * 64, -(-n_out // 64) * 64
            if rows * n_in * n_out <= (1 << 39) and n_in * n_out <= (1 << 26):
                return {"kind": kind, "rows": rows, "in": n_in, "out": n_out, "type": type_}
    while True:
        rows, features = _log(rng, 1, 40000), _log(rng, 16, 16384)
        if rng.random() < 0.5:
            features = -(-features // 64) * 64
        if rows * features <= (1 << 26):
            break
    case = {"kind": kind, "rows": rows, "features": features, "type": type_}
    if kind == "norm":
        case["checkpoint"] = type_ == "bf16" and rng.random() < 0.6
    if kind == "norm_back":
        case["per_example"] = 1
        if rng.random() < 0.4:                   # sequences of one length
            case["per_example"] = min(rows, _log(rng, 2, 4096))
            case["rows"] = rows // case["per_example"] * case["per_example"]
    return case


# ---- the 8-bit checkpoint: layout and values ----------------------------------------------------------------------------
# codes [rows][padded features] (e4m3, padded to 128 features with zeros), then for each 128 features and each row (padded
# to 128 rows) the four scale exponents of its blocks of 32
def _sizes(rows, features):
    return -(-features // 128) * 128, -(-rows // 128) * 128


def _encode(x):
    """x [rows][features] -> (codes [rows][padded] float8, exponents [rows][padded / 32] int32)"""
    rows, features = x.shape
    wide, _ = _sizes(rows, features)
    v = torch.zeros(rows, wide, dtype=torch.float32, device=x.device)
    v[:, :features] = x
    v = v.view(rows, wide // 32, 32)
    bits = v.abs().nan_to_num(nan=0.0, posinf=0.0).amax(2).view(torch.int32)
    e = (((bits + 0x1FFFFF) >> 23) - 8).clamp(min=1)
    scaled = v * ((254 - e) << 23).view(torch.float32)[:, :, None]
    return scaled.to(torch.float8_e4m3fn).view(rows, wide), e


def _decode(codes, e, features):
    rows, wide = codes.shape
    v = codes.to(torch.float32).view(rows, wide // 32, 32) * (e << 23).view(torch.float32)[:, :, None]
    return v.view(rows, wide)[:, :features]


def _pack(codes, e):
    """The checkpoint as the library keeps it: one buffer of bytes."""
    rows, wide = codes.shape
    _, tall = _sizes(rows, wide)
    scales = torch.zeros(wide // 128, tall, 4, dtype=torch.uint8, device=codes.device)
    scales[:, :rows] = e.view(rows, wide // 128, 4).permute(1, 0, 2).to(torch.uint8)
    return torch.cat([codes.view(torch.uint8).reshape(-1), scales.reshape(-1)])


def _unpack(buffer, rows, features):
    wide, tall = _sizes(rows, features)
    codes = buffer[:rows * wide].view(torch.float8_e4m3fn).view(rows, wide)
    scales = buffer[rows * wide:].view(wide // 128, tall, 4)[:, :rows]
    return codes, scales.permute(1, 0, 2).reshape(rows, wide // 32).to(torch.int32)


def _bytes(rows, features):
    wide, tall = _sizes(rows, features)
    return rows * wide + tall * wide // 32


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _activations(rows, features, type_, gen):
    """A residual stream: features of different size, a few of them large, a common offset."""
    size = torch.randn(features, device=DEV, generator=gen).mul_(0.5).exp_()
    size[torch.randperm(features, device=DEV, generator=gen)[:max(1, features // 200)]] *= 12
    x = torch.randn(rows, features, device=DEV, generator=gen)
    return x.mul_(size).add_(0.1).to(TYPES[type_])


def _errors(rows, features, type_, gen):
    """Errors of a loss averaged over the tokens: rows of different size, some of them padding (zero)."""
    size = torch.randn(rows, 1, device=DEV, generator=gen).exp_().mul_(1e-3)
    size[torch.rand(rows, 1, device=DEV, generator=gen) < 0.06] = 0
    size[rows // 2] = 1e-3
    return torch.randn(rows, features, device=DEV, generator=gen).mul_(size).to(TYPES[type_])


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    rows, t = case["rows"], TYPES[case["type"]]
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    s = dict(case, keep={})
    if case["kind"] == "wgrad":
        n_in, n_out = case["in"], case["out"]
        x = _activations(rows, n_in, "bf16", gen)
        s["checkpoint"] = _pack(*_encode(x))
        s["delta"] = _errors(rows, n_out, case["type"], gen)
        s["g"], s["S"] = new(n_out, n_in), new(n_out, n_in)
        return s
    C = case["features"]
    s["x"] = _activations(rows, C, case["type"], gen)
    if case["kind"] == "checkpoint":
        s["buffer"], s["back"] = new(_bytes(rows, C), dtype=torch.uint8), new(rows, C, dtype=torch.bfloat16)
        return s
    s["gamma"] = 1 + 0.2 * torch.randn(C, device=DEV, generator=gen)
    if case["kind"] == "norm":
        s["beta"] = 0.1 * torch.randn(C, device=DEV, generator=gen)
        s["y"], s["mean"], s["rstd"] = new(rows, C, dtype=t), new(rows), new(rows)
        if case["checkpoint"]:
            s["buffer"], s["back"] = new(_bytes(rows, C), dtype=torch.uint8), new(rows, C, dtype=torch.bfloat16)
        return s
    s["dy"] = _errors(rows, C, case["type"], gen)
    wide = s["x"].double()
    mean = wide.mean(1)
    s["mean"], s["rstd"] = mean.float(), (wide.var(1, unbiased=False) + EPS).rsqrt().float()
    s["dx"] = new(rows, C, dtype=t)
    s["vectors"] = [new(C) for _ in range(4)]
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    return {"norm": _norm, "norm_back": _norm_back, "checkpoint": _checkpoint, "wgrad": _wgrad}[s["kind"]](s)


def _own(s):
    import paper_1802_06058_b200 as vgc
    keep, kind = s["keep"], s["kind"]
    if kind == "norm":
        buffer = s.get("buffer")
        vgc.vgc_layernorm(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"], checkpoint=buffer)
        out = [s["y"], s["mean"], s["rstd"]]
        if buffer is not None:
            out.append(vgc.vgc_checkpoint_load(buffer, s["back"]))
        return out
    if kind == "checkpoint":
        vgc.vgc_checkpoint_store(s["x"], s["buffer"])
        return vgc.vgc_checkpoint_load(s["buffer"], s["back"])
    if kind == "norm_back":
        if "ws" not in keep:
            n = vgc.vgc_layernorm_backward_workspace_bytes(s["rows"], s["features"], s["per_example"])
            keep["ws"] = torch.zeros(n, dtype=torch.uint8, device=DEV)
        n = s["rows"] // s["per_example"]
        vgc.vgc_layernorm_backward(s["x"], s["dy"], s["gamma"], s["mean"], s["rstd"], s["dx"], *s["vectors"], scale_g=1.0 / n,
                                   scale_s=1.0 / n ** 2, rows_per_example=s["per_example"], ws=keep["ws"])
        return [s["dx"]] + s["vectors"]
    if "ws" not in keep:
        n = vgc.vgc_wgrad_checkpoint_workspace_bytes(s["rows"], s["in"], s["out"], s["delta"].dtype)
        keep["ws"] = torch.zeros(n, dtype=torch.uint8, device=DEV)
    vgc.vgc_wgrad_checkpoint(s["checkpoint"], s["delta"], s["g"], s["S"], scale_g=1.0 / s["rows"], scale_s=1.0 / s["rows"] ** 2,
                             ws=keep["ws"])
    return [s["g"], s["S"]]


def _norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / (d.square().mean(1) + EPS).sqrt()
    y = (d * rstd[:, None] * s["gamma"] + s["beta"]).to(s["x"].dtype)
    out = [y, mean, rstd]
    if s["checkpoint"]:
        codes, e = _encode(y)
        out.append(_decode(codes, e, s["features"]).to(torch.bfloat16))
    return out


def _checkpoint(s):
    codes, e = _encode(s["x"])
    return _decode(codes, e, s["features"]).to(torch.bfloat16)


def _norm_back(s):
    T, rows, C = s["per_example"], s["rows"], s["features"]
    n = rows // T
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    w = dy * s["gamma"]
    dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    gain, bias = (dy * xh).view(n, T, C).sum(1), dy.view(n, T, C).sum(1)
    return [dx.to(s["x"].dtype), gain.sum(0) / n, bias.sum(0) / n, gain.square().sum(0) / n ** 2, bias.square().sum(0) / n ** 2]


def _wgrad(s):
    x = _decode(*_unpack(s["checkpoint"], s["rows"], s["in"]), s["in"])
    d = s["delta"].float()
    return [(d.T @ x) / s["rows"], (d.square().T @ x.square()) / s["rows"] ** 2]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    t, rows = 4 if case["type"] == "fp32" else 2, case["rows"]
    if case["kind"] == "wgrad":
        n_in, n_out = case["in"], case["out"]
        return {"bytes": rows * n_in * 33 / 32 + rows * n_out * t + 8 * n_in * n_out, "flops": 4.0 * rows * n_in * n_out}
    n = rows * case["features"]
    if case["kind"] == "checkpoint":              # store: x in, codes out; load: codes in, bf16 out
        return {"bytes": n * (t + 2 * 33 / 32 + 2), "flops": 4.0 * n}
    if case["kind"] == "norm":
        return {"bytes": n * (2 * t + (2 * 33 / 32 + 2 if case["checkpoint"] else 0)) + 8 * rows, "flops": 8.0 * n}
    return {"bytes": 3.0 * n * t + 8 * rows + 20 * case["features"], "flops": 14.0 * n}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------
def _rounded_to_8_bits(x):
    """Every value of x [rows][features] (64 bits) as its block of 32 keeps it: three bits behind the leading one, the
    smallest power-of-two scale under which the block's largest value is at most 448."""
    rows, features = x.shape
    v = torch.nn.functional.pad(x, (0, -features % 32)).view(rows, -1, 32)
    most = v.abs().amax(2, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(most / 448)).clamp(min=-126))
    unit = torch.where(most > 448 * unit, 2 * unit, unit)
    unit = torch.where((most <= 448 * (unit / 2)) & (unit > 2.0 ** -126), unit / 2, unit)
    u = v / unit
    step = torch.exp2(torch.frexp(u)[1].double().sub(4).clamp(min=-9))
    return (torch.round(u / step) * step * unit).view(rows, -1)[:, :features]


def exact(case, seed):
    s = prepare(case, seed)
    rows = case["rows"]
    if case["kind"] == "wgrad":
        n_in = case["in"]
        codes, e = _unpack(s["checkpoint"], rows, n_in)
        unit = torch.exp2(e.double() - 127).repeat_interleave(32, 1)
        x, d = (codes.double() * unit)[:, :n_in], s["delta"].double()
        g = torch.einsum("zo,zi->oi", d, x).div_(rows)
        return [g, torch.einsum("zo,zi->oi", d.square_(), x.square_()).div_(rows ** 2)]
    x, C = s["x"].double(), case["features"]
    if case["kind"] == "checkpoint":
        return _rounded_to_8_bits(x)
    gamma = s["gamma"].double()
    if case["kind"] == "norm":
        var, mean = torch.var_mean(x, 1, correction=0)
        y = torch.addcmul(s["beta"].double(), (x - mean[:, None]) * torch.rsqrt(var + EPS)[:, None], gamma)
        out = [y, mean, torch.rsqrt(var + EPS)]
        if case["checkpoint"]:                    # of y as it is kept
            out.append(_rounded_to_8_bits(y.to(TYPES[case["type"]]).double()))
        return out
    rstd, dy, T = s["rstd"].double(), s["dy"].double(), case["per_example"]
    xh = torch.einsum("rc,r->rc", x - s["mean"].double()[:, None], rstd)
    first, second = (dy @ gamma) / C, torch.einsum("rc,rc,c->r", dy, xh, gamma) / C
    dx = (dy * gamma - first[:, None] - xh * second[:, None]) * rstd[:, None]
    gain = torch.einsum("ntc,ntc->nc", dy.view(-1, T, C), xh.view(-1, T, C))
    bias = torch.einsum("ntc->nc", dy.view(-1, T, C))
    n = rows // T
    return [dx, gain.sum(0) / n, bias.sum(0) / n, torch.einsum("nc,nc->c", gain, gain) / n ** 2, torch.einsum("nc,nc->c", bias, bias) / n ** 2]
