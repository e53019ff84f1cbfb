"""The operators with which a pruned network is fine-tuned from 8-bit checkpoints, as cases that can be timed, beside plain forms of them.

  norm       group norm with an activation over NHWC activations, forward (GroupNorm.forward): y and the statistics; or y in 8 bits alone, as the next
             pruned layer multiplies it and as its weight gradient takes it, and that read back (Activations8.dequantize)
  norm_back  its backward pass (GroupNorm.backward), from x as it was or from x in 8 bits
  grad       the weight gradient dW = dY^T X of a pruned layer from its 8-bit activations (HybridLayer.weight_gradient8), of all weights or of those under
             the mask
  grad_conv  the same of a convolution (HybridLayer.weight_gradient8_conv), activations and dY in NHWC

The 8-bit form holds x as code * 2^E: e4m3 codes, and for each 128 consecutive channels of a pixel (from a multiple of 128 on) the smallest E with which
the largest of them can be held.
"""
import math

import torch

own = False

EPS = 1e-5


# ------------------------------------------------------------------------------------------------------------------ cases

def _norm(name, batch, height, width, channels, groups, act, dtype, kept=False, back=False):
    return {"name": name, "kind": "norm_back" if back else "norm", "batch": batch, "height": height, "width": width, "channels": channels, "groups": groups,
            "act": act, "dtype": dtype, "kept": kept}


def _grad(name, rows, k, tokens, layout, out, masked=False, n=4, m=4, keep=1.0):
    return {"name": name, "kind": "grad", "rows": rows, "k": k, "tokens": tokens, "layout": layout, "out": out, "masked": masked, "n": n, "m": m,
            "keep": keep}


def _conv(name, rows, channels, kernel, pad, batch, height, width, out):
    return {"name": name, "kind": "grad_conv", "rows": rows, "channels": channels, "kernel": kernel, "pad": pad, "batch": batch, "height": height,
            "width": width, "out": out}


def listed():
    return [
        # the last layer of MobileNetV2 on one image: 63 thousand values, latency counts
        _norm("norm_7x7x1280", 1, 7, 7, 1280, 32, "relu6", "bf16"),
        # ResNet-50's first stage, a training batch; y only in 8 bits, for an 8-bit product and its gradient
        _norm("norm_56x56x256_to_8_bits", 32, 56, 56, 256, 32, "relu", "bf16", True),
        # VGG-16's first layers: 205 MB, more than L2 holds
        _norm("norm_224x224x64", 32, 224, 224, 64, 32, "silu", "bf16"),
        # odd sizes in fp32, four channels a group
        _norm("norm_27x31x100_fp32", 3, 27, 31, 100, 25, "none", "fp32"),
        # backward: ResNet-50's third stage, a small batch
        _norm("back_14x14x512", 8, 14, 14, 512, 32, "relu", "bf16", False, True),
        # backward of the second case's layer from its input in 8 bits
        _norm("back_56x56x256_from_8_bits", 32, 56, 56, 256, 32, "relu", "bf16", True, True),
        # backward of MobileNetV2's widest layer, three channels a group
        _norm("back_112x112x96", 32, 112, 112, 96, 32, "relu6", "bf16", False, True),
        # a pointwise layer of MobileNetV2 on one image
        _grad("grad_160x960_49_pixels", 160, 960, 49, "tokens", "fp32"),
        # a lowered 14x14 convolution of an incomplete batch, 2:4 inside a quarter of the blocks, dY as [rows, pixels]
        _grad("grad_512x4608_6076_masked", 512, 4608, 31 * 14 * 14, "rows", "fp32", True, 2, 4, 0.25),
        # a 4096 x 4096 linear layer, 8192 tokens: every weight's gradient (a saliency needs them all)
        _grad("grad_4096_8192_tokens", 4096, 4096, 8192, "tokens", "bf16"),
        # the same with half of the blocks kept
        _grad("grad_4096_8192_masked", 4096, 4096, 8192, "tokens", "fp32", True, 4, 4, 0.5),
        # ResNet-50's 3 x 3 convolutions at 28 x 28
        _conv("grad_conv_128_3x3_28x28", 128, 128, 3, 1, 32, 28, 28, "fp32"),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_back", "norm_back", "grad", "grad", "grad_conv"])
    if kind in ("norm", "norm_back"):
        groups, each = rng.choice([1, 2, 4, 8, 16, 25, 32, 32, 32]), _log(rng, 1, 64)
        channels = groups * each
        height, width = _log(rng, 1, 224), _log(rng, 1, 224)
        batch = max(1, min(_log(rng, 1, 32), (1 << 25) // (height * width * channels)))
        while batch * height * width * channels > 1 << 25:
            height = (height + 1) // 2
        return {"kind": kind, "batch": batch, "height": height, "width": width, "channels": channels, "groups": groups,
                "act": rng.choice(["none", "relu", "relu6", "silu"]), "dtype": rng.choice(["bf16", "bf16", "bf16", "fp16", "fp32"]), "kept": False} \
            | rng.choice([{}, {}, {"kept": True, "dtype": "bf16"}])
    if kind == "grad":
        n, m = rng.choice([(2, 4), (4, 4), (1, 4), (2, 8), (4, 8)])
        return {"kind": kind, "rows": _log(rng, 8, 4096), "k": _log(rng, 16, 4096), "tokens": _log(rng, 1, 8192), "layout": rng.choice(["tokens", "rows"]),
                "out": rng.choice(["fp32", "bf16"]), "masked": rng.random() < 0.5, "n": n, "m": m, "keep": rng.choice([1.0, 0.5, 0.25, rng.uniform(0.1, 1.0)])}
    kernel = rng.choice([1, 3, 3, 5])
    channels, height, width = _log(rng, 8, 512), _log(rng, kernel, 56), _log(rng, kernel, 56)
    batch = max(1, min(_log(rng, 1, 32), (1 << 27) // (height * width * channels * kernel * kernel)))
    return {"kind": kind, "rows": _log(rng, 8, 512), "channels": channels, "kernel": kernel, "pad": rng.choice([0, kernel // 2, kernel // 2]),
            "batch": batch, "height": height, "width": width, "out": rng.choice(["fp32", "bf16"])}


TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    rng = torch.Generator(device="cuda")
    rng.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=rng)  # noqa: E731
    rand = lambda *shape: torch.rand(*shape, device="cuda", generator=rng)  # noqa: E731
    kind = case["kind"]
    if kind == "grad":
        return _prepare_grad(case, randn, rand)
    if kind == "grad_conv":
        return _prepare_conv(case, randn, rand)
    # activations as a convolution leaves them: channels of different size and mean
    dtype = TYPES[case["dtype"]]
    batch, height, width, channels, groups = (case[q] for q in ("batch", "height", "width", "channels", "groups"))
    x = (randn(batch, height, width, channels) * torch.exp(randn(channels) * 0.3) + randn(channels) * 0.5).to(dtype)
    state = dict(case, x=x, weight=1 + 0.2 * randn(channels), bias=0.3 * randn(channels))
    if own:
        from paper_2311_14272_b200 import binding as B
        state["norm"] = B.GroupNorm(channels, groups, state["weight"], state["bias"], eps=EPS, activation=case["act"])
    if kind == "norm":
        return state
    state["dy"] = (randn(batch, height, width, channels) * torch.exp(randn(batch, 1, 1, 1) * 0.5) * 1e-2).to(dtype)
    # what the forward pass left: the statistics, and x as it was or in 8 bits
    state["statistics"] = torch.stack(_statistics(x, groups), 2)
    if case["kept"]:
        state["codes"], state["scale"] = _codes(x.view(-1, channels))
        state["kept_x"] = B.quantize8(x.view(-1, channels), tokens=True) if own else None
    return state


def _statistics(x, groups):
    """Mean and 1 / standard deviation of each sample's groups [batch, groups], from 64 bits."""
    v = x.reshape(x.shape[0], -1, groups, x.shape[-1] // groups)
    mean = v.mean((1, 3), dtype=torch.float64)
    var = torch.stack([(q.double() - c[None, :, None]).square().mean((0, 2)) for q, c in zip(v, mean)])
    return mean.float(), (var + EPS).rsqrt().float()


def _mask(rows, k, n, m, keep, weights, rand):
    """A saliency whose mask is known (blocks of 128 x 128): the kept blocks' is 2^20 times the others'.  -> saliency, mask of booleans"""
    nrt, nblk = -(-rows // 128), -(-k // 128)
    kept = int(math.floor(keep * nblk + 0.5))
    order = rand(nrt, nblk).argsort(1).argsort(1) < kept
    inside = order.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :k]
    s = weights.abs() * (0.5 + rand(rows, k)) + 1e-6 * (1 + rand(rows, k))
    groups = torch.nn.functional.pad(s, (0, -k % m)).view(rows, -1, m)
    best = torch.zeros(groups.shape, dtype=torch.bool, device="cuda").scatter_(2, groups.topk(n, 2).indices, True).view(rows, -1)[:, :k]
    return torch.where(inside, s * 2.0**20, s), inside & best


def _activations(tokens, k, randn, rand):
    """Activations behind a ReLU, tokens of different size, a few large features."""
    x = (randn(tokens, k) + 0.3).clamp(min=0) * torch.exp(randn(tokens, 1) * 0.5) * torch.where(rand(1, k) < 0.01, 20.0, 1.0)
    return x.bfloat16()


def _prepare_grad(case, randn, rand):
    rows, k, tokens = case["rows"], case["k"], case["tokens"]
    x = _activations(tokens, k, randn, rand)
    dy = (randn(tokens, rows) * torch.exp(randn(tokens, 1) * 0.5) * 1e-2).bfloat16()
    state = dict(case, x=x, dy=dy if case["layout"] == "tokens" else dy.t().contiguous())
    saliency, state["mask"] = _mask(rows, k, case["n"], case["m"], case["keep"], randn(rows, k), rand)
    state["codes"], state["scale"] = _codes(x)
    if own:
        from paper_2311_14272_b200 import binding as B
        state["layer"] = B.HybridLayer(rows, k, case["n"], case["m"], 128, 128, case["keep"]).build_mask(saliency)
        state["kept_x"] = B.quantize8(x, tokens=True)
    return state


def _prepare_conv(case, randn, rand):
    batch, height, width, channels, kernel, pad = (case[q] for q in ("batch", "height", "width", "channels", "kernel", "pad"))
    x = _activations(batch * height * width, channels, randn, rand)
    ho, wo = height + 2 * pad - kernel + 1, width + 2 * pad - kernel + 1
    dy = (randn(batch, ho, wo, case["rows"]) * torch.exp(randn(batch, 1, 1, 1) * 0.5) * 1e-2).bfloat16()
    state = dict(case, x=x, dy=dy)
    state["codes"], state["scale"] = _codes(x)
    if own:
        from paper_2311_14272_b200 import binding as B
        state["layer"] = B.HybridLayer(case["rows"], kernel * kernel * channels, 4, 4, 128, 128, 1.0)
        state["kept_x"] = B.quantize8(x, tokens=True)
    return state


# -------------------------------------------------------------------------------------------------------------- plain forms

def _codes(x):
    """x [tokens, k] in 8 bits: e4m3 codes [tokens, k] and the exponent of each 128 of a token [tokens, k-blocks]."""
    tokens, k = x.shape
    blocks = torch.nn.functional.pad(x.float(), (0, -k % 128)).view(tokens, -1, 128)
    largest = blocks.abs().amax(2)
    fraction, exponent = torch.frexp(largest)
    e = torch.where(largest > 0, exponent - 9 + (fraction * 2 > 448.0 / 256).int(), -126).clamp(-126, 127)
    codes = (blocks * torch.ldexp(torch.ones_like(largest), -e)[:, :, None]).to(torch.float8_e4m3fn)
    return codes.view(tokens, -1)[:, :k].contiguous(), e


def _values(codes, e):
    return codes.float() * torch.ldexp(torch.ones_like(e, dtype=torch.float32), e).repeat_interleave(128, 1)[:, :codes.shape[1]]


def _slope(p, act):
    """The activation's derivative; p in 64 bits, as it lies next to a border now and then."""
    if act == "relu":
        return (p > 0).float()
    if act == "relu6":
        return ((p > 0) & (p < 6)).float()
    if act == "silu":
        s = torch.sigmoid(p.float())
        return s * (1 + p.float() * (1 - s))
    return torch.ones_like(p, dtype=torch.float32)


def _plain_norm(s):
    x, groups, act = s["x"].float(), s["groups"], s["act"]
    batch, channels = x.shape[0], x.shape[-1]
    v = x.view(batch, -1, groups, channels // groups)
    mean = v.mean((1, 3), keepdim=True)
    rest = v - mean
    rstd = (rest.square().mean((1, 3), keepdim=True) + EPS).rsqrt()
    y = (rest * rstd).view(x.shape) * s["weight"] + s["bias"]
    if act == "silu":
        y = y * torch.sigmoid(y)
    elif act != "none":
        y = y.clamp(min=0, max=6 if act == "relu6" else None)
    statistics = torch.stack([mean.view(batch, groups), rstd.view(batch, groups)], 2)
    if s["kept"]:
        return [_values(*_codes(y.view(-1, channels))).bfloat16(), statistics]
    return [y.to(s["x"].dtype), statistics]


def _plain_norm_back(s):
    groups, channels = s["groups"], s["channels"]
    shape = s["dy"].shape
    x = (_values(s["codes"], s["scale"]) if s["kept"] else s["x"].float()).view(shape[0], -1, groups, channels // groups)
    mean, rstd = (q.view(shape[0], 1, groups, 1) for q in s["statistics"].unbind(2))
    weight, bias = s["weight"].view(groups, -1), s["bias"].view(groups, -1)
    e = s["dy"].float().view(x.shape) * _slope((x.double() - mean) * rstd * weight + bias, s["act"])
    xhat = (x - mean) * rstd
    dbias, dweight = e.sum((0, 1)), (e * xhat).sum((0, 1))
    g = e * weight
    dx = rstd * (g - g.mean((1, 3), keepdim=True) - xhat * (g * xhat).mean((1, 3), keepdim=True))
    return [dx.view(shape).to(s["dy"].dtype), dweight.view(channels), dbias.view(channels)]


def _plain_conv(s):
    batch, height, width, channels, kernel, pad = (s[q] for q in ("batch", "height", "width", "channels", "kernel", "pad"))
    x = torch.nn.functional.pad(_values(s["codes"], s["scale"]).view(batch, height, width, channels), (0, 0, pad, pad, pad, pad))
    windows = x.unfold(1, kernel, 1).unfold(2, kernel, 1).permute(0, 1, 2, 4, 5, 3)          # [batch, ho, wo, i, j, channel]
    dy = s["dy"].float().view(-1, s["rows"])
    return dy.t() @ windows.reshape(dy.shape[0], -1)


def run(s):
    kind = s["kind"]
    if kind == "norm":
        if not own:
            return _plain_norm(s)
        if s["kept"]:
            done = s["norm"].forward(s["x"], keep_y=True, plain_y=False)
            return [done.y8.dequantize(tokens=True), done.statistics]
        done = s["norm"].forward(s["x"])
        return [done.y, done.statistics]
    if kind == "norm_back":
        if not own:
            return _plain_norm_back(s)
        return list(s["norm"].backward(s["dy"], s["kept_x"] if s["kept"] else s["x"], s["statistics"]))
    if kind == "grad_conv":
        if not own:
            return _plain_conv(s).to(TYPES[s["out"]])
        return s["layer"].weight_gradient8_conv(s["dy"], s["kept_x"], s["kernel"], s["kernel"], s["pad"], dw_dtype=int(s["out"] == "fp32"))
    if own:
        return s["layer"].weight_gradient8(s["dy"], s["kept_x"], tokens=s["layout"] == "tokens", masked=s["masked"], dw_dtype=int(s["out"] == "fp32"))
    x, dy = _values(s["codes"], s["scale"]), s["dy"].float()
    dw = (dy.t() if s["layout"] == "tokens" else dy) @ x
    return (torch.where(s["mask"], dw, 0.0) if s["masked"] else dw).to(TYPES[s["out"]])


# --------------------------------------------------------------------------------------------------------------------- work

def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    if case["kind"] in ("norm", "norm_back"):
        count = case["batch"] * case["height"] * case["width"] * case["channels"]
        one = size[case["dtype"]]
        eight = count + count / case["channels"] * -(-case["channels"] // 128)
        if case["kind"] == "norm":
            # x, and y; or y in 8 bits, that read and written in bf16
            return {"bytes": count * one + (2 * eight + 2.0 * count if case["kept"] else count * one), "flops": 8.0 * count}
        return {"bytes": 2.0 * count * one + (eight if case["kept"] else count * one), "flops": 16.0 * count}
    if case["kind"] == "grad_conv":
        pixels = case["batch"] * case["height"] * case["width"]
        ho, wo = (case[q] + 2 * case["pad"] - case["kernel"] + 1 for q in ("height", "width"))
        k = case["kernel"] ** 2 * case["channels"]
        return {"bytes": 1.0 * pixels * case["channels"] + 2.0 * case["batch"] * ho * wo * case["rows"] + case["rows"] * k * size[case["out"]],
                "flops": 2.0 * case["batch"] * ho * wo * case["rows"] * k}
    rows, k, tokens = case["rows"], case["k"], case["tokens"]
    nblk = -(-k // 128)
    share = math.floor(case["keep"] * nblk + 0.5) / nblk if case["masked"] else 1.0
    return {"bytes": tokens * k * min(1.0, share * -(-rows // 128)) + 2.0 * tokens * rows + rows * k * size[case["out"]],
            "flops": 2.0 * tokens * rows * k * share}


# ------------------------------------------------------------------------------------------------------------ in 64 bits

def _held(x):
    """x [tokens, k] (64 bits) as its 8-bit form holds it: code * 2^E, codes with a spacing of 2^(exponent - 3) down to exponent -6, nearest even."""
    tokens, k = x.shape
    x = torch.cat([x, torch.zeros(tokens, -k % 128, dtype=torch.float64, device=x.device)], 1).reshape(tokens, -1, 128)
    largest = x.abs().amax(2, keepdim=True)
    e = torch.where(largest > 0, torch.ceil(torch.log2(largest.clamp(min=1e-300) / 448.0)), -126.0)
    e = torch.where(largest > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where(largest <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(-126, 127)
    y = x.abs() * torch.exp2(-e)
    _, exponent = torch.frexp(y)
    spacing = torch.exp2((exponent - 1).clamp(min=-6).double() - 3)
    return (torch.sign(x) * torch.round(y / spacing) * spacing * torch.exp2(e)).view(tokens, -1)[:, :k]


def _exact_sample(x, dy, s, b):
    """One sample [pixels, channels] of the norm: y and its statistics, or with dy: dx and its part of the sums for weight and bias."""
    groups, channels, act = s["groups"], s["channels"], s["act"]
    of = torch.arange(channels, device=x.device) // (channels // groups)
    weight, bias = s["weight"].double(), s["bias"].double()
    if dy is None:
        first = x.sum(0).view(groups, -1).sum(1) * groups / x.numel()
        var = ((x - first[of]) ** 2).sum(0).view(groups, -1).sum(1) * groups / x.numel()
        rstd = 1 / torch.sqrt(var + EPS)
        p = (x - first[of]) * (rstd[of] * weight) + bias
        y = {"none": lambda: p, "relu": lambda: torch.relu(p), "relu6": lambda: torch.minimum(torch.relu(p), torch.tensor(6.0, dtype=torch.float64, device=p.device)),
             "silu": lambda: p / (1 + torch.exp(-p))}[act]()
        return y, torch.stack([first, rstd], 1)
    mean, rstd = s["statistics"][b].double().unbind(1)
    hat = (x - mean[of]) * rstd[of]
    p = hat * weight + bias
    if act == "silu":
        q = 1 / (1 + torch.exp(-p))
        dy = dy * (q + p * q * (1 - q))
    elif act != "none":
        dy = dy * (p > 0)
        dy = dy * (p < 6) if act == "relu6" else dy
    db, dw = dy.sum(0), (dy * hat).sum(0)
    each = x.shape[0] * channels // groups
    m1, m2 = ((weight * q).view(groups, -1).sum(1) / each for q in (db, dw))
    return (weight * dy - m1[of] - hat * m2[of]) * rstd[of], dw, db


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "grad":
        dy = s["dy"].double()
        dw = (dy if case["layout"] == "rows" else dy.t()) @ _held(s["x"].double())
        return dw * s["mask"] if case["masked"] else dw
    if kind == "grad_conv":
        batch, height, width, channels, kernel, pad, rows = (case[q] for q in ("batch", "height", "width", "channels", "kernel", "pad", "rows"))
        x = torch.zeros(batch, height + 2 * pad, width + 2 * pad, channels, dtype=torch.float64, device="cuda")
        x[:, pad:pad + height, pad:pad + width] = _held(s["x"].double()).view(batch, height, width, channels)
        dy = s["dy"].double()
        ho, wo = dy.shape[1:3]
        taps = [dy.reshape(-1, rows).t() @ x[:, i:i + ho, j:j + wo].reshape(-1, channels) for i in range(kernel) for j in range(kernel)]
        return torch.cat(taps, 1)
    batch, channels = case["batch"], case["channels"]
    x = s["x"].view(batch, -1, channels)
    if kind == "norm":
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        statistics = torch.empty(batch, case["groups"], 2, dtype=torch.float64, device="cuda")
        for b in range(batch):
            one, statistics[b] = _exact_sample(x[b].double(), None, s, b)
            y[b] = _held(one) if case["kept"] else one
        return [y.view(-1, channels) if case["kept"] else y.view(s["x"].shape), statistics]
    dx = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    dw, db = (torch.zeros(channels, dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(batch):
        one = x[b].double()
        dx[b], w, v = _exact_sample(_held(one) if case["kept"] else one, s["dy"][b].view(-1, channels).double(), s, b)
        dw += w
        db += v
    return [dx.view(s["x"].shape), dw, db]
