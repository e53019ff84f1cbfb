"""The operators that fine-tune a pruned network and serve it in 8 bits, as cases that can be timed, beside plain forms of them.

  adamw    one AdamW step over all tensors of a network (AdamW.step): fp32 weights with the bf16 copy that the encoder takes, or bf16 weights;
           states in 32 bits, or in 8 with a power-of-two scale for each 128 elements; weights outside a layer's mask stay zero
  encode8  a pruned layer's weights to 8-bit floats with a scale for each kept block of 128 x 128, and back to what they stand for
           (HybridLayer.encode8, decode8)
  spmm8    Y = act(W X + bias) of such a layer, X quantised on the way with a scale for each 128 of a column (HybridLayer.spmm8)

Both 8-bit formats hold x as code * 2^E, with the smallest E that lets the largest value of the block be held.  Weights and activations are rounded
to the nearest e4m3 (even at ties).  Optimizer states (m: sign and e4m3; sqrt(v): e4m4 without sign) and bf16 weights are rounded at random: up where
the part below the code, plus an odd multiple of 2^-11 (m) or 2^-12 from a hash of (seed, step, tensor, element), reaches one.  sqrt(v) > 0 is never
held as 0.
"""
import math

import torch

own = False

MOBILENETV2 = ("32x32,16x32,96x16,24x96,144x24,24x144,144x24,32x144,192x32,32x192,192x32,32x192,192x32,64x192,384x64,64x384,384x64,64x384,384x64,"
               "64x384,384x64,96x384,576x96,96x576,576x96,96x576,576x96,160x576,960x160,160x960,960x160,160x960,960x160,320x960,1280x320")
VGG16 = ("64x27,1x64,64x576,1x64,128x576,1x128,128x1152,1x128,256x1152,1x256,256x2304,1x256,256x2304,1x256,512x2304,1x512,512x4608,1x512,"
         "512x4608,1x512,512x4608,1x512,512x4608,1x512,512x4608,1x512")
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 1e-2
M32 = 0xFFFFFFFF


# ------------------------------------------------------------------------------------------------------------------ cases

def _adamw(name, shapes, w32, g32, bits, masked, n=2, m=4, block=64, keep=0.5):
    return {"name": name, "kind": "adamw", "shapes": shapes, "w32": w32, "g32": g32, "bits": bits, "masked": masked, "n": n, "m": m, "block": block,
            "keep": keep}


def _encode8(name, rows, k, n, m, keep):
    return {"name": name, "kind": "encode8", "rows": rows, "k": k, "n": n, "m": m, "keep": keep}


def _spmm8(name, rows, k, ncols, n, m, keep, tokens, bias=False):
    return {"name": name, "kind": "spmm8", "rows": rows, "k": k, "ncols": ncols, "n": n, "m": m, "keep": keep, "tokens": tokens, "bias": bias}


def listed():
    return [
        # fine-tuning MobileNetV2's 35 pointwise layers after a pruning step: two million weights, the launches and the host's part count
        _adamw("adamw32_mobilenetv2", MOBILENETV2, True, False, 32, True, 2, 8, 32),
        # VGG-16's convolutions with their biases: ragged sizes (27 to 4608 a row), masks of 64 x 64 blocks
        _adamw("adamw32_vgg16", VGG16, True, True, 32, True, 2, 4, 64, 0.3),
        # eight 4096 x 4096 linear layers that are not pruned yet, everything in fp32
        _adamw("adamw32_linear_4096", ",".join(["4096x4096"] * 8), True, True, 32, False),
        # the smallest step: one linear layer of 256 x 1024 and its bias
        _adamw("adamw8_linear_256x1024", "256x1024,1x256", True, False, 8, False),
        # MobileNetV2 again, where memory is short: bf16 weights, states in 8 bits
        _adamw("adamw8_mobilenetv2", MOBILENETV2, False, False, 8, True, 2, 8, 32),
        # eight pruned 4096 x 4096 linear layers in bf16 with 8-bit states
        _adamw("adamw8_linear_4096", ",".join(["4096x4096"] * 8), False, False, 8, True, 2, 4, 128),
        # compressing a pruned linear layer for serving
        _encode8("encode8_4096_2of4", 4096, 4096, 2, 4, 0.5),
        # a classifier's odd number of classes and a k that ends inside a block
        _encode8("encode8_1000x2050", 1000, 2050, 4, 4, 1.0),
        # one token at a time through a layer whose blocks are all kept: bound by its weights
        _spmm8("spmm8_4096_1_token", 4096, 4096, 1, 4, 4, 1.0, True),
        # 37 requests decoding together, half of the blocks pruned
        _spmm8("spmm8_4096_37_tokens_half", 4096, 4096, 37, 4, 4, 0.5, True, True),
        # a lowered 14x14 convolution of an incomplete batch, 2:4 inside a quarter of the blocks, activations as [k, pixels]
        _spmm8("spmm8_512x4608_6076_pixels", 512, 4608, 31 * 14 * 14, 2, 4, 0.25, False, True),
        # 8192 tokens of prompts through a 4096 x 4096 layer
        _spmm8("spmm8_4096_8192_tokens", 4096, 4096, 8192, 4, 4, 1.0, True),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def draw(rng):
    kind = rng.choice(["adamw", "adamw", "encode8", "spmm8", "spmm8"])
    n, m = rng.choice([(2, 4), (4, 4), (1, 4), (2, 8), (4, 8)])
    keep = rng.choice([1.0, 0.5, 0.25, rng.uniform(0.1, 1.0)])
    if kind == "adamw":
        count, total, shapes = _log(rng, 1, 60), _log(rng, 1 << 10, 1 << 26), []
        for _ in range(count):
            k = _log(rng, 1, 6000)
            rows = max(1, min(8192, int(total / count * rng.uniform(0.2, 1.8) / k)))
            shapes.append("%dx%d" % (rows, k))
        return {"kind": kind, "shapes": ",".join(shapes), "w32": rng.random() < 0.5, "g32": rng.random() < 0.5, "bits": rng.choice([8, 32]),
                "masked": rng.random() < 0.5, "n": n, "m": m, "block": rng.choice([32, 64, 128]), "keep": keep}
    if kind == "encode8":
        return {"kind": kind, "rows": _log(rng, 1, 5000), "k": _log(rng, 1, 5000), "n": n, "m": m, "keep": keep}
    return {"kind": kind, "rows": _log(rng, 8, 5000), "k": _log(rng, 16, 5000), "ncols": _log(rng, 1, 5000), "n": n, "m": m, "keep": keep,
            "tokens": rng.random() < 0.5, "bias": rng.random() < 0.5}


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _places(shapes):
    """Where each tensor begins in the flat buffers (a multiple of 128 elements), and where the last one ends."""
    at = [0]
    for rows, k in shapes:
        at.append(at[-1] + (rows * k + 127) // 128 * 128)
    return at


# ------------------------------------------------------------------------------------------------------------------ inputs

def _mask(rows, k, n, m, block_rows, block_k, keep, weights, rng):
    """A saliency whose mask is known: the kept blocks' is 2^20 times the others'.  -> saliency, mask of booleans"""
    nrt, nblk = -(-rows // block_rows), -(-k // block_k)
    kept = int(math.floor(keep * nblk + 0.5))
    order = torch.rand(nrt, nblk, device="cuda", generator=rng).argsort(1).argsort(1) < kept
    inside = order.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(block_k, 1)[:, :k]
    s = weights.float().abs() * (0.5 + torch.rand(rows, k, device="cuda", generator=rng)) + 1e-6 * (1 + torch.rand(rows, k, device="cuda", generator=rng))
    groups = torch.nn.functional.pad(s, (0, -k % m)).view(rows, -1, m)
    best = torch.zeros(groups.shape, dtype=torch.bool, device="cuda").scatter_(2, groups.topk(n, 2).indices, True).view(rows, -1)[:, :k]
    return torch.where(inside, s * 2.0**20, s), inside & best


def _layer(case, rows, k, block_rows, block_k, saliency):
    from paper_2311_14272_b200 import binding as B
    return B.HybridLayer(rows, k, case["n"], case["m"], block_rows, block_k, case["keep"]).build_mask(saliency)


def prepare(case, seed):
    rng = torch.Generator(device="cuda")
    rng.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=rng)  # noqa: E731
    if case["kind"] == "adamw":
        return _prepare_adamw(case, seed, rng, randn)
    rows, k = case["rows"], case["k"]
    w = (randn(rows, k) * 0.02).bfloat16()
    saliency, mask = _mask(rows, k, case["n"], case["m"], 128, 128, case["keep"], w, rng)
    state = {"kind": case["kind"], "rows": rows, "k": k, "w": w, "mask": mask}
    if own:
        state["layer"] = _layer(case, rows, k, 128, 128, saliency)
    if case["kind"] == "encode8":
        return state
    # columns of different size, as tokens have them, with a few large features
    ncols = case["ncols"]
    x = randn(k, ncols) * torch.exp(randn(1, ncols) * 0.5) * torch.where(torch.rand(k, 1, device="cuda", generator=rng) < 0.01, 20.0, 1.0)
    x = x.bfloat16()
    state["x"] = x.t().contiguous() if case["tokens"] else x
    state["tokens"] = case["tokens"]
    state["bias"] = randn(rows) if case["bias"] else None
    state["codes"], state["scale"] = _weight_codes(w, mask)
    if own:
        state["layer"].encode8(w)
        if case["bias"]:
            state["layer"].set_epilogue8(state["bias"], relu=True)
    return state


def _prepare_adamw(case, seed, rng, randn):
    shapes = _shapes(case)
    at = _places(shapes)
    total = at[-1]
    real = torch.zeros(total, dtype=torch.bool, device="cuda")
    mask = torch.ones(total, dtype=torch.bool, device="cuda")
    index = torch.zeros(total, dtype=torch.int64, device="cuda")
    tensor = torch.zeros(total, dtype=torch.int64, device="cuda")
    layers = []
    weights = randn(total) * 0.05
    for i, (rows, k) in enumerate(shapes):
        here = slice(at[i], at[i] + rows * k)
        real[here] = True
        index[here] = torch.arange(rows * k, device="cuda")
        tensor[here] = i
        if case["masked"] and rows > 1:
            saliency, bits = _mask(rows, k, case["n"], case["m"], case["block"], case["block"], case["keep"], weights[here].view(rows, k), rng)
            mask[here] = bits.reshape(-1)
            layers.append(_layer(case, rows, k, case["block"], case["block"], saliency) if own else None)
        else:
            layers.append(None)
    inside = real & mask
    weights = torch.where(inside, weights, 0.0)
    # the state of a training that is under way; gradients of different size in different places, some of them zero
    size = torch.exp(randn(total) * 1.5) * 1e-2
    m = torch.where(inside, randn(total) * size * 0.3, 0.0)
    root = torch.where(inside, size * (0.5 + torch.rand(total, device="cuda", generator=rng)), 0.0)
    grad = torch.where(real & (torch.rand(total, device="cuda", generator=rng) > 0.02), randn(total) * size, 0.0)
    state = {"kind": "adamw", "bits": case["bits"], "w32": case["w32"], "seed": seed % 1000003, "step": 9, "mask": mask, "index": index, "tensor": tensor,
             "w": weights if case["w32"] else weights.bfloat16(), "grad": grad if case["g32"] else grad.bfloat16()}
    if case["w32"]:
        state["copy"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    if case["bits"] == 32:
        state["m"], state["v"] = m, root * root
    else:
        half = torch.full((total,), 1 << 18, dtype=torch.int32, device="cuda")
        state["m"], state["m_exp"] = _round_state(m, half * 2, False)
        state["v"], state["v_exp"] = _round_state(root, half, True)
    if own:
        from paper_2311_14272_b200 import binding as B
        views = lambda flat: [flat[at[i]:at[i] + rows * k].view(rows, k) for i, (rows, k) in enumerate(shapes)]  # noqa: E731
        opt = B.AdamW(views(state["w"]), copies=views(state["copy"]) if case["w32"] else None, masks=layers, lr=LR, betas=(BETA1, BETA2), eps=EPS,
                      weight_decay=DECAY, state_bits=case["bits"], seed=state["seed"], step=state["step"])
        for name in ("m", "v", "m_exp", "v_exp"):
            if name in state:
                getattr(opt, name).copy_(state[name])
        state["opt"], state["grads"] = opt, views(state["grad"])
    return state


# -------------------------------------------------------------------------------------------------------------- plain forms

def _scale_exponent(largest, top):
    """The smallest E with largest <= top * 2^E, top = f * 2^8 and 1 <= f < 2 (at least -126: what is smaller is held less finely)."""
    fraction, exponent = torch.frexp(largest)
    e = exponent - 9 + (fraction * 2 > top / 256).int()
    return torch.where(largest > 0, e, -126).clamp(-126, 127)


def _power(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def _weight_codes(w, mask):
    """e4m3 codes [rows, k] and the exponent of each 128 x 128 block [row tiles, k-blocks]."""
    rows, k = w.shape
    w = torch.nn.functional.pad(torch.where(mask, w.float(), 0.0), (0, -k % 128, 0, -rows % 128))
    blocks = w.view(w.shape[0] // 128, 128, w.shape[1] // 128, 128)
    e = _scale_exponent(blocks.abs().amax((1, 3)), 448.0)
    codes = (blocks * _power(-e)[:, None, :, None]).to(torch.float8_e4m3fn)
    return codes.view(w.shape)[:rows, :k].contiguous(), e


def _weight_values(codes, e):
    rows, k = codes.shape
    return codes.float() * _power(e).repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :k]


def _activation_values(x):
    """x [ncols, k] as its 8-bit form holds it."""
    ncols, k = x.shape
    blocks = torch.nn.functional.pad(x.float(), (0, -k % 128)).view(ncols, -1, 128)
    e = _scale_exponent(blocks.abs().amax(2, keepdim=True), 448.0)
    return ((blocks * _power(-e)).to(torch.float8_e4m3fn).float() * _power(e)).view(ncols, -1)[:, :k]


def _mix(h):
    """A bijection of 32-bit numbers that spreads every bit over all (xorshift-multiply, "lowbias32")."""
    h = h ^ (h >> 16)
    h = (h * 0x7FEB352D) & M32
    h = h ^ (h >> 15)
    h = (h * 0x846CA68B) & M32
    return h ^ (h >> 16)


def _hash(seed, step, tensor, index):
    key = _mix(_mix(_mix(_mix(seed & M32) ^ (seed >> 32)) ^ (step & M32)) ^ tensor)
    return _mix((index & M32) ^ _mix((index >> 32) ^ key))


def _round_state(x, random, root):
    """Codes (uint8) and biased exponents (uint8, one for each 128) of a flat state; random: an integer an element, in units of the last bit of the 20
    (root: 19) below the code.  root: e4m4 without a sign, not 0."""
    blocks, random = x.view(-1, 128), random.view(-1, 128)
    e = _scale_exponent(blocks.abs().amax(1, keepdim=True), 496.0 if root else 448.0)
    bits = (blocks.abs() * _power(-e) * 2.0**-120).view(torch.int32)       # exponent field as the code has it, 19 or 20 bits of fraction below
    if root:
        codes = torch.where(blocks > 0, ((bits + random) >> 19).clamp(min=1), 0)
    else:
        codes = ((bits + random) >> 20) | torch.where(blocks < 0, 128, 0)
    return codes.to(torch.uint8).view(-1), (e + 127).to(torch.uint8).view(-1)


def _state_values(codes, e, root):
    c = codes.view(-1, 128).int()
    scale = _power(e.view(-1, 1).int() - 127)
    if root:
        return ((c << 19).view(torch.float32) * 2.0**120 * scale).view(-1)
    return (torch.where(c >= 128, -1.0, 1.0) * ((c & 127) << 20).view(torch.float32) * 2.0**120 * scale).view(-1)


def _plain_adamw(s):
    s["step"] += 1
    t, narrow = s["step"], s["bits"] == 8
    grad = s["grad"].float()
    m = _state_values(s["m"], s["m_exp"], False) if narrow else s["m"]
    v = _state_values(s["v"], s["v_exp"], True).square() if narrow else s["v"]
    m = m * BETA1 + grad * (1 - BETA1)
    v = v * BETA2 + grad * grad * (1 - BETA2)
    w = s["w"].float() * (1 - LR * DECAY) - LR / (1 - BETA1**t) * (m / (v.sqrt() / math.sqrt(1 - BETA2**t) + EPS))
    m, v, w = (torch.where(s["mask"], q, 0.0) for q in (m, v, w))
    h = _hash(s["seed"], t, s["tensor"], s["index"]) if narrow or not s["w32"] else None
    if s["w32"]:
        s["w"].copy_(w)
        s["copy"].copy_(w)
        out = [s["w"], s["copy"]]
    else:
        up = (((h >> 21) << 5) + 16).int()
        s["w"].copy_(((w.view(torch.int32) + up) & -65536).view(torch.float32))
        out = [s["w"]]
    if not narrow:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return out + [s["m"], s["v"]]
    s["m"], s["m_exp"] = _round_state(m, (((h & 0x3FF) << 10) + 512).int(), False)
    s["v"], s["v_exp"] = _round_state(v.sqrt(), (((h >> 10 & 0x7FF) << 8) + 128).int(), True)
    return out + [_state_values(s["m"], s["m_exp"], False).bfloat16(), _state_values(s["v"], s["v_exp"], True).bfloat16()]


def run(s):
    if s["kind"] == "adamw":
        if not own:
            return _plain_adamw(s)
        s["opt"].step(s["grads"])
        states = [s["opt"].m, s["opt"].v] if s["bits"] == 32 else list(s["opt"].moments())
        return [s["w"]] + ([s["copy"]] if s["w32"] else []) + states
    if s["kind"] == "encode8":
        if own:
            return s["layer"].encode8(s["w"]).decode8()
        return _weight_values(*_weight_codes(s["w"], s["mask"])).bfloat16()
    if own:
        return s["layer"].spmm8(s["x"], tokens=s["tokens"])
    w = _weight_values(s["codes"], s["scale"])
    x = _activation_values(s["x"] if s["tokens"] else s["x"].t())
    y = x @ w.t() if s["tokens"] else w @ x.t()
    if s["bias"] is not None:
        y = (y + (s["bias"] if s["tokens"] else s["bias"][:, None])).clamp(min=0)
    return y.bfloat16()


# --------------------------------------------------------------------------------------------------------------------- work

def work(case):
    if case["kind"] == "adamw":
        count = sum(rows * k for rows, k in _shapes(case))
        wide = case["bits"] == 32
        each = 2 * (4 if case["w32"] else 2) + (2 if case["w32"] else 0) + (4 if case["g32"] else 2) + (16 if wide else 4 + 4 / 128)
        masked = sum(rows * k for rows, k in _shapes(case) if rows > 1) if case["masked"] else 0
        # 8-bit states come back as the bf16 values that they stand for, too
        return {"bytes": count * (each + (0 if wide else 4)) + masked / 8, "flops": 15.0 * count}
    rows, k = case["rows"], case["k"]
    nblk = -(-k // 128)
    share = math.floor(case["keep"] * nblk + 0.5) / nblk
    kept = rows * k * share * case["n"] / case["m"]
    if case["kind"] == "encode8":
        # the weights under the mask, its bits, the codes; and the dense bf16 matrix that they stand for
        return {"bytes": 2 * kept + rows * k / 8 + kept + 2.0 * rows * k, "flops": 2.0 * kept}
    ncols = case["ncols"]
    return {"bytes": kept + 2.0 * ncols * k * min(1.0, share * -(-rows // 128)) + 2.0 * rows * ncols, "flops": 2.0 * kept * ncols}


# ------------------------------------------------------------------------------------------------------------ in 64 bits

def _held(x, largest, fraction_bits, top, random=None, never_zero=False):
    """x (64 bits) as code * 2^E: E from the block's largest value, codes with a spacing of 2^(exponent - fraction_bits) down to exponent -6; nearest
    even, or up with the chance that the part below the code says (random in [0, 1))."""
    e = torch.where(largest > 0, torch.ceil(torch.log2(largest.clamp(min=1e-300) / top)), -126.0)
    e = torch.where(largest > top * torch.exp2(e), e + 1, e)
    e = torch.where(largest <= top * torch.exp2(e - 1), e - 1, e).clamp(-126, 127)
    y = x.abs() * torch.exp2(-e)
    _, exponent = torch.frexp(y)
    spacing = torch.exp2((exponent - 1).clamp(min=-6).double() - fraction_bits)
    code = torch.round(y / spacing) if random is None else torch.floor(y / spacing + random)
    if never_zero:
        code = torch.where((y > 0) & (code == 0), 1.0, code)
    return torch.sign(x) * code * spacing * torch.exp2(e)


def _exact_blocks(x, random, root):
    x = x.view(-1, 128)
    return _held(x, x.abs().amax(1, keepdim=True), 4 if root else 3, 496.0 if root else 448.0, random.view(-1, 128), root).view(-1)


def _exact_adamw(s):
    t, narrow = s["step"] + 1, s["bits"] == 8
    grad = s["grad"].double()
    if narrow:
        # codes stand for: sign, exponent, fraction
        c = s["m"].view(-1, 128).long()
        field, part = (c >> 3) & 15, (c & 7).double()
        size = torch.where(field > 0, (1 + part / 8) * torch.exp2(field.double() - 7), part / 8 * 2.0**-6)
        m = (torch.where(c > 127, -size, size) * torch.exp2(s["m_exp"].view(-1, 1).double() - 127)).view(-1)
        c = s["v"].view(-1, 128).long()
        field, part = c >> 4, (c & 15).double()
        size = torch.where(field > 0, (1 + part / 16) * torch.exp2(field.double() - 7), part / 16 * 2.0**-6)
        v = (size * torch.exp2(s["v_exp"].view(-1, 1).double() - 127)).view(-1) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m = BETA1 * m + (1 - BETA1) * grad
    v = BETA2 * v + (1 - BETA2) * grad**2
    step = (m / (1 - BETA1**t)) / (torch.sqrt(v / (1 - BETA2**t)) + EPS)
    w = s["w"].double()
    w = w - LR * DECAY * w - LR * step
    m, v, w = m * s["mask"], v * s["mask"], w * s["mask"]
    if narrow or not s["w32"]:
        number = [int(q) for q in (s["seed"] & M32, s["seed"] >> 32, t)]
        word = lambda h: ((((h ^ (h >> 16)) * 0x7FEB352D) & M32))  # noqa: E731
        spread = lambda h: (lambda a: (lambda b: b ^ (b >> 16))(((a ^ (a >> 15)) * 0x846CA68B) & M32))(word(h))  # noqa: E731
        key = spread(spread(spread(number[0]) ^ number[1]) ^ number[2])
        h = spread((s["index"] % 2**32) ^ spread((s["index"] // 2**32) ^ spread(key ^ s["tensor"])))
    if s["w32"]:
        out = [w, w]
    else:
        _, exponent = torch.frexp(w)
        spacing = torch.exp2((exponent - 1).double() - 7)
        out = [torch.sign(w) * torch.floor(w.abs() / spacing + (2 * (h // 2**21) + 1).double() / 4096) * spacing]
    if not narrow:
        return out + [m, v]
    return out + [_exact_blocks(m, (2 * (h % 1024) + 1).double() / 2048, False), _exact_blocks(torch.sqrt(v), (2 * (h // 1024 % 2048) + 1).double() / 4096, True)]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    rows, k = case["rows"], case["k"]
    w = torch.zeros(-(-rows // 128) * 128, -(-k // 128) * 128, dtype=torch.float64, device="cuda")
    w[:rows, :k] = s["w"].double() * s["mask"]
    largest = torch.nn.functional.max_pool2d(w.abs()[None], 128)[0]
    w = _held(w, torch.kron(largest, torch.ones(128, 128, dtype=torch.float64, device="cuda")), 3, 448.0)[:rows, :k]
    if case["kind"] == "encode8":
        return w
    x = (s["x"].t() if case["tokens"] else s["x"]).double()
    x = torch.cat([x, torch.zeros(-k % 128, x.shape[1], dtype=torch.float64, device="cuda")])
    x = x.reshape(-1, 128, x.shape[1])
    x = _held(x, x.abs().amax(1, keepdim=True), 3, 448.0).reshape(-1, x.shape[2])[:k]
    y = w @ x
    if s["bias"] is not None:
        y = torch.relu(y + s["bias"].double()[:, None])
    return y.t().contiguous() if case["tokens"] else y
