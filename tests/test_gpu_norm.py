"""Group norm with an activation on the GPU against the same in 64 bits (norm_reference.py says where the tolerances come from); results in 16 bits add half a step,
finfo.eps / 2 of the value.  The gradient also against differences of the forward pass."""
import numpy as np
import pytest

import block8_reference as held
import norm_reference as ref
from paper_2311_14272_b200 import workloads as wl

pytestmark = pytest.mark.gpu

# batch, pixels, channels, groups: one value; one a group; odd ones, groups that a thread's channels meet; one slice, many; clusters; one large image and groups of more
# channels than a CTA holds (two kernels)
SIZES = [(1, 1, 1, 1), (2, 1, 8, 8), (2, 7, 40, 5), (1, 49, 1280, 32), (3, 100, 24, 3), (2, 17, 25, 5), (2, 33, 26, 13), (1, 3000, 64, 32), (4, 784, 512, 32),
         (2, 5, 4100, 2), (1, 9, 5000, 1), (1, 50176, 64, 32), (1, 20000, 20, 4), (33, 10, 96, 32), (5, 200, 256, 256)]
TYPES = ["bf16", "fp16", "fp32"]
ACTS = ["none", "relu", "relu6", "silu"]


def kind(torch, name):
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def numbers(t):
    return t.detach().double().cpu().numpy()


def padded(torch, a, dtype, pitch, odd):
    """a [batch, pixels, channels] with `pitch` elements between pixels that are not its own (7s), `odd` elements from an aligned address"""
    batch, pixels, channels = a.shape
    whole = torch.full((batch * pixels * (channels + pitch) + odd,), 7.0, dtype=dtype, device="cuda")
    t = whole[odd:].view(batch, pixels, channels + pitch)[:, :, :channels]
    t.copy_(torch.from_numpy(a))
    return t, whole


def inputs(torch, batch, pixels, channels, groups, seed, mean=0.5):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((batch, pixels, channels)) * np.exp(rng.standard_normal(channels) * 0.3) + mean * rng.standard_normal(channels)
    gamma, beta = (1 + 0.3 * rng.standard_normal(channels)).astype(np.float32), (0.4 * rng.standard_normal(channels)).astype(np.float32)
    dy = rng.standard_normal((batch, pixels, channels)) * np.exp(rng.standard_normal((batch, 1, 1)))
    return x, gamma, beta, dy


def cuda(torch, a):
    return torch.from_numpy(a).cuda()


def check(got, want, tol, dtype, torch):
    tol = tol + (0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2 * (np.abs(want) + tol)) + (2.0**-25 if dtype == torch.float16 else 1e-37)
    if dtype == torch.float16:                                               # (65504 is its largest; what is 65520 or more rounds to infinity)
        over = np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + tol >= 65520)
        got = np.where(over, want, got)
    off = np.abs(got - want)
    assert np.all(off <= tol), (float((off / tol).max()), np.unravel_index(np.argmax(off / tol), off.shape))


def outside(whole, shape, pitch, odd):
    batch, pixels, channels = shape
    rest = whole[odd:].view(batch, pixels, channels + pitch)[:, :, channels:]
    return bool((rest == 7.0).all() and (whole[:odd] == 7.0).all())


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pitch,odd", [(0, 0), (8, 0), (3, 1)])
def test_forward_and_backward(size, dtype, pitch, odd):
    import torch
    from paper_2311_14272_b200 import binding as B
    batch, pixels, channels, groups = size
    T = kind(torch, dtype)
    for i, act in enumerate(ACTS):
        x, gamma, beta, dy = inputs(torch, *size, seed=i)
        d_x, _ = padded(torch, x, T, pitch, odd)
        d_dy, _ = padded(torch, dy, T, pitch, odd)
        x, dy = numbers(d_x), numbers(d_dy)
        plain = i == 0                                                       # without weight and bias
        norm = B.GroupNorm(channels, groups, None if plain else cuda(torch, gamma), None if plain else cuda(torch, beta), eps=1e-4, activation=act)
        g, b = (np.ones(channels), np.zeros(channels)) if plain else (gamma.astype(np.float64), beta.astype(np.float64))
        d_y, whole = padded(torch, np.zeros(x.shape), T, pitch, odd)
        done = norm.forward(d_x, y=d_y)
        y, mean, rstd, tol = ref.forward(x, groups, g, b, 1e-4, act, dtype == "fp32")
        check(numbers(done.y), y, tol, T, torch)
        assert done.y is d_y and outside(whole, x.shape, pitch, odd)
        s = numbers(done.statistics)
        far = np.abs(ref.grouped(x, groups) - mean[:, None, :, None]).max((1, 3))
        assert np.all(np.abs(s[..., 0] - mean) <= ref.U * (16 * far + 4 * np.abs(mean)) + 1e-37)
        assert np.all(np.abs(s[..., 1] / rstd - 1) <= 48 * ref.U)
        d_dx, whole = padded(torch, np.zeros(x.shape), T, pitch, odd)
        dx, dgamma, dbeta = norm.backward(d_dy, d_x, done.statistics, dx=d_dx)
        want = ref.backward(dy, x, s[..., 0], s[..., 1], groups, g, b, act, dtype == "fp32")
        check(numbers(dx), want[0], want[3], T, torch)
        assert dx is d_dx and outside(whole, x.shape, pitch, odd)
        check(numbers(dgamma), want[1], want[4], torch.float32, torch)
        check(numbers(dbeta), want[2], want[5], torch.float32, torch)
        # the same again, to the bit
        again, both = norm.forward(d_x), norm.backward(d_dy, d_x, done.statistics)
        assert torch.equal(again.y, done.y) and torch.equal(again.statistics, done.statistics)
        assert all(torch.equal(p, q) for p, q in zip(both, (dx, dgamma, dbeta)))


def held_rows(a):
    return held.activations(a.T).T


@pytest.mark.parametrize("size", SIZES + [(1, 9, 128, 4), (3, 41, 384, 6), (2, 50, 136, 17)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pitch,odd", [(0, 0), (3, 1)])
def test_8_bit_forms(size, dtype, pitch, odd):
    """x in 8 bits is what quantize8 makes of it; y in 8 bits stands for y; the backward pass from x in 8 bits is that of the values that it stands for."""
    import torch
    from paper_2311_14272_b200 import binding as B
    batch, pixels, channels, groups = size
    T = kind(torch, dtype)
    x, gamma, beta, dy = inputs(torch, *size, seed=5)
    d_x, _ = padded(torch, x, T, pitch, odd)
    d_dy, _ = padded(torch, dy, T, pitch, odd)
    x, dy = numbers(d_x), numbers(d_dy)
    for act in ("relu6", "silu"):
        norm = B.GroupNorm(channels, groups, cuda(torch, gamma), cuda(torch, beta), activation=act)
        done = norm.forward(d_x, keep_x=True, keep_y=True)
        alone = norm.forward(d_x, keep_y=True, plain_y=False)
        assert alone.y is None and alone.x8 is None
        values = held_rows(x.reshape(-1, channels))
        assert np.array_equal(numbers(done.x8.dequantize(tokens=True)), values)
        y, _, _, tol = ref.forward(x, groups, gamma.astype(np.float64), beta.astype(np.float64), 1e-5, act, dtype == "fp32")
        check(numbers(done.y), y, tol, T, torch)
        y, tol = y.reshape(-1, channels), tol.reshape(-1, channels)
        blocks = np.pad(np.abs(y) + tol, ((0, 0), (0, -channels % 128))).reshape(len(y), -1, 128).max(2)
        least = np.repeat(2.0**np.vectorize(held.exponent)(blocks).astype(np.float64), 128, 1)[:, :channels]
        for q in (done.y8, alone.y8):
            off = np.abs(numbers(q.dequantize(tokens=True)) - y)
            assert np.all(off <= 2.0**-4 * np.abs(y) + 2.0**-10 * least + 2 * tol), float(off.max())
            assert np.array_equal(numbers(q.dequantize()), numbers(q.dequantize(tokens=True)).T)
        s = numbers(done.statistics)
        got = norm.backward(d_dy, done.x8, done.statistics)
        want = ref.backward(dy, values.reshape(x.shape), s[..., 0], s[..., 1], groups, gamma.astype(np.float64), beta.astype(np.float64), act, dtype == "fp32")
        check(numbers(got[0]), want[0], want[3], T, torch)
        check(numbers(got[1]), want[1], want[4], torch.float32, torch)
        check(numbers(got[2]), want[2], want[5], torch.float32, torch)


def test_the_8_bit_form_of_x_is_quantize8s():
    import torch
    from paper_2311_14272_b200 import binding as B
    for channels, pixels in ((256, 64), (100, 37), (128, 8)):
        x = torch.randn(2, pixels, channels, device="cuda").bfloat16()
        x[0, 3, 5], x[1, 2, 7] = float("inf"), float("nan")
        one, two = B.quantize8(x.view(-1, channels), tokens=True), B.GroupNorm(channels, 4).forward(x, keep_x=True).x8
        a, b = one.dequantize(), two.dequantize()
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
        assert a.isnan().sum() == 2


@pytest.mark.parametrize("dtype", TYPES)
def test_a_mean_far_from_zero(dtype):
    """Values about 300 with a spread of 1 (as far as the type holds it): the variance is theirs, not that of roundings.  And a first value far from the others."""
    import torch
    from paper_2311_14272_b200 import binding as B
    T = kind(torch, dtype)
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 500, 32)) * (4 if dtype == "bf16" else 1) + 300
    x[1] -= 300
    x[1, 0] = 1000
    d_x = torch.from_numpy(x).to("cuda", T)
    x = numbers(d_x)
    done = B.GroupNorm(32, 4, eps=0.0).forward(d_x)
    y, mean, rstd, tol = ref.forward(x, 4, 1.0, 0.0, 0.0, "none", dtype == "fp32")
    check(numbers(done.y), y, tol, T, torch)
    assert np.all(np.abs(numbers(done.statistics)[..., 1] / rstd - 1) <= 48 * ref.U)


def test_equal_values_and_what_is_not_finite():
    import torch
    from paper_2311_14272_b200 import binding as B
    x = torch.full((1, 40, 64), 3.0, device="cuda", dtype=torch.bfloat16)
    norm = B.GroupNorm(64, 8, bias=torch.full((64,), 0.5, device="cuda"))
    done = norm.forward(x)
    assert torch.all(done.y == 0.5) and torch.all(done.statistics[..., 0] == 3.0)
    x[0, 7, 9] = float("inf")
    x[0, 9, 17] = float("nan")
    done = norm.forward(x, keep_y=True)
    bad = torch.zeros(64, dtype=torch.bool, device="cuda")
    bad[8:24] = True                                                         # the two groups, and no other
    assert torch.equal(done.y[0].isnan(), bad.expand(40, 64)) and torch.all(done.y[0][:, ~bad] == 0.5)
    assert torch.equal(done.y8.dequantize(tokens=True).isnan(), bad.expand(40, 64))


@pytest.mark.parametrize("act", ["relu", "relu6"])
def test_values_on_a_border(act):
    """p is exactly 0 (and 6): the slope there is 0, as the formula in 64 bits has it."""
    import torch
    from paper_2311_14272_b200 import binding as B
    x = torch.tensor([-1.0, 1.0] * 64, device="cuda").view(1, 128, 1).expand(1, 128, 8).contiguous()
    stats = torch.tensor([0.0, 1.0], device="cuda").expand(1, 8, 2).contiguous()
    gamma, beta = torch.tensor([1.0, 3.0, 1.0, 0.1, 2.0, 3.0, 5.0, 7.0], device="cuda"), torch.tensor([1.0, 3.0, -1.0, 0.1, 4.0, -3.0, 1.0, 1.0], device="cuda")
    dx, dg, db = B.GroupNorm(8, 8, gamma, beta, activation=act).backward(torch.ones_like(x), x, stats)
    want = ref.backward(np.ones((1, 128, 8)), numbers(x), np.zeros((1, 8)), np.ones((1, 8)), 8, numbers(gamma), numbers(beta), act, True)
    check(numbers(db), want[2], want[5], torch.float32, torch)
    check(numbers(dx), want[0], want[3], torch.float32, torch)


def test_gradient_against_differences():
    """sum(dy y) along a direction, by central differences of the forward pass in fp32: the statistics' part of the gradient is in it."""
    import torch
    from paper_2311_14272_b200 import binding as B
    torch.manual_seed(0)
    x, dy, way = (torch.randn(2, 6, 5, 24, device="cuda") for _ in range(3))
    gamma, beta = 1 + 0.2 * torch.randn(24, device="cuda"), torch.randn(24, device="cuda")
    norm = B.GroupNorm(24, 3, gamma, beta, activation="silu")
    value = lambda t: (norm.forward(t).y.double() * dy.double()).sum().item()  # noqa: E731
    step = 2.0**-7
    slope = (value(x + step * way) - value(x - step * way)) / (2 * step)
    dx, dg, db = norm.backward(dy, x, norm.forward(x).statistics)
    # third derivatives of a sum of 1440 terms of size one, times step^2 / 6 = 1e-5, and y's roundings (1440^0.5 2^-24 / step = 3e-4)
    assert abs(slope - (dx.double() * way.double()).sum().item()) <= 2e-2
    for p, g in ((gamma, dg), (beta, db)):
        d = torch.randn(24, device="cuda")
        old = p.clone()
        p.copy_(old + step * d)
        up = value(x)
        p.copy_(old - step * d)
        down = value(x)
        p.copy_(old)
        assert abs((up - down) / (2 * step) - (g.double() * d.double()).sum().item()) <= 2e-2


def test_in_place():
    import torch
    from paper_2311_14272_b200 import binding as B
    for shape in ((4, 28, 28, 128), (1, 224, 224, 32)):                      # one kernel, and two
        x, dy = (torch.randn(shape, device="cuda").bfloat16() for _ in range(2))
        norm = B.GroupNorm(shape[-1], 8, activation="relu")
        done = norm.forward(x)
        want = norm.backward(dy, x, done.statistics)
        for place in ("dy", "x"):
            a, b = x.clone(), dy.clone()
            assert torch.equal(norm.backward(b, a, done.statistics, dx=b if place == "dy" else a)[0], want[0])
        assert torch.equal(norm.forward(x, y=x).y, done.y) and torch.equal(x, done.y)


def test_shapes_and_empty_batches():
    import torch
    from paper_2311_14272_b200 import binding as B
    norm = B.GroupNorm(32, 4)
    x = torch.randn(3, 4, 5, 64, device="cuda").bfloat16()
    for t in (x[..., 32:], x[..., :32].contiguous(), x[:, :, :, :32][:1], x[1:2, 2:3, :, 32:], x[:, 0, 0, :32].contiguous()):
        y = norm.forward(t).y
        assert y.shape == t.shape and torch.equal(y, norm.forward(t.contiguous()).y)
    with pytest.raises(AssertionError):
        norm.forward(x[:, :, 1:, :32])
    empty = x[:0, :, :, :32]
    done = norm.forward(empty)
    assert done.y.shape == empty.shape and done.statistics.shape == (0, 4, 2)
    dx, dg, db = norm.backward(empty, empty, done.statistics)
    assert dx.shape == empty.shape and not dg.any() and not db.any()


def test_streams_and_graphs():
    import torch
    from paper_2311_14272_b200 import binding as B
    x, dy = (torch.randn(2, 56, 56, 64, device="cuda").bfloat16() for _ in range(2))
    norm = B.GroupNorm(64, 32, torch.rand(64, device="cuda"), torch.rand(64, device="cuda"), activation="relu")
    done = norm.forward(x, keep_x=True)
    want = norm.backward(dy, done.x8, done.statistics)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = norm.forward(x, keep_x=True, stream=side)
    back = norm.backward(dy, other.x8, other.statistics, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(other.y, done.y) and all(torch.equal(a, b) for a, b in zip(back, want))
    graphs = []
    for _ in range(2):                                                       # two graphs, replayed in turn and then together
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            one = norm.forward(x, keep_x=True)
            got = norm.backward(dy, one.x8, one.statistics)
        graphs.append((g, one, got))
    x.copy_(torch.randn_like(x))
    done = norm.forward(x, keep_x=True)
    want = norm.backward(dy, done.x8, done.statistics)
    torch.cuda.synchronize()
    for (g, _, _), s in zip(graphs, (torch.cuda.Stream(), torch.cuda.Stream())):
        with torch.cuda.stream(s):
            for _ in range(3):
                g.replay()
    torch.cuda.synchronize()
    for _, one, got in graphs:
        assert torch.equal(one.y, done.y) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_pixels_beyond_32_bits():
    """Offsets of more than 2^31 elements, in tensors and in the 8-bit form."""
    import torch
    from paper_2311_14272_b200 import binding as B
    batch, pixels, channels = 3, 1 << 18, 2944
    x = torch.empty(batch, pixels, channels, dtype=torch.bfloat16, device="cuda")
    for b in range(batch):
        x[b].normal_(b, 1 + b)
    norm = B.GroupNorm(channels, 23, activation="relu")
    done = norm.forward(x, keep_x=True)
    alone = norm.forward(x[-1:], keep_x=True)
    # (a batch of one is cut otherwise: sums of another order.  Two values next to a border of bf16's rounding, however near, may be a step apart: 2^(e - 7) for values from 2^e on,
    # at most 2^-7 of the value)
    near = lambda a, b: (a.float() - b.float()).abs().max().item() <= 2.0**-7 * b.float().abs().max().item()  # noqa: E731
    assert near(done.y[-1:], alone.y) and near(done.statistics[-1:], alone.statistics)
    part = B.quantize8(x[-1, -64:], tokens=True).dequantize(tokens=True)
    assert torch.equal(done.x8.dequantize(tokens=True)[-64:], part)
    del alone
    dx, dg, db = norm.backward(done.y, x, done.statistics)
    assert near(dx[-1:], norm.backward(done.y[-1:], x[-1:], done.statistics[-1:])[0])


@pytest.mark.parametrize("size", [(2, 4000, 384, 6), (1, 5000, 640, 40), (1, 1600, 2048, 32), (3, 1100, 896, 7), (2, 9001, 128, 16)])
@pytest.mark.parametrize("dtype", TYPES)
def test_large_backward_passes_from_8_bits(size, dtype):
    """Two kernels, whose threads share the places that codes are fetched to; odd and even numbers of pixels at a time.  With statistics and parameters that put values on the borders, so
    that some threads of a block take another way than the others."""
    import torch
    from paper_2311_14272_b200 import binding as B
    batch, pixels, channels, groups = size
    T = kind(torch, dtype)
    rng = np.random.default_rng(channels)
    values = held_rows(np.round(rng.standard_normal((batch * pixels, channels)) * 2) / 2)           # (multiples of 1/2: exact in 8 bits)
    d_x = cuda(torch, np.ascontiguousarray(values).reshape(batch, pixels, channels)).to(T)
    x = numbers(d_x)
    dy = cuda(torch, rng.standard_normal(x.shape)).to(T)
    gamma, beta = rng.choice([1.0, 2.0, 3.0, 0.5], channels).astype(np.float32), rng.choice([0.0, 1.0, -0.5, 3.0, 5.0], channels).astype(np.float32)
    stats = np.stack([np.zeros((batch, groups)), np.ones((batch, groups))], 2).astype(np.float32)
    given = B.quantize8(d_x.bfloat16().view(-1, channels), tokens=True)
    assert np.array_equal(numbers(given.dequantize(tokens=True)).reshape(x.shape), x)
    for act in ("relu", "relu6", "silu"):
        norm = B.GroupNorm(channels, groups, cuda(torch, gamma), cuda(torch, beta), activation=act)
        got = norm.backward(dy, given, cuda(torch, stats))
        want = ref.backward(numbers(dy), x, stats[..., 0].astype(np.float64), stats[..., 1].astype(np.float64), groups, gamma.astype(np.float64), beta.astype(np.float64), act, dtype == "fp32")
        check(numbers(got[0]), want[0], want[3], T, torch)
        check(numbers(got[1]), want[1], want[4], torch.float32, torch)
        check(numbers(got[2]), want[2], want[5], torch.float32, torch)
        assert all(torch.equal(a, b) for a, b in zip(got, norm.backward(dy, given, cuda(torch, stats))))


# batch, pixels, channels, groups: a thread's channels of one group, and of several; one kernel and two
@pytest.mark.parametrize("size", [(2, 300000, 64, 8), (2, 300000, 64, 32), (9, 50000, 48, 16), (1, 50176, 64, 8), (3, 9000, 20, 4)])
@pytest.mark.parametrize("dtype", TYPES)
def test_the_variance_behind_outliers(size, dtype):
    """Values far from the others where threads begin, wherever else, one and several of them; a border of zeros, and values about 100.  The variance is the formula's all the same."""
    import torch
    from paper_2311_14272_b200 import binding as B
    batch, pixels, channels, groups = size
    T, each = kind(torch, dtype), channels // groups
    rng = np.random.default_rng(pixels)
    x = rng.standard_normal((batch, pixels, channels)).astype(np.float32)
    far = [100, 300, 1000, 3000, -1000, 30000]
    for b in range(batch):
        for g in range(groups):
            at = x[b, :, g * each:(g + 1) * each]
            what = (b * groups + g) % 8
            if what < 6:
                at[0, 0] = far[what]
            elif what == 6:
                at[:3] = 1000 / (1 + np.arange(3)[:, None])                   # several, one behind the other
            else:
                at += 100
                at[:pixels // 50] = 0
            if g % 3 == 1:
                at[rng.integers(0, pixels, 5), rng.integers(0, each, 5)] = 700
    d_x = torch.from_numpy(x).to("cuda", T)
    norm = B.GroupNorm(channels, groups, eps=0.0)
    got = numbers(norm.forward(d_x).statistics)
    for b in range(batch):
        v = numbers(d_x[b]).reshape(pixels, groups, each)
        mean = v.mean((0, 2))
        rstd = 1 / np.sqrt(((v - mean[None, :, None])**2).mean((0, 2)))
        off = np.abs(v - mean[None, :, None]).max((0, 2))
        assert np.all(np.abs(got[b, :, 0] - mean) <= ref.U * (16 * off + 4 * np.abs(mean)))
        assert np.all(np.abs(got[b, :, 1] / rstd - 1) <= 48 * ref.U), (np.abs(got[b, :, 1] / rstd - 1) / ref.U).max()


@pytest.mark.parametrize("shape,groups", [((40000, 64), 8), ((32768, 2, 24), 3), ((70000, 128), 4), ((66000, 3, 8), 8)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_samples(shape, groups, dtype):
    """More samples than 32767, of a row or a few pixels each, from x as it is and from its 8-bit form."""
    import torch
    from paper_2311_14272_b200 import binding as B
    channels = shape[-1]
    size = (shape[0], int(np.prod(shape[1:-1], dtype=int)), channels, groups)
    x, gamma, beta, dy = inputs(torch, *size, seed=3)
    d_x, d_dy = (cuda(torch, a).to(kind(torch, dtype)).view(shape) for a in (x, dy))
    x, dy = (numbers(t).reshape(size[:3]) for t in (d_x, d_dy))
    norm = B.GroupNorm(channels, groups, cuda(torch, gamma), cuda(torch, beta), eps=1e-2, activation="relu")
    done = norm.forward(d_x, keep_x=True)
    y, _, _, tol = ref.forward(x, groups, gamma.astype(np.float64), beta.astype(np.float64), 1e-2, "relu", dtype == "fp32")
    check(numbers(done.y).reshape(x.shape), y, tol, d_x.dtype, torch)
    s = numbers(done.statistics)
    for given, values in ((d_x, x), (done.x8, held_rows(x.reshape(-1, channels)).reshape(x.shape))):
        dx, dg, db = norm.backward(d_dy, given, done.statistics)
        want = ref.backward(dy, values, s[..., 0], s[..., 1], groups, gamma.astype(np.float64), beta.astype(np.float64), "relu", dtype == "fp32")
        check(numbers(dx).reshape(x.shape), want[0], want[3], d_x.dtype, torch)
        check(numbers(dg), want[1], want[4], torch.float32, torch)
        check(numbers(db), want[2], want[5], torch.float32, torch)


@pytest.mark.parametrize("size", [(2, 1, 768, 64), (2, 300, 64, 8), (1, 40, 100, 25), (1, 70000, 96, 32), (3, 25000, 64, 4)])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_mean_that_is_many_deviations_from_zero(size, dtype):
    """Values about 3000, and groups of one value: results are the formula's at the statistics that the call itself leaves, with x - mean rounded once, not with roundings of mean times
    gamma / deviation (a group of -700 was off by 0.02 where y is the bias)."""
    import torch
    from paper_2311_14272_b200 import binding as B
    batch, pixels, channels, groups = size
    T = kind(torch, dtype)
    for i, act in enumerate(ACTS):
        x, gamma, beta, dy = inputs(torch, *size, seed=i)
        x += 3000
        ref.grouped(x, groups)[0, :, ::2] = -700
        ref.grouped(x, groups)[0, :, ::4] = 0.1
        d_x, d_dy = cuda(torch, x).to(T), cuda(torch, dy).to(T)
        x, dy = numbers(d_x), numbers(d_dy)
        norm = B.GroupNorm(channels, groups, cuda(torch, gamma), cuda(torch, beta), activation=act)
        done = norm.forward(d_x)
        s = numbers(done.statistics)
        about = x - ref.spread(s[..., 0], channels)                           # (exact in 64 bits)
        h = about * ref.spread(s[..., 1], channels)
        p = gamma * h + beta
        y = ref.act(p, act)
        # x - mean, gamma / deviation and the sum are rounded; the sigmoid as norm_reference.py has it
        tol = ref.U * (3 * np.abs(gamma * h) + np.abs(p) + np.abs(beta))
        if act == "silu":
            tol = 1.2 * tol + (8 * ref.U if dtype == "fp32" else 2.0**-19) * np.abs(y)
        check(numbers(done.y), y, tol, T, torch)
        same = np.broadcast_to(ref.spread(np.ptp(ref.grouped(x, groups), axis=(1, 3)) == 0, channels), x.shape)
        assert same.any()
        if act == "none" and dtype == "fp32":
            assert np.array_equal(numbers(done.y)[same], np.broadcast_to(beta, x.shape)[same])
        got = norm.backward(d_dy, d_x, done.statistics)
        want = ref.backward(dy, about, 0 * s[..., 0], s[..., 1], groups, gamma.astype(np.float64), beta.astype(np.float64), act, dtype == "fp32")
        check(numbers(got[0]), want[0], want[3], T, torch)
        check(numbers(got[1]), want[1], want[4], torch.float32, torch)
        check(numbers(got[2]), want[2], want[5], torch.float32, torch)
