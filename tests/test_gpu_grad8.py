"""Weight gradients from 8-bit activations on the GPU against the same in 64 bits: x as its 8-bit form holds it, then a plain product.

Tolerances.  A product of dY (8 bits of significand) and a code times a power of two (4) is exact in fp32.  The tensor cores add chains of at most 512 of them; each addition may
lose a unit of the last place of the larger operand, 2^-23 of a partial sum that is at most S = sum |dY||x| of the chain: independent errors, sqrt(512) 2^-23 S.  The chains' sums are
added rounding to nearest, 2^-24 S each.  The tests allow (4 sqrt(min(tokens, 512)) + chains + 4) 2^-23 S for every element; bf16 results half a step more, 2^-8 of the value, added ones
that of the sum."""
import numpy as np
import pytest

import block8_reference as held
from helpers import bf16_dev, to_dev
from paper_2311_14272_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def bits_of(x):
    return wl.f32_to_bf16_bits(np.asarray(x, np.float32))


def values_of(bits):
    return wl.bf16_bits_to_f32(bits).astype(np.float64)


def numbers(t):
    return t.detach().double().cpu().numpy()


def inputs(rng, tokens, rows, k):
    x = np.maximum(rng.standard_normal((tokens, k)) + 0.3, 0) * np.exp(rng.standard_normal((tokens, 1))) * np.where(rng.random((1, k)) < 0.02, 20, 1)
    dy = rng.standard_normal((tokens, rows)) * np.exp(rng.standard_normal((tokens, 1)))
    return bits_of(x), bits_of(dy)


def padded(torch, bits, pitch, odd, dtype=None):
    """A matrix with `pitch` more elements a row (7s), `odd` elements from an aligned address."""
    n, m = bits.shape
    whole = torch.full((n * (m + pitch) + odd,), 7.0, dtype=dtype or torch.bfloat16, device="cuda")
    t = whole[odd:].view(n, m + pitch)[:, :m]
    t.copy_(bf16_dev(np.ascontiguousarray(bits), torch))
    return t, whole


def layer(B, torch, rows, k, n=4, m=4, block=128, keep=1.0, seed=0, mask=True):
    L = B.HybridLayer(rows, k, n, m, block, block, keep)
    if not mask:
        return L, np.ones((rows, k), bool)
    L.build_mask(to_dev(np.random.default_rng(seed).random((rows, k)).astype(np.float32), torch))
    return L, np.unpackbits(L.export_mask()[1].view(np.uint8), axis=1, bitorder="little")[:rows, :k].astype(bool)


def check(got, want, size, tokens, f32, old=None):
    chains = -(-tokens // 512)
    tol = (4 * np.sqrt(min(tokens, 512)) + chains + 4) * 2.0**-23 * size
    if old is not None:
        want = want + old
        tol = tol + 2.0**-24 * np.abs(want)
    tol = tol + (0 if f32 else 2.0**-8 * np.abs(want)) + 1e-37
    off = np.abs(got - want)
    assert np.all(off <= tol), (float((off / tol).max()), np.unravel_index(np.argmax(off / tol), off.shape))


SIZES = [(1, 1, 1), (8, 16, 3), (128, 128, 64), (160, 960, 49), (130, 200, 65), (64, 64, 1000), (300, 1000, 777), (512, 2304, 600), (129, 257, 3000), (1000, 77, 130), (31, 4100, 520),
         (256, 512, 5000)]


@pytest.mark.parametrize("rows,k,tokens", SIZES)
@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("f32", [0, 1])
def test_products(rows, k, tokens, by_token, f32):
    import torch
    from paper_2311_14272_b200 import binding as B
    xb, dyb = inputs(np.random.default_rng(rows + k + tokens), tokens, rows, k)
    x, dy = held.activations(values_of(xb).T).T, values_of(dyb)
    act = B.quantize8(bf16_dev(xb, torch), tokens=True)
    want, size = dy.T @ x, np.abs(dy).T @ np.abs(x)
    L, _ = layer(B, torch, rows, k, mask=False)
    for pitch, odd in ((0, 0), (8, 0), (3, 1)):
        d_dy, _ = padded(torch, dyb if by_token else dyb.T, pitch, odd)
        dw, whole = padded(torch, np.zeros((rows, k), np.uint16), pitch, odd, torch.float32 if f32 else torch.bfloat16)
        got = L.weight_gradient8(d_dy, act, dw=dw, dw_dtype=f32, tokens=by_token)
        assert got is dw
        check(numbers(dw), want, size, tokens, f32)
        assert bool((whole[odd:].view(rows, k + pitch)[:, k:] == 7.0).all() and (whole[:odd] == 7.0).all())
        again = L.weight_gradient8(d_dy, act, dw_dtype=f32, tokens=by_token)
        assert torch.equal(again, dw)
        old = numbers(dw)
        L.weight_gradient8(d_dy, act, dw=dw, dw_dtype=f32, tokens=by_token, accumulate=True)
        check(numbers(dw), want, size, tokens, f32, old)
    assert L.gradient_status() == 0


@pytest.mark.parametrize("rows,k,n,m,block,keep", [(128, 128, 4, 4, 128, 1.0), (256, 512, 2, 4, 128, 0.5), (300, 1000, 4, 8, 128, 0.3), (512, 640, 4, 4, 128, 0.6), (130, 200, 1, 4, 128, 0.0),
                                                    (200, 300, 2, 4, 64, 0.5), (96, 97, 2, 8, 32, 0.4), (1000, 2050, 4, 4, 128, 0.25), (64, 576, 2, 4, 96, 0.5)])
@pytest.mark.parametrize("f32", [0, 1])
def test_under_a_mask(rows, k, n, m, block, keep, f32):
    import torch
    from paper_2311_14272_b200 import binding as B
    if block == 96:
        L = B.HybridLayer(rows, k, n, m, 64, 96, keep)
        L.build_mask(to_dev(np.random.default_rng(1).random((rows, k)).astype(np.float32), torch))
        mask = np.unpackbits(L.export_mask()[1].view(np.uint8), axis=1, bitorder="little")[:rows, :k].astype(bool)
    else:
        L, mask = layer(B, torch, rows, k, n, m, block, keep, 1)
    for tokens in (40, 700):
        xb, dyb = inputs(np.random.default_rng(tokens), tokens, rows, k)
        x, dy = held.activations(values_of(xb).T).T, values_of(dyb)
        act = B.quantize8(bf16_dev(xb, torch), tokens=True)
        want, size = np.where(mask, dy.T @ x, 0.0), np.abs(dy).T @ np.abs(x) * mask
        for pitch, odd in ((0, 0), (3, 1)):
            dw, whole = padded(torch, np.full((rows, k), 0x4040, np.uint16), pitch, odd, torch.float32 if f32 else torch.bfloat16)
            L.weight_gradient8(bf16_dev(dyb, torch), act, dw=dw, dw_dtype=f32, tokens=True, masked=True)
            check(numbers(dw), want, size, tokens, f32)                       # (what is outside the mask: 0 exactly)
            assert bool((whole[odd:].view(rows, k + pitch)[:, k:] == 7.0).all() and (whole[:odd] == 7.0).all())
            dw.fill_(3.0)
            L.weight_gradient8(bf16_dev(dyb, torch), act, dw=dw, dw_dtype=f32, tokens=True, masked=True, accumulate=True)
            check(numbers(dw), want, size, tokens, f32, np.full((rows, k), 3.0))
            assert np.all(numbers(dw)[~mask] == 3.0)
    assert L.gradient_status() == 0


CONVS = [(1, 3, 3, 8, 16, 3, 3, 1), (2, 7, 7, 64, 64, 3, 3, 1), (3, 14, 10, 128, 130, 3, 3, 1), (1, 5, 9, 20, 7, 5, 3, 2), (4, 28, 28, 64, 32, 1, 1, 0), (2, 9, 8, 96, 64, 3, 3, 0),
         (33, 4, 4, 130, 40, 2, 2, 1), (1, 1, 1, 8, 8, 3, 3, 1), (2, 56, 56, 24, 40, 3, 3, 1)]


def lowered(x, kh, kw, pad):
    """[batch, height, width, channels] -> [batch * ho * wo, kh * kw * channels]"""
    x = np.pad(x, ((0, 0), (pad, pad), (pad, pad), (0, 0)))
    ho, wo = x.shape[1] - kh + 1, x.shape[2] - kw + 1
    return np.concatenate([x[:, i:i + ho, j:j + wo] for i in range(kh) for j in range(kw)], 3).reshape(x.shape[0] * ho * wo, -1), ho, wo


@pytest.mark.parametrize("batch,height,width,channels,rows,kh,kw,pad", CONVS)
@pytest.mark.parametrize("f32", [0, 1])
def test_convolutions(batch, height, width, channels, rows, kh, kw, pad, f32):
    import torch
    from paper_2311_14272_b200 import binding as B
    rng = np.random.default_rng(height)
    pixels = batch * height * width
    xb, _ = inputs(rng, pixels, 1, channels)
    x = held.activations(values_of(xb).T).T.reshape(batch, height, width, channels)
    low, ho, wo = lowered(x, kh, kw, pad)
    _, dyb = inputs(rng, batch * ho * wo, rows, 1)
    dy = values_of(dyb)
    act = B.quantize8(bf16_dev(xb, torch), tokens=True)
    want, size = dy.T @ low, np.abs(dy).T @ np.abs(low)
    for block, n, keep, masked in ((128, 4, 1.0, False), (128, 2, 0.5, True), (64, 4, 0.4, True)):
        L, mask = layer(B, torch, rows, kh * kw * channels, n, 4, block, keep, 2)
        mask = mask if masked else np.ones_like(mask)
        for pitch, odd in ((0, 0), (3, 1)):
            d_dy, _ = padded(torch, dyb, pitch, odd)
            d_dy = d_dy.unflatten(0, (batch, ho, wo))
            dw = L.weight_gradient8_conv(d_dy, act, kh, kw, pad, dw_dtype=f32, masked=masked)
            check(numbers(dw), np.where(mask, want, 0.0), size * mask, batch * ho * wo, f32)
        # Y [rows, pixels], too
        conv = B.ConvDesc(batch, height, width, channels, kh, kw, pad, 0)
        d_dy, out = bf16_dev(np.ascontiguousarray(dyb.T), torch), torch.empty_like(dw)
        g = B.WeightGrad8(rows, kh * kw * channels, batch * ho * wo, B.C.pointer(conv), d_dy.data_ptr(), batch * ho * wo, 0, f32, act.buffer.data_ptr(),
                          L.mask if masked else None, out.data_ptr(), kh * kw * channels, 0, 0, None, 0)
        B.crisp_weight_grad8(g, torch.empty(B.crisp_weight_grad8_sizes(g), dtype=torch.uint8, device="cuda"))
        check(numbers(out), np.where(mask, want, 0.0), size * mask, batch * ho * wo, f32)
        assert L.gradient_status() == 0


@pytest.mark.parametrize("rows,k,tokens", [(2650, 2000, 200), (2560, 2048, 1100), (300, 9500, 70), (2433, 2113, 64)])
@pytest.mark.parametrize("by_token", [False, True])
def test_tiles_for_every_sm(rows, k, tokens, by_token):
    """So many tiles that two SMs share one: odd numbers of row tiles and of boxes, rows and columns that end within one."""
    import torch
    from paper_2311_14272_b200 import binding as B
    xb, dyb = inputs(np.random.default_rng(rows), tokens, rows, k)
    x, dy = held.activations(values_of(xb).T).T, values_of(dyb)
    act = B.quantize8(bf16_dev(xb, torch), tokens=True)
    want, size = dy.T @ x, np.abs(dy).T @ np.abs(x)
    for block, n, keep, masked in ((128, 4, 1.0, False), (64, 2, 0.5, True), (128, 2, 1.0, True)):
        L, mask = layer(B, torch, rows, k, n, 4, block, keep, 3, mask=masked)
        for pitch, odd, f32 in ((0, 0, 1), (3, 1, 0)):
            d_dy, _ = padded(torch, dyb if by_token else np.ascontiguousarray(dyb.T), pitch, odd)
            dw, whole = padded(torch, np.zeros((rows, k), np.uint16), pitch, odd, torch.float32 if f32 else torch.bfloat16)
            L.weight_gradient8(d_dy, act, dw=dw, dw_dtype=f32, tokens=by_token, masked=masked)
            check(numbers(dw), want * mask, size * mask, tokens, f32)
            assert bool((whole[odd:].view(rows, k + pitch)[:, k:] == 7.0).all() and (whole[:odd] == 7.0).all())
            old = numbers(dw)
            L.weight_gradient8(d_dy, act, dw=dw, dw_dtype=f32, tokens=by_token, masked=masked, accumulate=True)
            check(numbers(dw), want * mask, size * mask, tokens, f32, old)
    assert L.gradient_status() == 0


@pytest.mark.parametrize("rows,k,tokens,keep", [(2600, 2048, 1100, 0.5), (2600, 2049, 1100, 0.5), (739, 1739, 2, 0.17)])
@pytest.mark.parametrize("f32", [0, 1])
def test_zeros_of_many_blocks(rows, k, tokens, keep, f32):
    """Blocks that are not kept, beside long products and short ones, in rows that begin anywhere."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, mask = layer(B, torch, rows, k, 4, 4, 128, keep, 2)
    xb, dyb = inputs(np.random.default_rng(rows + k), tokens, rows, k)
    x, dy = held.activations(values_of(xb).T).T, values_of(dyb)
    act = B.quantize8(bf16_dev(xb, torch), tokens=True)
    want, size = np.where(mask, dy.T @ x, 0.0), np.abs(dy).T @ np.abs(x) * mask
    for pitch, odd in ((0, 0), (5, 3)):
        dw, whole = padded(torch, np.full((rows, k), 0x4040, np.uint16), pitch, odd, torch.float32 if f32 else torch.bfloat16)
        L.weight_gradient8(bf16_dev(dyb, torch), act, dw=dw, dw_dtype=f32, tokens=True, masked=True)
        check(numbers(dw), want, size, tokens, f32)
        assert np.all(numbers(dw)[~mask] == 0.0)
        assert bool((whole[odd:].view(rows, k + pitch)[:, k:] == 7.0).all() and (whole[:odd] == 7.0).all())
    assert L.gradient_status() == 0


def test_convolution_tiles_for_every_sm():
    import torch
    from paper_2311_14272_b200 import binding as B
    batch, height, width, channels, rows = 2, 9, 7, 200, 2400
    rng = np.random.default_rng(0)
    xb, _ = inputs(rng, batch * height * width, 1, channels)
    x = held.activations(values_of(xb).T).T.reshape(batch, height, width, channels)
    low, ho, wo = lowered(x, 3, 3, 1)
    _, dyb = inputs(rng, batch * ho * wo, rows, 1)
    dy = values_of(dyb)
    L, _ = layer(B, torch, rows, 9 * channels, mask=False)
    dw = L.weight_gradient8_conv(bf16_dev(dyb, torch).view(batch, ho, wo, rows), B.quantize8(bf16_dev(xb, torch), tokens=True), 3, 3, 1)
    check(numbers(dw), dy.T @ low, np.abs(dy).T @ np.abs(low), batch * ho * wo, 1)


def test_what_is_not_finite():
    import torch
    from paper_2311_14272_b200 import binding as B
    x, dy = torch.ones(100, 256, device="cuda").bfloat16(), torch.ones(100, 256, device="cuda").bfloat16()
    x[5, 9], dy[7, 130] = float("nan"), float("inf")
    L, mask = layer(B, torch, 256, 256, 2, 4, 128, 0.5)
    act = B.quantize8(x, tokens=True)
    dw = L.weight_gradient8(dy, act, tokens=True)
    bad = torch.zeros(256, 256, dtype=torch.bool, device="cuda")
    bad[:, 9] = bad[130] = True
    assert torch.equal(~dw.isfinite(), bad) and torch.all(dw[~bad] == 100)
    dw = L.weight_gradient8(dy, act, tokens=True, masked=True)
    inside = torch.from_numpy(mask).cuda()
    assert torch.equal(~dw.isfinite(), bad & inside) and torch.all(dw[~inside] == 0)


def test_a_gradient_against_differences():
    """The loss sum(G * (W x~)) along a direction of W, by differences (it is linear in W: any step)."""
    import torch
    from paper_2311_14272_b200 import binding as B
    torch.manual_seed(0)
    x, g, w, way = (torch.randn(s, device="cuda").bfloat16() for s in ((200, 300), (200, 130), (130, 300), (130, 300)))
    act = B.quantize8(x, tokens=True)
    held_x = act.dequantize(tokens=True).double()
    value = lambda t: (g.double() * (held_x @ t.double().t())).sum().item()  # noqa: E731
    dw = layer(B, torch, 130, 300, mask=False)[0].weight_gradient8(g, act, tokens=True)
    slope = (value(w.double() + way.double()) - value(w.double() - way.double())) / 2
    # 39000 products of sums over 200 tokens, each off by 60 2^-23 of sum |g||x| ~ 130: independent, sqrt(39000) * 60 * 1.2e-7 * 130
    assert abs(slope - (dw.double() * way.double()).sum().item()) < 0.2


@pytest.mark.parametrize("rows,k,tokens", [(256, 512, 600), (2560, 2048, 600)])
def test_a_wait_that_runs_out(rows, k, tokens):
    """Copies that never come: the kernel gives up after the limit, says so and returns; the next call is as ever.  One SM a tile, and pairs."""
    import torch
    from paper_2311_14272_b200 import binding as B
    x, dy = torch.randn(tokens, k, device="cuda").bfloat16(), torch.randn(tokens, rows, device="cuda").bfloat16()
    act, dw, status = B.quantize8(x, tokens=True), torch.empty(rows, k, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    g = B.WeightGrad8(rows, k, tokens, None, dy.data_ptr(), rows, 1, 1, act.buffer.data_ptr(), None, dw.data_ptr(), k, 0, 2, status.data_ptr(), 2000000)
    workspace = torch.empty(B.crisp_weight_grad8_sizes(g), dtype=torch.uint8, device="cuda")
    B.crisp_weight_grad8(g, workspace)
    assert status.item() == B.TIMEOUT
    status.zero_()
    g.skip_fill, g.wait_limit_cycles = 0, 0
    B.crisp_weight_grad8(g, workspace)
    want = dy.double().t() @ act.dequantize(tokens=True).double()
    assert status.item() == 0 and (dw - want).abs().max().item() <= 1e-4 * want.abs().max().item()


def test_streams_and_graphs():
    import torch
    from paper_2311_14272_b200 import binding as B
    x, dy = torch.randn(3000, 512, device="cuda").bfloat16(), torch.randn(3000, 256, device="cuda").bfloat16()
    L, _ = layer(B, torch, 256, 512, 2, 4, 128, 0.5)
    act = B.quantize8(x, tokens=True)
    want = [L.weight_gradient8(dy, act, tokens=True, masked=m) for m in (False, True)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, side.cuda_stream):
        got = [L.weight_gradient8(dy, act, tokens=True, masked=m, stream=s) for m in (False, True)]
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = [L.weight_gradient8(dy, B.quantize8(x, tokens=True), tokens=True, masked=m) for m in (False, True)]
        graphs.append((g, got))
    x.copy_(torch.randn_like(x))
    want = [L.weight_gradient8(dy, B.quantize8(x, tokens=True), tokens=True, masked=m) for m in (False, True)]
    torch.cuda.synchronize()
    for (g, _), s in zip(graphs, (torch.cuda.Stream(), torch.cuda.Stream())):
        with torch.cuda.stream(s):
            for _ in range(3):
                g.replay()
    torch.cuda.synchronize()
    for _, got in graphs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_step_of_fine_tuning():
    """The run of them together, as a network's step has it: convolution, norm (its input and output kept in 8 bits), an 8-bit product of what was kept; backward through all of it and
    an AdamW step under the masks.  Every gradient against the formula's in 64 bits."""
    import torch
    from paper_2311_14272_b200 import binding as B
    import norm_reference as ref
    torch.manual_seed(1)
    batch, height, width, channels, mid, rows = 2, 12, 10, 64, 128, 256
    image = torch.randn(batch, height, width, channels, device="cuda").bfloat16()
    conv, head = B.HybridLayer(mid, 9 * channels, 4, 4, 64, 64, 0.5), B.HybridLayer(rows, mid, 2, 4, 128, 128, 1.0)
    weights = [torch.randn(mid, 9 * channels, device="cuda") * 0.05, torch.randn(rows, mid, device="cuda") * 0.1]
    copies = [w.bfloat16() for w in weights]
    for L, w in zip((conv, head), weights):
        L.build_mask(w.abs())
    conv.encode(copies[0])
    head.encode8(copies[1])
    gamma, beta = 1 + 0.1 * torch.randn(mid, device="cuda"), 0.1 * torch.randn(mid, device="cuda")
    norm = B.GroupNorm(mid, 8, gamma, beta, activation="relu")
    image8 = B.quantize8(image.view(-1, channels), tokens=True)
    y = conv.spmm_conv(image, 3, 3, 1, nhwc_out=True)
    done = norm.forward(y, keep_x=True, keep_y=True, plain_y=False)
    out = head.spmm8(done.y8, tokens=True)
    d_out = torch.randn_like(out)
    dw_head = head.weight_gradient8(d_out, done.y8, tokens=True, masked=True)
    dz = (d_out @ head.decode8()).view(batch, height, width, mid)
    dy, dgamma, dbeta = norm.backward(dz, done.x8, done.statistics)
    dw_conv = conv.weight_gradient8_conv(dy, image8, 3, 3, 1, masked=True)
    mask = [torch.from_numpy(np.unpackbits(L.export_mask()[1].view(np.uint8), axis=1, bitorder="little")[:w.shape[0], :w.shape[1]].astype(bool)) for L, w in zip((conv, head), weights)]
    tokens = batch * height * width
    x = numbers(done.y8.dequantize(tokens=True))
    g = numbers(d_out)
    check(numbers(dw_head), np.where(mask[1], g.T @ x, 0), np.abs(g).T @ np.abs(x), tokens, 1)
    s = numbers(done.statistics)
    want = ref.backward(numbers(dz).reshape(batch, -1, mid), numbers(done.x8.dequantize(tokens=True)).reshape(batch, -1, mid), s[..., 0], s[..., 1], 8, numbers(gamma), numbers(beta),
                        "relu", False)
    assert np.all(np.abs(numbers(dy).reshape(batch, -1, mid) - want[0]) <= want[3] + 2.0**-8 * np.abs(want[0]) + 1e-37)
    assert np.all(np.abs(numbers(dgamma) - want[1]) <= want[4]) and np.all(np.abs(numbers(dbeta) - want[2]) <= want[5])
    low, _, _ = lowered(numbers(image8.dequantize(tokens=True)).reshape(batch, height, width, channels), 3, 3, 1)
    g = numbers(dy).reshape(-1, mid)
    check(numbers(dw_conv), np.where(mask[0], g.T @ low, 0), np.abs(g).T @ np.abs(low), tokens, 1)
    before = [w.clone() for w in weights]
    opt = B.AdamW(weights + [gamma, beta], copies=copies + [None, None], masks=[conv, head, None, None], lr=1e-2)
    opt.step([dw_conv, dw_head, dgamma, dbeta])
    for w, old, m, d in zip(weights, before, mask, (dw_conv, dw_head)):
        m = m.cuda()
        assert torch.all(w[~m] == 0) and torch.all((w != old)[m & (d != 0)])


@pytest.mark.parametrize("channels", [160, 192, 320, 448, 960])
@pytest.mark.parametrize("batch,height,width,rows,pad", [(1, 7, 7, 130, 0), (2, 5, 6, 64, 1), (8, 28, 28, 128, 0), (1, 4, 5, 9700, 0)])
@pytest.mark.parametrize("f32", [0, 1])
def test_one_tap_whose_last_block_is_not_whole(channels, batch, height, width, rows, pad, f32):
    """1 x 1 convolutions under a list of blocks, the last of which ends within its first or second 64 columns: nothing behind the last column, of parts of the pixels and of all at once."""
    import torch
    from paper_2311_14272_b200 import binding as B
    rng = np.random.default_rng(channels)
    L = B.HybridLayer(rows, channels, 2, 4, 128, 128, 0.5)
    assert L.kkeep < L.nblk
    liking = rng.random((rows, channels)).astype(np.float32)
    liking[:, channels // 128 * 128:] *= 100                                  # (the last block is kept by every row tile)
    L.build_mask(to_dev(liking, torch))
    mask = np.unpackbits(L.export_mask()[1].view(np.uint8), axis=1, bitorder="little")[:rows, :channels].astype(bool)
    assert mask[:, channels // 128 * 128:].any(1).all()
    xb, _ = inputs(rng, batch * height * width, 1, channels)
    x = held.activations(values_of(xb).T).T.reshape(batch, height, width, channels)
    low, ho, wo = lowered(x, 1, 1, pad)
    tokens = batch * ho * wo
    _, dyb = inputs(rng, tokens, rows, 1)
    dy = values_of(dyb)
    act, d_dy = B.quantize8(bf16_dev(xb, torch), tokens=True), bf16_dev(dyb, torch).view(batch, ho, wo, rows)
    want, size = np.where(mask, dy.T @ low, 0.0), np.abs(dy).T @ np.abs(low) * mask
    for pitch, odd in ((0, 0), (8, 0), (3, 1)):
        whole = torch.full((odd + (rows + 64) * (channels + pitch),), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        dw, behind = whole[odd:].view(rows + 64, channels + pitch)[:rows, :channels], whole[odd:].view(rows + 64, channels + pitch)
        L.weight_gradient8_conv(d_dy, act, 1, 1, pad, dw=dw, dw_dtype=f32, masked=True)
        check(numbers(dw), want, size, tokens, f32)
        assert bool((behind[rows:] == 7.0).all() and (behind[:, channels:] == 7.0).all() and (whole[:odd] == 7.0).all())
        dw.fill_(3.0)
        L.weight_gradient8_conv(d_dy, act, 1, 1, pad, dw=dw, dw_dtype=f32, masked=True, accumulate=True)
        check(numbers(dw), want, size, tokens, f32, np.full(dw.shape, 3.0))
        assert np.all(numbers(dw)[~mask] == 3.0)
        assert bool((behind[rows:] == 7.0).all() and (behind[:, channels:] == 7.0).all() and (whole[:odd] == 7.0).all())
    assert L.gradient_status() == 0


def test_the_layers_status_is_reset():
    """A wait that ran out, written to the layer's own word: said until it is reset, and not of the gradients after that."""
    import torch
    from paper_2311_14272_b200 import binding as B
    x, dy = torch.randn(300, 256, device="cuda").bfloat16(), torch.randn(300, 128, device="cuda").bfloat16()
    L, _ = layer(B, torch, 128, 256, mask=False)
    act, dw = B.quantize8(x, tokens=True), torch.empty(128, 256, device="cuda")
    g = B.WeightGrad8(128, 256, 300, None, dy.data_ptr(), 128, 1, 1, act.buffer.data_ptr(), None, dw.data_ptr(), 256, 0, 1, L._grad_status.data_ptr(), 2000000)
    workspace = torch.empty(B.crisp_weight_grad8_sizes(g), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream, 0):
        B.crisp_weight_grad8(g, workspace)
        assert L.gradient_status() == B.TIMEOUT
        L.weight_gradient8(dy, act, tokens=True)
        assert L.gradient_status() == B.TIMEOUT                              # (of the one before; whoever resets it knows of which)
        L.reset_gradient_status(stream)
        assert L.gradient_status() == 0
        got = L.weight_gradient8(dy, act, tokens=True)
        want = dy.double().t() @ act.dequantize(tokens=True).double()
        assert L.gradient_status() == 0 and (got - want).abs().max().item() <= 1e-4 * want.abs().max().item()


@pytest.mark.parametrize("batch,height,width,channels,rows,kh,kw,pad", [(1, 9, 11, 64, 64, 3, 3, 0), (2, 9, 11, 40, 130, 3, 3, 1), (3, 27, 31, 24, 40, 5, 5, 0), (1, 7, 5, 130, 2500, 3, 2, 1),
                                                                        (1, 13, 13, 16, 32, 7, 7, 3), (2, 11, 9, 8, 16, 7, 7, 0), (1, 1, 2, 64, 64, 5, 5, 2), (1, 3, 70, 72, 9700, 1, 3, 0),
                                                                        (1, 30, 1, 64, 64, 3, 1, 0), (4, 28, 28, 64, 64, 3, 3, 1), (2, 9, 11, 64, 64, 1, 1, 2),
                                                                                                                                                                (2, 9, 11, 128, 256, 3, 3, 1), (1, 10, 10, 64, 1300, 7, 7, 3)])
def test_what_is_not_finite_at_pixels_that_a_tap_does_not_cover(batch, height, width, channels, rows, kh, kw, pad):
    """NaN at the last column, the last line and the corners of the images: in the weights of the taps that come by there, and in no other, as the sum over output pixels has it."""
    import torch
    from paper_2311_14272_b200 import binding as B
    rng = np.random.default_rng(width)
    xb, _ = inputs(rng, batch * height * width, 1, channels)
    x = torch.from_numpy(values_of(xb)).view(batch, height, width, channels)
    places = [(batch - 1, height - 1, width - 1, 0), (0, 0, width - 1, 1), (0, height - 1, 0, 2), (0, 0, 0, 3), (0, height // 2, max(width - 2, 0), 4), (batch - 1, max(height - 2, 0), width // 2, 5),
              (0, height // 2, width // 2, 6)]
    for p in places:
        x[p] = float("nan")
    act = B.quantize8(x.to("cuda", torch.bfloat16).view(-1, channels), tokens=True)
    low, ho, wo = lowered(numbers(act.dequantize(tokens=True)).reshape(batch, height, width, channels), kh, kw, pad)
    _, dyb = inputs(rng, batch * ho * wo, rows, 1)
    dy = values_of(dyb)
    bad = np.isnan(low).any(0)
    low = np.where(bad, 0, low)
    want, size = dy.T @ low, np.abs(dy).T @ np.abs(low)
    L, mask = layer(B, torch, rows, kh * kw * channels, 2, 4, 128, 0.6, 2)
    for masked in (False, True):
        inside = mask if masked else np.ones_like(mask)
        for f32 in (0, 1):
            dw = numbers(L.weight_gradient8_conv(bf16_dev(dyb, torch).view(batch, ho, wo, rows), act, kh, kw, pad, dw_dtype=f32, masked=masked))
            assert np.array_equal(np.isnan(dw), bad & inside)
            check(np.where(bad, 0, dw), np.where(inside, want, 0), size * inside, batch * ho * wo, f32)
    assert L.gradient_status() == 0


def test_a_layers_status_word_is_its_own():
    """Layers are made without a launch each (their words come out of blocks), and a wait that ran out in one is not said of another."""
    import torch
    from paper_2311_14272_b200 import binding as B
    layers = [B.HybridLayer(128, 256, 4, 4, 128, 128, 1.0) for _ in range(200)]
    assert len({L._grad_status.data_ptr() for L in layers}) == 200 and all(L.gradient_status() == 0 for L in layers)
    x, dy = torch.randn(300, 256, device="cuda").bfloat16(), torch.randn(300, 128, device="cuda").bfloat16()
    act, dw = B.quantize8(x, tokens=True), torch.empty(128, 256, device="cuda")
    g = B.WeightGrad8(128, 256, 300, None, dy.data_ptr(), 128, 1, 1, act.buffer.data_ptr(), None, dw.data_ptr(), 256, 0, 1, layers[77]._grad_status.data_ptr(), 2000000)
    B.crisp_weight_grad8(g, torch.empty(B.crisp_weight_grad8_sizes(g), dtype=torch.uint8, device="cuda"))
    assert [i for i, L in enumerate(layers) if L.gradient_status()] == [77]
    graph = torch.cuda.CUDAGraph()
    B._status_words.clear()
    with torch.cuda.graph(graph):                                            # (one that is made in a capture)
        L = B.HybridLayer(128, 256, 4, 4, 128, 128, 1.0)
        got = L.weight_gradient8(dy, act, tokens=True)
    assert not B._status_words
    other = B.HybridLayer(128, 256, 4, 4, 128, 128, 1.0)
    graph.replay()
    assert torch.equal(got, other.weight_gradient8(dy, act, tokens=True)) and L.gradient_status() == other.gradient_status() == 0
