"""Products in 8 bits on the GPU against the same in 64 bits: weights and activations as their 8-bit forms hold them (to the bit), then a plain product.

Tolerances of the product.  A product of two codes has 8 bits and is exact in fp32, as is its scaling by a power of two.  The tensor cores add K of them into an fp32
accumulator; each addition may lose a unit of the last place of the larger operand (they need not round to nearest), 2^-23 of a partial sum that is at most
S = sum |w||x|: K 2^-23 S in the worst case, of which the first runs say how much is there; the tests allow sqrt(K) * 4 * 2^-23 S + K-independent 2^-22 S, the size of
independent errors, for every element.  bf16 results add half a step, 2^-8... of the value: 2^-9 |y| relative to round to nearest (8 bits of significand: half a step is 2^-9
of the power of two above, at most 2^-8 of the value)."""
import numpy as np
import pytest

import block8_reference as ref
from helpers import bf16_dev, to_dev
from paper_2311_14272_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def bits_of(x):
    return wl.f32_to_bf16_bits(np.asarray(x, np.float32))


def numbers(t):
    return t.detach().double().cpu().numpy()


def layer(B, torch, rows, k, n, m, keep, seed, w=None, pitch=0, odd=0):
    rng = np.random.default_rng(seed)
    if w is None:
        w = rng.standard_normal((rows, k)) * np.exp(rng.standard_normal((rows, 1))) * 0.05
    bits = bits_of(w)
    L = B.HybridLayer(rows, k, n, m, 128, 128, keep)
    L.build_mask(to_dev(rng.random((rows, k)).astype(np.float32), torch))
    words = L.export_mask()[1]
    mask = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:rows, :k].astype(bool)
    whole = torch.full((rows * (k + pitch) + odd,), 9.0, dtype=torch.bfloat16, device="cuda")
    d_w = whole[odd:].view(rows, k + pitch)[:, :k]
    d_w.copy_(bf16_dev(bits, torch))
    L.encode8(d_w)
    return L, ref.weights(wl.bf16_bits_to_f32(bits).astype(np.float64), mask), mask


def activations(rng, k, ncols):
    x = rng.standard_normal((k, ncols)) * np.exp(rng.standard_normal((1, ncols))) * np.where(rng.random((k, 1)) < 0.02, 20, 1)
    return bits_of(x)


def check(y, w, x, k, f32, bias=None, relu=False):
    want, size = w @ x, np.abs(w) @ np.abs(x)
    if bias is not None:
        want, size = want + bias[:, None], size + np.abs(bias)[:, None]
    if relu:
        want = np.maximum(want, 0.0)
    tol = (4 * np.sqrt(k) + 2) * 2.0**-23 * size + (0 if f32 else 2.0**-8 * np.abs(want))
    off = np.abs(y - want)
    assert np.all(off <= tol + 1e-37), float((off / (tol + 1e-37)).max())


@pytest.mark.parametrize("rows,k,n,m,keep", [(128, 128, 4, 4, 1.0), (256, 512, 2, 4, 0.5), (130, 200, 1, 4, 0.5), (1, 1, 4, 4, 1.0), (300, 1000, 4, 8, 0.3),
                                              (64, 27, 2, 4, 1.0), (129, 4100, 2, 8, 0.25), (256, 384, 4, 4, 0.0)])
@pytest.mark.parametrize("pitch,odd", [(0, 0), (8, 0), (3, 1)])
def test_weights_are_held_to_the_bit(rows, k, n, m, keep, pitch, odd):
    import torch
    from paper_2311_14272_b200 import binding as B
    L, want, _ = layer(B, torch, rows, k, n, m, keep, 1, pitch=pitch, odd=odd)
    assert np.array_equal(numbers(L.decode8()), want)
    out = torch.full((rows, k + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    B.crisp_decode8(L.handle8, out, k + 5)
    assert np.array_equal(numbers(out[:, :k]), want) and torch.all(out[:, k:] == 7.0)


@pytest.mark.parametrize("ncols", [1, 7, 16, 17, 33, 64, 100, 224, 257])
@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("f32", [0, 1])
def test_products(ncols, tokens, f32):
    import torch
    from paper_2311_14272_b200 import binding as B
    for rows, k, n, m, keep in ((128, 128, 4, 4, 1.0), (300, 1000, 2, 4, 0.5), (512, 2304, 4, 4, 1.0)):
        L, w, _ = layer(B, torch, rows, k, n, m, keep, 2)
        x = activations(np.random.default_rng(ncols), k, ncols)
        held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
        d_x = bf16_dev(x, torch)
        y = L.spmm8(d_x.t().contiguous() if tokens else d_x, y_dtype=f32, tokens=tokens)
        assert L.device_status8() == 0
        check(numbers(y.t() if tokens else y), w, held, k, f32)


@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("f32", [0, 1])
@pytest.mark.parametrize("pad_x,pad_y,odd", [(1, 1, 1), (3, 5, 0), (8, 8, 0), (0, 2, 1)])
def test_pitches_odd_addresses_and_what_lies_beside(pad_x, pad_y, odd, f32, tokens):
    import torch
    from paper_2311_14272_b200 import binding as B
    rows, k, ncols = 200, 333, 75
    L, w, _ = layer(B, torch, rows, k, 4, 4, 0.7, 3)
    bias = np.random.default_rng(4).standard_normal(rows).astype(np.float32)
    L.set_epilogue8(to_dev(bias, torch), relu=True)
    x = activations(np.random.default_rng(5), k, ncols)
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    a, b = (ncols, k) if tokens else (k, ncols)
    d_x = torch.full((odd + a * (b + pad_x),), float("nan"), dtype=torch.bfloat16, device="cuda")[odd:].view(a, b + pad_x)[:, :b]
    d_x.copy_(bf16_dev(x, torch).t() if tokens else bf16_dev(x, torch))
    a, b = (ncols, rows) if tokens else (rows, ncols)
    whole = torch.full((odd + a * (b + pad_y) + 64,), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    y = whole[odd:odd + a * (b + pad_y)].view(a, b + pad_y)[:, :b]
    L.spmm8(d_x, y, y_dtype=f32, tokens=tokens)
    check(numbers(y.t() if tokens else y), w, held, k, f32, bias.astype(np.float64), True)
    y.fill_(7.0)
    assert torch.all(whole == 7.0)


@pytest.mark.parametrize("rows,k,ncols,keep", [(4096, 4096, 1, 1.0), (1024, 4096, 40, 0.5), (640, 2304, 700, 0.25), (4096, 1024, 2000, 0.5), (128, 8192, 5, 1.0)])
def test_tiles_of_every_width_and_parts(rows, k, ncols, keep):
    """Few columns (a cluster shares a tile's blocks), waves of wide tiles, tiles that begin inside a chunk of 128 scales."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, rows, k, 4, 4, keep, 6)
    x = activations(np.random.default_rng(7), k, ncols)
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    d_x = bf16_dev(x, torch).t().contiguous()
    act = L.quantize8(d_x, tokens=True)
    for f32 in (0, 1):
        y = L.spmm8(d_x, tokens=True, y_dtype=f32)
        check(numbers(y.t()), w, held, k, f32)
        again = L.spmm8(act, tokens=True, y_dtype=f32)
        if ncols > 4:                                        # (fewer columns: another kernel, another order of the sums)
            assert torch.equal(y, again)
        check(numbers(again.t()), w, held, k, f32)
    assert L.device_status8() == 0
    info = L.last_launch8()
    assert info["tile_cols"] <= 16 or ncols > 16
    assert info["ctas"] <= 148 or info["stack"] == 1


@pytest.mark.parametrize("tile", [64, 128, 192, 256])
@pytest.mark.parametrize("split", [1, 2, 3, 8])
def test_the_result_does_not_depend_on_the_tiling(tile, split):
    """Every tile width, alone and with clusters: the sums of the parts differ in their roundings only."""
    import torch
    from paper_2311_14272_b200 import binding as B
    rows, k, ncols = 300, 1500, 333
    L, w, _ = layer(B, torch, rows, k, 4, 4, 0.8, 30)
    x = activations(np.random.default_rng(31), k, ncols)
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    d_x = bf16_dev(x, torch)
    bias = np.random.default_rng(32).standard_normal(rows).astype(np.float32)
    L.set_epilogue8(to_dev(bias, torch), relu=True)
    L.set_tuning8(tile_cols=tile, split=split)
    for tokens in (False, True):
        for f32 in (0, 1):
            y = L.spmm8(d_x.t().contiguous() if tokens else d_x, tokens=tokens, y_dtype=f32)
            info = L.last_launch8()
            assert info["tile_cols"] == tile and info["stack"] == split
            check(numbers(y.t() if tokens else y), w, held, k, f32, bias.astype(np.float64), True)
    with pytest.raises(B.CrispError):
        L.set_tuning8(tile_cols=96)
    with pytest.raises(B.CrispError):
        L.set_tuning8(split=9)


@pytest.mark.parametrize("ncols", [1, 2, 3, 4])
@pytest.mark.parametrize("rows,k,keep", [(1, 1, 1.0), (129, 1000, 1.0), (300, 4500, 0.4), (512, 130, 1.0), (256, 12000, 1.0), (256, 5000, 0.7)])
def test_a_few_columns(rows, k, keep, ncols):
    """One to four columns on the CUDA cores where their codes fit in shared memory, on the tensor cores else and where a tile is asked for."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, rows, k, 4, 4, keep, 40)
    x = activations(np.random.default_rng(41), k, ncols)
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    bias = np.random.default_rng(42).standard_normal(rows).astype(np.float32)
    L.set_epilogue8(to_dev(bias, torch), relu=True)
    d_x = bf16_dev(x, torch)
    odd = torch.full((k * ncols + 1,), 3.0, dtype=torch.bfloat16, device="cuda")[1:].view(ncols, k)
    odd.copy_(d_x.t())
    fits = L.kkeep * ncols * 513 <= 100 * 1024
    for tile in (0, 16):
        L.set_tuning8(tile_cols=tile)
        for f32 in (0, 1):
            for tokens, src in ((False, d_x), (True, d_x.t().contiguous()), (True, odd)):
                y = L.spmm8(src, tokens=tokens, y_dtype=f32)
                assert (L.last_launch8()["path"] == B.PATH_DIRECT) == (fits and not tile) and L.device_status8() == 0
                check(numbers(y.t() if tokens else y), w, held, k, f32, bias.astype(np.float64), True)


@pytest.mark.parametrize("tile", [128, 192, 256])
@pytest.mark.parametrize("rows,k,ncols", [(256, 128, 256), (257, 1000, 333), (640, 2304, 700), (130, 512, 65), (512, 700, 3000)])
def test_pairs_of_sms(rows, k, ncols, tile):
    """Two row tiles (the last of an odd number with itself) multiplied by one instruction; as many tiles as pairs, and more."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, rows, k, 4, 4, 1.0, 35)
    x = activations(np.random.default_rng(36), k, ncols)
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    d_x = bf16_dev(x, torch)
    bias = np.random.default_rng(37).standard_normal(rows).astype(np.float32)
    L.set_epilogue8(to_dev(bias, torch), relu=True)
    L.set_tuning8(tile_cols=tile, split=-1)
    for tokens in (False, True):
        for f32 in (0, 1):
            y = L.spmm8(d_x.t().contiguous() if tokens else d_x, tokens=tokens, y_dtype=f32)
            info = L.last_launch8()
            assert info["tile_cols"] == tile and info["stack"] == -1 and L.device_status8() == 0
            check(numbers(y.t() if tokens else y), w, held, k, f32, bias.astype(np.float64), True)
    L.set_tuning8(tile_cols=tile, split=-1, wait_limit_cycles=2_000_000, skip_fill=0)
    L.spmm8(d_x)
    assert L.device_status8() == B.TIMEOUT
    L.reset_status8()
    L.set_tuning8(tile_cols=tile, split=-1)
    again = L.spmm8(d_x)
    assert L.device_status8() == 0
    check(numbers(again), w, held, k, 0, bias.astype(np.float64), True)


@pytest.mark.parametrize("ncols,tile", [(1, 32), (16, 64), (20, 64), (32, 32)])
def test_narrow_tiles_that_are_not_the_first_choice(ncols, tile):
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, 256, 1024, 4, 4, 1.0, 33)
    x = activations(np.random.default_rng(34), 1024, ncols)
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    for split in (1, 4):
        L.set_tuning8(tile_cols=tile, split=split)
        act = L.quantize8(bf16_dev(x, torch))
        y = L.spmm8(act, y_dtype=1)
        assert L.last_launch8()["tile_cols"] == tile
        check(numbers(y), w, held, 1024, 1)
        check(numbers(L.spmm8(bf16_dev(x, torch), y_dtype=1)), w, held, 1024, 1)


def test_no_kept_block_gives_the_bias():
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, 200, 300, 4, 4, 0.0, 8)
    bias = torch.linspace(-1, 1, 200, device="cuda")
    L.set_epilogue8(bias, relu=True)
    x = torch.full((300, 50), float("nan"), dtype=torch.bfloat16, device="cuda")
    for ncols in (1, 50):
        y = L.spmm8(x[:, :ncols], y_dtype=1)
        assert torch.equal(y, bias.clamp(min=0)[:, None].expand(200, ncols))
    assert not L.decode8().any()


@pytest.mark.parametrize("tokens", [False, True])
def test_what_is_not_finite_stays_in_its_column_and_its_row_tiles(tokens):
    import torch
    from paper_2311_14272_b200 import binding as B
    rows, k, ncols = 256, 512, 40
    rng = np.random.default_rng(9)
    w0 = rng.standard_normal((rows, k))
    w0[5, 130], w0[200, 400] = np.nan, np.inf
    L, w, mask = layer(B, torch, rows, k, 4, 4, 0.5, 9, w=w0)
    xf = wl.bf16_bits_to_f32(activations(rng, k, ncols)).astype(np.float64)
    xf[3, 4], xf[140, 7], xf[300, 9] = np.nan, np.inf, -np.inf
    held = ref.activations(xf)
    assert np.array_equal(numbers(L.decode8()), w, equal_nan=True)
    d_x = bf16_dev(bits_of(xf), torch)
    y = L.spmm8(d_x.t().contiguous() if tokens else d_x, tokens=tokens, y_dtype=1)
    got = numbers(y.t() if tokens else y)
    # NaN where a NaN code meets any code of its block, also a zero one
    bad = np.zeros((rows, ncols), bool)
    kept = np.stack([mask[rt * 128:(rt + 1) * 128].reshape(-1, k // 128, 128).any((0, 2)) for rt in range(2)])
    for row, col in ((3, 4), (140, 7), (300, 9)):
        for rt in range(2):
            if kept[rt, row // 128]:
                bad[rt * 128:(rt + 1) * 128, col] = True
    bad[np.isnan(w).any(1)] = True
    assert np.array_equal(np.isnan(got), bad)
    clean_w, clean_x = np.nan_to_num(w), np.nan_to_num(held)
    want, size = clean_w @ clean_x, np.abs(clean_w) @ np.abs(clean_x)
    tol = (4 * np.sqrt(k) + 2) * 2.0**-23 * size + 1e-37
    assert np.all((np.abs(got - want) <= tol) | bad)


@pytest.mark.parametrize("power_w,power_x", [(0, -100), (-60, -60), (60, 60), (100, 20), (-120, 110)])
def test_values_of_any_size(power_w, power_x):
    import torch
    from paper_2311_14272_b200 import binding as B
    rng = np.random.default_rng(10)
    L, w, _ = layer(B, torch, 128, 256, 4, 4, 1.0, 10, w=rng.standard_normal((128, 256)) * 2.0**power_w)
    x = bits_of(rng.standard_normal((256, 30)) * 2.0**power_x)
    y = numbers(L.spmm8(bf16_dev(x, torch), y_dtype=1))
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    size = np.abs(w) @ np.abs(held)
    assert np.all(np.abs(y - w @ held) <= 66 * 2.0**-23 * size + 2.0**-140)


def test_identity_gives_the_weights():
    """One product a result: every code, scale and place shows."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, 300, 700, 2, 4, 0.6, 11)
    y = numbers(L.spmm8(torch.eye(700, dtype=torch.bfloat16, device="cuda"), y_dtype=1))
    assert np.array_equal(y, w)


def test_a_stage_that_never_fills_ends_with_a_status():
    import torch
    from paper_2311_14272_b200 import binding as B
    for ncols in (3, 600):
        L, w, _ = layer(B, torch, 512, 2048, 4, 4, 1.0, 12)
        x = activations(np.random.default_rng(13), 2048, ncols)
        d_x = bf16_dev(x, torch)
        L.set_tuning8(wait_limit_cycles=2_000_000, skip_fill=1)
        L.spmm8(d_x)
        assert L.device_status8() == B.TIMEOUT
        L.set_tuning8()
        L.reset_status8()
        y = L.spmm8(d_x)
        assert L.device_status8() == 0
        check(numbers(y), w, ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64)), 2048, 0)


def test_captured_products_and_a_layer_encoded_anew_in_between():
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, 384, 1024, 4, 4, 1.0, 14)
    x = torch.zeros(1024, 24, dtype=torch.bfloat16, device="cuda")
    d_w = torch.zeros(384, 1024, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(384, 24, dtype=torch.float32, device="cuda")
    L.spmm8(x, y, y_dtype=1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = B.crisp_encode8(d_w, 1024, L.mask, L.buf8)
        L.spmm8(x, y, y_dtype=1)
    rng = np.random.default_rng(15)
    for _ in range(3):
        wb, xb = bits_of(rng.standard_normal((384, 1024))), activations(rng, 1024, 24)
        d_w.copy_(bf16_dev(wb, torch))
        x.copy_(bf16_dev(xb, torch))
        graph.replay()
        torch.cuda.synchronize()
        held = ref.weights(wl.bf16_bits_to_f32(wb).astype(np.float64), np.ones((384, 1024), bool))
        check(numbers(y), held, ref.activations(wl.bf16_bits_to_f32(xb).astype(np.float64)), 1024, 1)
    B.crisp_destroy8(again)


def test_encode_and_multiply_in_a_row_on_a_side_stream():
    """The product begins to fetch weights while X is quantised; an encode right in front of it has finished by then."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, _, _ = layer(B, torch, 1024, 2048, 4, 4, 1.0, 16)
    rng = np.random.default_rng(17)
    w = [bf16_dev(bits_of(rng.standard_normal((1024, 2048))), torch) for _ in range(2)]
    x = [bf16_dev(activations(rng, 2048, 9), torch) for _ in range(2)]
    want = {}
    for i in range(2):
        for j in range(2):
            L.encode8(w[i])
            torch.cuda.synchronize()
            want[i, j] = L.spmm8(x[j])
            torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    with torch.cuda.stream(side):
        for n in range(60):
            L.encode8(w[n % 2])
            got.append((n % 2, n // 2 % 2, L.spmm8(x[n // 2 % 2])))
    side.synchronize()
    assert all(torch.equal(y, want[i, j]) for i, j, y in got)


def test_host_threads_share_a_layer():
    import threading
    import torch
    from paper_2311_14272_b200 import binding as B
    L, _, _ = layer(B, torch, 512, 1024, 4, 4, 0.5, 18)
    rng = np.random.default_rng(19)
    xs = [bf16_dev(activations(rng, 1024, n), torch) for n in (1, 33, 300, 64)]
    want = [L.spmm8(x) for x in xs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(40):
                if not torch.equal(L.spmm8(xs[i]), want[i]):
                    wrong.append(i)
        stream.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


def test_prune_fine_tune_and_serve_in_8_bits():
    """Mask, two steps of AdamW with 8-bit states under it, the result in 8 bits, two layers in a row for some tokens."""
    import torch
    from paper_2311_14272_b200 import binding as B
    rng = np.random.default_rng(20)
    shapes = [(384, 256), (130, 384)]
    weights = [bf16_dev(bits_of(rng.standard_normal(s) * 0.05), torch) for s in shapes]
    net = B.PruningNetwork(shapes, 2, 4, 128, 128)
    net.step(weights, [[to_dev(rng.standard_normal(s).astype(np.float32), torch)] for s in shapes], 0.6)
    opt = net.optimizer(weights, state_bits=8, seed=1)
    for _ in range(2):
        opt.step([to_dev(rng.standard_normal(s).astype(np.float32), torch) for s in shapes])
    x = bits_of(rng.standard_normal((256, 20)))
    y = bf16_dev(x, torch).t().contiguous()
    for L, w in zip(net.layers, weights):
        L.encode8(w)
        rows, k = w.shape
        mask = np.unpackbits(L.export_mask()[1].view(np.uint8), axis=1, bitorder="little")[:rows, :k].astype(bool)
        assert not numbers(w)[~mask].any()
        held = ref.weights(numbers(w), mask)
        assert np.array_equal(numbers(L.decode8()), held)
        before = ref.activations(numbers(y).T)
        y = L.set_epilogue8(None, relu=True).spmm8(y, tokens=True)
        check(numbers(y.t()), held, before, k, 0, relu=True)
    net.close()


def test_the_first_products_of_a_process_may_be_captured():
    """A process whose first product of each kind is captured: nothing that a call looks up once is refused in a capture."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2311_14272_b200 import binding as B
torch.manual_seed(0)
L = B.HybridLayer(300, 700, 4, 4, 128, 128, 1.0).build_mask(torch.rand(300, 700, device="cuda"))
w = torch.randn(300, 700, device="cuda").bfloat16()
L.encode8(w)
xs = [torch.randn(n, 700, device="cuda").bfloat16() for n in (1, 9, 40, 400, 3000)]
opt = B.AdamW([w], state_bits=8)
g = torch.randn(300, 700, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    ys = [L.spmm8(x, tokens=True) for x in xs]
    zs = [L.spmm8(x.t().contiguous()) for x in xs]
graph.replay()
torch.cuda.synchronize()
for x, y, z in zip(xs, ys, zs):
    assert torch.equal(L.spmm8(x, tokens=True), y) and torch.equal(L.spmm8(x.t().contiguous()), z)
graph2 = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph2):
    opt.step([g])
    m, root = opt.moments()
graph2.replay()
torch.cuda.synchronize()
assert m.abs().sum() > 0 and root.min() >= 0
print("captured")
"""
    env = dict(os.environ, PYTHONPATH=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, env=env)
    assert out.stdout.strip().endswith("captured"), out.stderr[-2000:]


@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("rows,k,n,ncols,keep", [(128, 1024, 4, 40, 0.25), (256, 1000, 2, 700, 0.25), (300, 4100, 4, 129, 0.1), (100, 9000, 4, 33, 0.5)])
def test_what_no_row_tile_keeps_is_not_read(rows, k, n, ncols, keep, tokens):
    """NaN in X under blocks that no row tile kept changes nothing, with the masks of two encodings into one buffer."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, mask = layer(B, torch, rows, k, n, 4, keep, 31)
    rng = np.random.default_rng(32)
    x = activations(rng, k, ncols)
    for again in range(2):
        if again:
            score = rng.random((rows, k)).astype(np.float32)
            L.build_mask(to_dev(score, torch))
            words = L.export_mask()[1]
            mask = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:rows, :k].astype(bool)
            dense = rng.standard_normal((rows, k))
            L.encode8(bf16_dev(bits_of(dense), torch))
            w = ref.weights(wl.bf16_bits_to_f32(bits_of(dense)).astype(np.float64), mask)
        kept = np.array([mask[:, b * 128:(b + 1) * 128].any() for b in range((k + 127) // 128)])
        assert kept.any() and not kept.all()
        spoilt = x.copy()
        spoilt[~np.repeat(kept, 128)[:k]] = 0x7FC0
        y = []
        for bits in (x, spoilt):
            d_x = bf16_dev(np.ascontiguousarray(bits.T if tokens else bits), torch)
            out = L.spmm8(d_x, y_dtype=1, tokens=tokens)
            y.append(numbers(out.t() if tokens else out))
        assert np.array_equal(y[0], y[1])
        check(y[1], w, ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64)), k, 1)


@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("k,ncols", [(1100, 77), (600, 300), (4200, 2500)])
def test_activations_at_any_even_address(k, ncols, tokens):
    """Every address and pitch of activations gives the bits of the aligned ones; what lies around them, NaN, is in no result."""
    import torch
    from paper_2311_14272_b200 import binding as B
    L, _, _ = layer(B, torch, 128, k, 4, 4, 1.0, 41)
    x = torch.randn(k, ncols, device="cuda").bfloat16()
    x[torch.rand(k, ncols, device="cuda") < 0.001] *= 500
    x = x.t().contiguous() if tokens else x
    rows, cols = x.shape
    want = None
    for pitch in (-cols % 8, -cols % 8 + 1, -cols % 8 + 2, -cols % 8 + 3, 7 + -cols % 8, 4 + -cols % 8):
        for odd in (0, 1, 2, 3, 4, 5, 7) if want is not None else (0,):
            whole = torch.full((rows * (cols + pitch) + odd + 16,), float("nan"), dtype=torch.bfloat16, device="cuda")
            d_x = whole[odd:odd + rows * (cols + pitch)].view(rows, cols + pitch)[:, :cols]
            d_x.copy_(x)
            y = L.spmm8(d_x, y_dtype=1, tokens=tokens)
            if want is None:
                want = y.clone()
            assert torch.equal(y, want) and not torch.isnan(y).any(), (pitch, odd)


@pytest.mark.parametrize("power_w,power_x", [(0, -100), (-60, -60), (60, 60), (100, 20), (-120, 110), (120, -120), (124, -133), (-133, 120), (-133, 30)])
@pytest.mark.parametrize("tokens,ncols", [(False, 1), (True, 4), (False, 5), (True, 12), (True, 40), (False, 300)])
def test_values_of_any_size_in_every_kernel(tokens, ncols, power_w, power_x):
    """On the CUDA cores, quantised within the product, and quantised apart, with scales whose product lies in fp32's range where one of them does not (tolerance
    as for the products above; sums below 2^-140 are not looked at)."""
    import torch
    from paper_2311_14272_b200 import binding as B
    rng = np.random.default_rng(43)
    k = 256
    L, w, _ = layer(B, torch, 200, k, 4, 4, 1.0, 43, w=np.clip(rng.standard_normal((200, k)) * 2.0**power_w, -3e38, 3e38))
    x = bits_of(rng.standard_normal((k, ncols)) * 2.0**power_x)
    held = ref.activations(wl.bf16_bits_to_f32(x).astype(np.float64))
    d_x = bf16_dev(np.ascontiguousarray(x.T if tokens else x), torch)
    size = np.abs(w) @ np.abs(held)
    tol = (4 * np.sqrt(k) + 2) * 2.0**-23 * size + 2.0**-140
    for quantised in (False, True):
        y = numbers(L.spmm8(L.quantize8(d_x, tokens=tokens) if quantised else d_x, y_dtype=1, tokens=tokens))
        assert (L.last_launch8()["path"] == B.PATH_DIRECT) == (ncols <= 4 and not quantised)
        assert np.all(np.abs((y.T if tokens else y) - w @ held) <= tol)


@pytest.mark.parametrize("compiled", [True, False])
def test_an_encoding_that_is_refused_leaves_the_one_before_with_its_bias(compiled):
    import torch
    from paper_2311_14272_b200 import binding as B
    L, w, _ = layer(B, torch, 200, 300, 4, 4, 1.0, 44)
    if not compiled:
        L._gpu = None
    x = torch.randn(300, 9, device="cuda").bfloat16()
    L.set_epilogue8(torch.linspace(-1, 1, 200, device="cuda"), relu=True)
    want, bias, mask = L.spmm8(x), L._bias8, L.mask
    for bad_mask, bad_w in ((0, torch.zeros(200, 300, dtype=torch.bfloat16, device="cuda")), (mask, torch.zeros(200, 301, dtype=torch.bfloat16, device="cuda"))):
        L.mask = bad_mask
        with pytest.raises((B.CrispError, AssertionError)):
            L.encode8(bad_w)
        L.mask = mask
        # (the bias is still the layer's: what is allocated now does not take its place)
        assert L._bias8 is bias
        torch.full((200,), 5.0, device="cuda")
        assert torch.equal(L.spmm8(x), want)
    L.encode8(torch.zeros(200, 300, dtype=torch.bfloat16, device="cuda"))
    assert L._bias8 is None and not L.spmm8(x).any()


@pytest.mark.parametrize("keep", [1.0, 0.5])
def test_offsets_beyond_32_bits(keep):
    """Activations, then weights, of more than 2^32 elements: their last ones give the bits that they give alone."""
    import torch
    from paper_2311_14272_b200 import binding as B
    if torch.cuda.mem_get_info()[0] < 80e9:
        pytest.skip("needs 60 GB")
    k, n = 4096, 2**20 + 50_003
    L = B.HybridLayer(130, k, 4, 4, 128, 128, keep).build_mask(torch.rand(130, k, device="cuda"))
    L.encode8(torch.randn(130, k, device="cuda").bfloat16())
    L.set_tuning8(tile_cols=256, split=1)
    x = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    x[-1000:].normal_()
    want = L.spmm8(x[-1000:].clone(), tokens=True)
    for split in (1, -1) if keep == 1.0 else (1,):
        L.set_tuning8(tile_cols=256, split=split)
        y = L.spmm8(x, tokens=True)
        assert L.device_status8() == 0 and torch.equal(y[-1000:], want) and not y[:-1000].any()
    x = x.t().contiguous()
    y = L.spmm8(x)
    assert torch.equal(y[:, -1000:].t(), want) and not y[:, :-1000].any()
    del x, y
    score = torch.rand(n, k, device="cuda")
    w = torch.empty(n, k, dtype=torch.bfloat16, device="cuda").normal_()
    L = B.HybridLayer(n, k, 2, 4, 128, 128, keep).build_mask(score).encode8(w)
    at = (n - 1000) // 128 * 128
    last = B.HybridLayer(n - at, k, 2, 4, 128, 128, keep).build_mask(score[at:].clone()).encode8(w[at:].clone())
    assert torch.equal(L.decode8()[at:], last.decode8())
    for ncols in (3, 40):
        x = torch.randn(ncols, k, device="cuda").bfloat16()
        for one in (L, last):
            one.set_tuning8(tile_cols=64, split=1)
        assert torch.equal(L.spmm8(x, tokens=True)[:, at:], last.spmm8(x, tokens=True)) and L.device_status8() == 0
    del L, last, score, w
    torch.cuda.empty_cache()


def test_pairs_of_sms_on_two_streams_and_in_graphs_at_once():
    import torch
    from paper_2311_14272_b200 import binding as B
    L, _, _ = layer(B, torch, 700, 1024, 4, 4, 1.0, 45)
    rng = np.random.default_rng(46)
    xs = [bf16_dev(activations(rng, 1024, n), torch) for n in (3000, 2001)]
    L.set_tuning8(tile_cols=256, split=-1)
    want = [L.spmm8(x) for x in xs]
    assert L.last_launch8()["stack"] == -1
    torch.cuda.synchronize()
    streams, graphs, made = [torch.cuda.Stream() for _ in xs], [], []
    for x in xs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            made.append([L.spmm8(x) for _ in range(3)])
        graphs.append(graph)
    got = []
    for _ in range(20):
        for x, stream, graph in zip(xs, streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
                got.append(L.spmm8(x))
    torch.cuda.synchronize()
    assert L.device_status8() == 0
    assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(got))
    assert all(torch.equal(y, w) for ys, w in zip(made, want) for y in ys)
