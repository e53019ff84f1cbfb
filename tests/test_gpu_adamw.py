"""AdamW over many tensors on the GPU against the same step in 64 bits, from the GPU's own weights and states before it, so that each step's error
is that of one step.

Tolerances.  u = 2^-24, half a step of fp32.  v is made by four roundings of terms that are not negative: 4u of it.  m by three, each of at most the size of
its larger term: 4u (|b1 m| + |(1 - b1) g|) + the constants' rounding, 6u in all.  sqrt adds u and halves v's error; the root's product, sum, the division (2 ulp = 4u), two
products and constants: 16u of the update plus m's error relative to it; w: 3u of its own size.  Held in 8 bits or as bf16 weights, a value differs from
the reference's by a whole step where that error crosses the threshold of the random rounding: it reaches at most 64u of the value = 2^-18, a code's step is 2^-4
of it or more, so a share of about 2^-14 of the values; a thousandth (and one) may."""
import numpy as np
import pytest

import adamw_reference as ref
from helpers import to_dev

pytestmark = pytest.mark.gpu
U = 2.0**-24


def make(torch, shapes, w32, g32, seed, pitch=0, odd=0):
    rng = np.random.default_rng(seed)
    out = []
    for sh in shapes:
        rows, k = sh
        def tensor(x, dtype):
            whole = torch.full((rows * (k + pitch) + odd + 8,), 7.0, dtype=dtype, device="cuda")
            view = whole[odd:odd + rows * (k + pitch)].view(rows, k + pitch)[:, :k]
            view.copy_(to_dev(x.astype(np.float32), torch))
            return whole, view
        size = np.exp(rng.standard_normal(sh) * 2) * 1e-2
        out.append((tensor(rng.standard_normal(sh) * 0.05, torch.float32 if w32 else torch.bfloat16),
                    tensor(rng.standard_normal(sh) * size * (rng.random(sh) > 0.05), torch.float32 if g32 else torch.bfloat16),
                    tensor(np.zeros(sh), torch.bfloat16)))
    return out


def masks_for(B, torch, shapes, n, m, block, keep, seed):
    rng = np.random.default_rng(seed)
    layers, bits = [], []
    for rows, k in shapes:
        L = B.HybridLayer(rows, k, n, m, block, block, keep)
        L.build_mask(to_dev(rng.random((rows, k)).astype(np.float32), torch))
        words = L.export_mask()[1]
        flat = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:rows, :k].astype(bool)
        layers.append(L)
        bits.append(flat.reshape(-1))
    return layers, bits


def numbers(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def states(opt, i, count):
    at = opt.starts[i]
    if opt.state_bits == 32:
        return numbers(opt.m[at:at + count]), numbers(opt.v[at:at + count])
    codes = [b[at:at + count].cpu().numpy() for b in (opt.m, opt.v)]
    exps = [b[at // 128:(at + count + 127) // 128].cpu().numpy() for b in (opt.m_exp, opt.v_exp)]
    return ref.decode(codes[0], exps[0], False), ref.decode(codes[1], exps[1], True)**2


def check_held(got, want, step, least=0.0):
    """Equal, but for few that lie a step beside it.  What is below 2^13 times `least` may also be off by that."""
    off = np.abs(got - want)
    assert np.all(off <= step * 1.0001 + np.where(np.abs(want) < 2.0**13 * least, least, 0.0))
    assert np.count_nonzero((off > step * 1e-6) & (np.abs(want) >= 2.0**13 * least)) <= 1 + got.size // 1000


def check_step(opt, weights, grads, copies, masks, scalars=None, grad_scale=None, torch=None):
    """One step of the optimizer, compared tensor by tensor."""
    scalars = scalars or {}
    before = [(numbers(w), numbers(g) if g is not None else None) + states(opt, i, w.numel()) for i, (w, g) in enumerate(zip(weights, grads))]
    t = opt.step_count + 1
    opt.step(grads, grad_scale=grad_scale)
    for i, (w, g, m, v) in enumerate(before):
        got_w, (got_m, got_v) = numbers(weights[i]), states(opt, i, w.size)
        if g is None:
            assert np.array_equal(got_w, w) and np.array_equal(got_m, m) and np.array_equal(got_v, v)
            continue
        if w.size == 0:
            continue
        scale = 1.0 if grad_scale is None else float(grad_scale)
        want_w, want_m, want_v = ref.step(w, g, m, v, t, masks[i], grad_scale=scale, **scalars)
        b1, b2 = scalars.get("betas", (0.9, 0.999))
        wide = np.abs(b1 * m) + np.abs((1 - b1) * g * scale)
        lr, eps = scalars.get("lr", 1e-3), scalars.get("eps", 1e-8)
        _, full_m, full_v = ref.step(w, g, m, v, t, None, grad_scale=scale, **scalars)
        update = abs(lr) / (1 - b1**t) / (np.sqrt(full_v) / np.sqrt(1 - b2**t) + eps)
        w_tol = 4 * U * (np.abs(w) + np.abs(want_w)) + update * (24 * U * np.abs(full_m) + 6 * U * wide)
        random = ref.hashes(opt.seed, t, i, w.size)
        if weights[i].dtype.itemsize == 4:
            assert np.all(np.abs(got_w - want_w) <= w_tol)
            if copies[i] is not None:
                assert torch.equal(copies[i], weights[i].bfloat16())
        else:
            step = ref.spacing(want_w, 7, -126)
            held = np.sign(want_w) * np.floor(np.abs(want_w) / step + (2 * (random >> np.uint64(21)).astype(np.float64) + 1) / 4096) * step
            off = np.abs(got_w - held)
            assert np.all(off <= step * 1.0001 + 2 * w_tol)
            assert np.count_nonzero(off > step * 1e-6) <= 1 + off.size // 100     # (small weights: the update's error against their own, smaller step)
        if opt.state_bits == 32:
            assert np.all(np.abs(got_m - want_m) <= 6 * U * wide)
            assert np.all(np.abs(got_v - want_v) <= 6 * U * np.abs(want_v))
        else:
            held, step, _ = ref.hold(want_m, (2 * (random & np.uint64(1023)).astype(np.float64) + 1) / 2048, False)
            check_held(got_m, held, step)
            held, step, _ = ref.hold(np.sqrt(want_v), (2 * (random >> np.uint64(10) & np.uint64(2047)).astype(np.float64) + 1) / 4096, True)
            # (v is a number of fp32: three roundings to multiples of 2^-149 are at most 2^-148 off, sqrt(v) then at most 2^-74)
            check_held(np.sqrt(got_v), held, step, 2.0**-74)
        if masks[i] is not None:
            out = ~masks[i]
            assert not got_w[out].any() and not got_m[out].any() and not got_v[out].any()


SHAPES = {
    "one": [(1, 1)],
    "ends": [(1, 127), (1, 128), (1, 129), (1, 2047), (1, 2048), (1, 2049), (3, 5)],
    "matrices": [(64, 27), (33, 136), (130, 257), (256, 1024), (1, 64)],
    "many": [(1 + i % 7, 1 + (i * 37) % 203) for i in range(150)],
}


@pytest.mark.parametrize("w32,g32", [(True, True), (True, False), (False, False), (False, True)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("which", list(SHAPES))
def test_steps_match_64_bits(which, bits, w32, g32):
    import torch
    from paper_2311_14272_b200 import binding as B
    shapes = SHAPES[which]
    data = make(torch, shapes, w32, g32, 5)
    weights, grads, copies = ([d[j][1] for d in data] for j in range(3))
    opt = B.AdamW(weights, copies=copies if w32 else None, state_bits=bits, seed=(3 << 32) + 17)
    for s in range(3):
        check_step(opt, weights, grads, copies, [None] * len(shapes), torch=torch)
        for g in grads:                                      # (another gradient for the next step; its old place is reused)
            g.copy_((torch.randn(g.shape, generator=torch.Generator("cuda").manual_seed(s), device="cuda") * 1e-2))


@pytest.mark.parametrize("pitch,odd", [(0, 1), (3, 0), (8, 0), (5, 3)])
@pytest.mark.parametrize("w32,bits", [(True, 32), (False, 8)])
def test_pitches_and_odd_addresses_and_what_lies_beside(pitch, odd, w32, bits):
    import torch
    from paper_2311_14272_b200 import binding as B
    shapes = [(17, 40), (5, 129), (9, 256)]
    data = make(torch, shapes, w32, False, 6, pitch, odd)
    weights, grads, copies = ([d[j][1] for d in data] for j in range(3))
    layers, bits_of = masks_for(B, torch, shapes, 2, 4, 32, 0.6, 1)
    opt = B.AdamW(weights, copies=copies if w32 else None, masks=layers, state_bits=bits)
    for _ in range(2):
        check_step(opt, weights, grads, copies, bits_of, torch=torch)
    for (rows, k), d in zip(shapes, data):
        for whole, _ in (d[0], d[2]):
            inside = torch.zeros_like(whole, dtype=torch.bool)
            inside[odd:odd + rows * (k + pitch)].view(rows, k + pitch)[:, :k] = True
            assert torch.all(whole[~inside] == 7.0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n,m,block,keep", [(2, 4, 64, 0.5), (1, 4, 32, 0.0), (2, 8, 128, 0.25), (4, 4, 32, 1.0), (3, 8, 32, 0.4)])
def test_masked_weights_become_zero_whatever_their_gradient(n, m, block, keep, bits):
    import torch
    from paper_2311_14272_b200 import binding as B
    shapes = [(96, 27), (64, 576), (130, 250)]
    data = make(torch, shapes, True, True, 7)
    weights, grads, copies = ([d[j][1] for d in data] for j in range(3))
    layers, bits_of = masks_for(B, torch, shapes, n, m, block, keep, 2)
    opt = B.AdamW(weights, copies=copies, masks=layers, state_bits=bits)
    for g, b in zip(grads, bits_of):
        bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda")
        out = torch.from_numpy(~b).cuda().view(g.shape)
        g[out] = bad[torch.arange(int(out.sum()), device="cuda") % 3]
    opt.step(grads)
    for i, b in enumerate(bits_of):
        m, v = states(opt, i, b.size)
        for x in (numbers(weights[i]), numbers(copies[i]), m, v):
            assert not x[~b].any() and np.all(np.isfinite(x))
    for g, b in zip(grads, bits_of):
        g[torch.from_numpy(~b).cuda().view(g.shape)] = 1.0
    check_step(opt, weights, grads, copies, bits_of, torch=torch)


def test_layers_that_got_no_mask_and_tensors_that_got_no_gradient():
    import torch
    from paper_2311_14272_b200 import binding as B
    shapes = [(64, 64), (8, 8), (0, 5), (40, 32)]
    data = make(torch, shapes, False, True, 8)
    weights, grads, copies = ([d[j][1] for d in data] for j in range(3))
    bare = B.HybridLayer(64, 64, 2, 4, 32, 32, 0.5)
    opt = B.AdamW(weights, masks=[bare, None, None, None], state_bits=8)
    check_step(opt, weights, [grads[0], None, grads[2], grads[3]], copies, [None] * 4, torch=torch)
    check_step(opt, weights, grads, copies, [None] * 4, torch=torch)
    B.AdamW([]).step([])


@pytest.mark.parametrize("scalars", [dict(lr=0.0), dict(betas=(0.0, 0.0)), dict(weight_decay=0.5, eps=1e-3), dict(betas=(0.95, 0.9999), lr=-1e-2)])
def test_scalars(scalars):
    import torch
    from paper_2311_14272_b200 import binding as B
    shapes = [(16, 300)]
    data = make(torch, shapes, True, True, 9)
    weights, grads, copies = ([d[j][1] for d in data] for j in range(3))
    opt = B.AdamW(weights, copies=copies, step=1000, **scalars)
    clip = torch.tensor([0.37], device="cuda")
    for grad_scale in (None, clip):
        check_step(opt, weights, grads, copies, [None], scalars, grad_scale, torch=torch)


def test_elements_that_are_not_finite_leave_their_block_as_it_would_be():
    import torch
    from paper_2311_14272_b200 import binding as B
    data = [make(torch, [(3, 200)], True, True, 10)[0] for _ in range(2)]
    a, b = (B.AdamW([d[0][1]], state_bits=8, seed=4) for d in data)
    at = [5, 130, 131, 400]
    grads = [d[1][1] for d in data]
    grads[0].view(-1)[at] = 0.0
    grads[1].view(-1)[at] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e30], device="cuda")
    a.step([grads[0]])
    b.step([grads[1]])
    keep = np.ones(600, bool)
    keep[at] = False
    wa, wb = (numbers(d[0][1]) for d in data)
    assert np.array_equal(wa[keep], wb[keep])
    assert np.all(np.isnan(wb[[5, 130, 131]])) and np.isfinite(wb[400])
    for x, y in zip(states(a, 0, 600), states(b, 0, 600)):
        assert np.all(np.isfinite(y))
        blocks = [1, 3, 4]                                   # (1e30 is finite: the block that holds it takes its scale from it, as m; its square is not)
        same = keep.copy()
        same[3 * 128:4 * 128] = False
        assert np.array_equal(x[same], y[same]), blocks
        assert not y[[5, 130, 131]].any()


@pytest.mark.parametrize("power", [-120, -60, -16, 3, 8, 30, 60])
def test_8_bit_states_of_any_size(power):
    """Gradients of about 2^power: scales near both ends of their range, beyond the one factor that both powers of two usually fit in."""
    import torch
    from paper_2311_14272_b200 import binding as B
    data = make(torch, [(5, 700)], True, True, 21)
    data[0][1][1].mul_(2.0**power)
    opt = B.AdamW([data[0][0][1]], state_bits=8)
    for _ in range(3):
        check_step(opt, [data[0][0][1]], [data[0][1][1]], [None], [None], torch=torch)


def test_averages_that_move_less_than_half_a_step_still_move():
    """sqrt(v) loses 0.05 % a step without gradients, its codes lie 3 to 6 % apart.  After 1000 steps v is 0.368 of what it was; the mean over 65536 elements of
    sqrt(v), whose random walk spreads by less than a step of 6 %, lies within a hundredth of sqrt(0.368)."""
    import torch
    from paper_2311_14272_b200 import binding as B
    w = torch.ones(65536, device="cuda")
    opt = B.AdamW([w], state_bits=8, lr=0.0)
    opt.step([torch.ones(65536, device="cuda")])
    before = numbers(opt.moments()[1]).mean()
    zero = torch.zeros(65536, device="cuda")
    for _ in range(1000):
        opt.step([zero])
    root = numbers(opt.moments()[1])
    assert abs(root.mean() / before / 0.999**500 - 1) < 0.01 + 0.03          # (E[u] falls by half a per mille; the variance of u adds up to 3 % to u^2's mean)
    assert root.std() / root.mean() < 0.3


def test_a_captured_step_goes_on_counting():
    import torch
    from paper_2311_14272_b200 import binding as B
    made = [make(torch, [(40, 129), (64, 64)], False, False, 11) for _ in range(2)]
    opts = []
    for data, capturable in zip(made, (False, True)):
        opts.append(B.AdamW([d[0][1] for d in data], state_bits=8, seed=9, capturable=capturable))
    grads = [[d[1][1] for d in data] for data in made]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opts[1].step(grads[1])
        with torch.cuda.graph(graph, stream=side):
            opts[1].step(grads[1])
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        graph.replay()
    for _ in range(5):
        opts[0].step(grads[0])
    torch.cuda.synchronize()
    assert int(opts[1].d_step) == 5
    # the bias corrections are made in fp32 on the device: a few values cross a rounding threshold
    for i in range(2):
        a, b = (numbers(made[j][i][0][1]) for j in range(2))
        assert np.mean(a != b) < 2e-3 and np.all(np.abs(a - b) <= np.maximum(np.abs(a), np.abs(b)) * 2.0**-6 + 1e-5)
    opts[1].d_lr.zero_()
    held = numbers(made[1][0][0][1])
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(numbers(made[1][0][0][1]), held)


def test_elements_beyond_32_bits():
    """The last elements of a tensor of 2^32 + 5000 (bf16 weights, 8-bit states, a mask-less row): their addresses and their random numbers."""
    import torch
    from paper_2311_14272_b200 import binding as B
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 30 GB")
    n, tail = 2**32 + 5000, 5000
    w = torch.full((n,), 0.75, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(50)
    values = (rng.standard_normal(tail) * 0.01).astype(np.float32)
    g[-tail:] = to_dev(values, torch).bfloat16()
    gt = numbers(g[-tail:])
    opt = B.AdamW([w], state_bits=8, seed=6)
    opt.step([g])
    want_w, want_m, want_v = ref.step(np.full(tail, 0.75), gt, np.zeros(tail), np.zeros(tail), 1)
    h = ref.hashes(6, 1, 0, tail, n - tail)
    m = ref.decode(opt.m[n - tail:n].cpu().numpy(), opt.m_exp[(n - tail) // 128:].cpu().numpy(), False)
    root = ref.decode(opt.v[n - tail:n].cpu().numpy(), opt.v_exp[(n - tail) // 128:].cpu().numpy(), True)
    assert (n - tail) % 128 == 0
    held, step, _ = ref.hold(want_m, (2 * (h & np.uint64(1023)).astype(np.float64) + 1) / 2048, False)
    check_held(m, held, step)
    held, step, _ = ref.hold(np.sqrt(want_v), (2 * (h >> np.uint64(10) & np.uint64(2047)).astype(np.float64) + 1) / 4096, True)
    check_held(root, held, step)
    step = ref.spacing(want_w, 7, -126)
    held = np.floor(want_w / step + (2 * (h >> np.uint64(21)).astype(np.float64) + 1) / 4096) * step
    off = np.abs(numbers(w[-tail:]) - held)
    assert np.all(off <= step * 1.0001) and np.count_nonzero(off) <= 50
    # (before them: no gradients, so weight decay alone moves the weights, by at most one rounding)
    assert not opt.m[:n - tail].any() and float((w[:1000].float() - 0.75).abs().max()) <= 0.004
    torch.cuda.empty_cache()


def test_autograd_is_told_that_weights_change():
    import torch
    from paper_2311_14272_b200 import binding as B
    for kind in (list, tuple):
        w = torch.nn.Parameter(torch.ones(4, 8, device="cuda"))
        loss = (w * w).sum()
        B.AdamW([w]).step(kind([torch.ones(4, 8, device="cuda")]))
        with pytest.raises(RuntimeError):
            loss.backward()


def test_a_scale_that_is_not_finite_leaves_pruned_weights_zero():
    import torch
    from paper_2311_14272_b200 import binding as B
    for bits in (8, 32):
        data = make(torch, [(64, 128)], False, True, 51)
        layers, bits_of = masks_for(B, torch, [(64, 128)], 2, 4, 32, 0.5, 3)
        opt = B.AdamW([data[0][0][1]], masks=layers, state_bits=bits)
        opt.step([data[0][1][1]], grad_scale=torch.tensor([float("inf")], device="cuda"))
        out = ~bits_of[0]
        assert not numbers(data[0][0][1])[out].any()
        m, v = states(opt, 0, out.size)
        assert not m[out].any() and not v[out].any()


def test_a_step_that_is_refused_changes_nothing():
    import torch
    from paper_2311_14272_b200 import binding as B
    w = torch.ones(8, 16, device="cuda")
    for capturable in (False, True):
        opt = B.AdamW([w], capturable=capturable)
        for bad in ([torch.ones(16, 8, device="cuda").t()], [torch.ones(8, 15, device="cuda")], [torch.ones(8, 16)], [torch.ones(8, 16, device="cuda").double()],
                    [torch.ones(8, 16, device="cuda").half()], [], [None, None]):
            with pytest.raises((AssertionError, B.CrispError)):
                opt.step(bad)
        opt.betas = (1.0, 0.999)
        with pytest.raises(B.CrispError):
            opt.step([torch.ones(8, 16, device="cuda")])
        assert opt.step_count == 0 and (not capturable or int(opt.d_step) == 0) and torch.all(w == 1) and not opt.m.any()
    with pytest.raises(AssertionError):
        B.AdamW([w, w])
    with pytest.raises(AssertionError):
        B.AdamW([w, w[1:3]])
    with pytest.raises(AssertionError):
        B.AdamW([w.half()])
    with pytest.raises(AssertionError):
        B.AdamW([w.bfloat16()], copies=[w.bfloat16()])
    other = B.HybridLayer(8, 20, 2, 4, 32, 32, 0.5).build_mask(torch.rand(8, 20, device="cuda"))
    with pytest.raises(B.CrispError) as e:
        B.AdamW([w], masks=[other]).step([torch.ones(8, 16, device="cuda")])
    assert e.value.code == B.BAD_SHAPE


def test_tuples_of_gradients_and_weights_that_have_moved():
    """The calls that the C++ path leaves to Python, and a parameter whose storage has been exchanged."""
    import torch
    from paper_2311_14272_b200 import binding as B
    got = []
    for kind in (list, tuple):
        w = torch.nn.Parameter(torch.linspace(-1, 1, 640, device="cuda").view(10, 64))
        opt = B.AdamW([w])
        g = torch.linspace(1, 2, 640, device="cuda").view(10, 64)
        opt.step(kind([g]))
        w.data = w.data.clone()
        opt.step(kind([g.bfloat16()]))
        got.append((w.detach().clone(), opt.m.clone(), opt.v.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert not torch.equal(got[0][0], torch.linspace(-1, 1, 640, device="cuda").view(10, 64))


def test_pitched_gradients_and_streams():
    """A gradient that a side stream makes, in rows 3 elements further apart; the step is issued there too."""
    import torch
    from paper_2311_14272_b200 import binding as B
    w = torch.randn(64, 100, device="cuda")
    start = numbers(w)
    opt = B.AdamW([w])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g = torch.zeros(64, 103, device="cuda")
        torch.cuda._sleep(2_000_000)
        g.fill_(0.5)
        opt.step([g[:, :100]], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want, _, _ = ref.step(start, np.full(6400, 0.5), np.zeros(6400), np.zeros(6400), 1)
    assert np.all(np.abs(numbers(w) - want) <= 1e-6 * (1 + np.abs(want)))


def test_the_same_step_gives_the_same_bits():
    import torch
    from paper_2311_14272_b200 import binding as B
    got = []
    for _ in range(2):
        data = make(torch, SHAPES["matrices"], False, False, 12)
        opt = B.AdamW([d[0][1] for d in data], state_bits=8, seed=1)
        for _ in range(3):
            opt.step([d[1][1] for d in data])
        got.append([d[0][0] for d in data] + [opt.m, opt.v, opt.m_exp, opt.v_exp])
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*got))


def test_prune_fine_tune_and_serve():
    """Algorithm 1's iteration with its fine-tuning: prune, two steps under the masks, encode what is left, multiply.  The pruned weights stay pruned, so
    the encoding stands for the whole of the weights."""
    import torch
    from paper_2311_14272_b200 import binding as B
    shapes = [(128, 256), (96, 128)]
    rng = np.random.default_rng(3)
    master = [to_dev((rng.standard_normal(s) * 0.1).astype(np.float32), torch) for s in shapes]
    weights = [w.bfloat16() for w in master]
    net = B.PruningNetwork(shapes, 2, 4, 32, 32)
    opt = net.optimizer(master, copies=weights)
    for kappa in (0.6, 0.8):
        grads = [[to_dev((rng.standard_normal(s) * 0.01).astype(np.float32), torch) for _ in range(2)] for s in shapes]
        net.step(weights, grads, kappa)
        masks = []
        for L, (rows, k) in zip(net.layers, shapes):
            masks.append(np.unpackbits(L.export_mask()[1].view(np.uint8), axis=1, bitorder="little")[:rows, :k].astype(bool).reshape(-1))
        for _ in range(2):
            check_step(opt, master, [to_dev((rng.standard_normal(s) * 0.01).astype(np.float32), torch) for s in shapes], weights, masks, torch=torch)
        x = to_dev(rng.standard_normal((256, 64)).astype(np.float32), torch).bfloat16()
        net.layers[0].encode(weights[0])
        assert torch.equal(net.layers[0].decode(), weights[0])
        y, want = net.layers[0].spmm(x).double(), weights[0].double() @ x.double()
        assert float((y - want).norm() / want.norm()) < 5e-3
    net.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_a_gradient_whose_square_leaves_fp32_moves_no_weight_later(bits):
    """|m| / sqrt(v) of gradients that fp32 can square is at most (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)) = 7.3, the corrections of early steps only lower it, and
    a step of lr = 1e-3 then moves a weight by 7.3e-3 and its decay; codes that are off by a step of 1/8 and 1/16 make less than 1e-2 of it.  (1 - b2) g^2 is beyond
    fp32 from 5.83e20 on: v is infinite there, held as 0 in 8 bits, and so has to be m."""
    import torch
    from paper_2311_14272_b200 import binding as B
    at, sizes = [0, 3, 130, 140, 255, 299], [6e20, -1e21, 1e30, -3e38, 5.7e20, -5.8e20]
    rng = np.random.default_rng(60)
    grads = [(rng.standard_normal(300) * 1e-2 * (s != 1)).astype(np.float32) for s in range(5)]
    got = []
    for outliers in (sizes, [0.0] * len(at)):
        w = torch.ones(300, device="cuda")
        opt = B.AdamW([w], state_bits=bits, seed=5)
        grads[0][at] = outliers
        before = numbers(w)
        for s, g in enumerate(grads):
            opt.step([to_dev(g, torch)])
            now = numbers(w)
            assert np.all(np.abs(now - before) <= 1e-2), s
            before = now
            if s == 0 and bits == 8 and outliers is sizes:
                m, v = states(opt, 0, 300)
                assert not m[at[:4]].any() and not v[at[:4]].any() and np.all(v[at[4:]] > 1e38) and np.all(np.abs(m[at[4:]]) > 1e19)
        got.append(now)
    # (the first block has no value that large beside those held as 0)
    others = np.setdiff1d(np.arange(128), at)
    assert np.array_equal(got[0][others], got[1][others])


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("which,value", [("d_lr", float("nan")), ("d_lr", float("inf")), ("d_step", 0), ("d_step", -3), ("lr", 1e39), ("weight_decay", -1e300)])
def test_scalars_that_are_not_finite_leave_pruned_weights_zero(which, value, bits):
    """(A step number below 1 makes the corrections infinite or NaN; 1e39 is a number of the host's and none of fp32.)"""
    import torch
    from paper_2311_14272_b200 import binding as B
    data = make(torch, [(64, 128), (3, 37)], True, True, 52)
    weights, grads = ([d[j][1] for d in data] for j in range(2))
    layers, bits_of = masks_for(B, torch, [(64, 128), (3, 37)], 2, 4, 32, 0.5, 3)
    opt = B.AdamW(weights, masks=layers, state_bits=bits, capturable=which.startswith("d_"))
    getattr(opt, which).fill_(value) if which.startswith("d_") else setattr(opt, which, value)
    for _ in range(2):
        opt.step(grads)
    for i, b in enumerate(bits_of):
        m, v = states(opt, i, b.size)
        assert not numbers(weights[i])[~b].any() and not m[~b].any() and not v[~b].any()


@pytest.mark.parametrize("bits", [8, 32])
def test_steps_that_count_on_the_device_on_any_stream(bits):
    """A stream, its address, the default stream's address 0: the counter goes up before the step on the stream that the step is on."""
    import torch
    from paper_2311_14272_b200 import binding as B
    side = torch.cuda.Stream()
    got = []
    for streams in ((None, None, None), (side, side.cuda_stream, 0)):
        w = torch.linspace(-1, 1, 640, device="cuda")
        g = torch.linspace(1, 2, 640, device="cuda")
        opt = B.AdamW([w], state_bits=bits, seed=2, capturable=True)
        for stream in streams:
            opt.step([g], stream=stream)
            torch.cuda.synchronize()
        with pytest.raises((AssertionError, B.CrispError)):
            opt.step([g[:5]], stream=streams[1])
        torch.cuda.synchronize()
        assert int(opt.d_step) == 3
        got.append((w, opt.m, opt.v))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("bits", [8, 32])
def test_an_lr_that_is_assigned_is_the_next_steps(bits):
    """As by a schedule, between steps and between replays of a captured one, where lr is kept on the device as where it is the host's."""
    import torch
    from paper_2311_14272_b200 import binding as B
    rates = [1e-2, 0.0, 3e-3, 1e-4]
    got = []
    for how in ("host", "device", "replayed"):
        w = torch.linspace(-1, 1, 640, device="cuda")
        g = torch.linspace(1, 2, 640, device="cuda")
        opt = B.AdamW([w], state_bits=bits, seed=2, lr=rates[0], capturable=how != "host")
        opt.step([g])
        torch.cuda.synchronize()
        if how == "replayed":
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                opt.step([g])
        for lr in rates[1:]:
            before = w.clone()
            opt.lr = lr
            assert opt.lr == pytest.approx(lr, rel=2.0**-23, abs=0)
            graph.replay() if how == "replayed" else opt.step([g])
            assert torch.equal(w, before) == (lr == 0.0)
        got.append((numbers(w), numbers(opt.m.float())))
    # (lr and the corrections are numbers of fp32 on the device: at most eight roundings in each of four updates of at most 1.01 lr in all, and one of w each)
    for w, m in got[1:]:
        assert np.all(np.abs(w - got[0][0]) <= 8 * U * 1.01 * sum(rates) + 4 * U) and np.array_equal(m, got[0][1])
    assert np.array_equal(got[1][0], got[2][0])


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("again", [False, True])
def test_what_is_saved_after_replays_goes_on_as_they_would(bits, again):
    """m, v, their exponents, the step count and the seed are all of an optimizer's state, also where replays of a captured step have counted."""
    import torch
    from paper_2311_14272_b200 import binding as B
    w = torch.linspace(-1, 1, 640, device="cuda").bfloat16()
    g = torch.linspace(1, 2, 640, device="cuda")
    opt = B.AdamW([w], state_bits=bits, seed=2, step=3, capturable=True)
    assert opt.step_count == 3
    opt.step([g])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([g])
    for _ in range(5):
        graph.replay()
    assert opt.step_count == 9 == int(opt.d_step)
    held = w.clone()
    other = B.AdamW([held], state_bits=bits, seed=opt.seed, capturable=True, step=opt.step_count if not again else 0)
    if again:
        other.step_count = opt.step_count
    for name in ("m", "v", "m_exp", "v_exp"):
        if getattr(opt, name) is not None:
            getattr(other, name).copy_(getattr(opt, name))
    graph.replay()
    other.step([g])
    torch.cuda.synchronize()
    assert other.step_count == opt.step_count == 10
    assert torch.equal(w, held) and torch.equal(opt.m, other.m) and torch.equal(opt.v, other.v)


@pytest.mark.parametrize("kind", [list, tuple])
def test_a_copy_that_was_given_up_is_not_written(kind):
    import torch
    from paper_2311_14272_b200 import binding as B
    w = [torch.ones(8, 16, device="cuda") for _ in range(2)]
    copies = [torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    g = kind(torch.ones(8, 16, device="cuda") for _ in range(2))
    opt = B.AdamW(w, copies=copies)
    opt.step(g)
    opt.copies[0] = None
    held = copies[0].clone()
    opt.step(g)
    assert torch.equal(copies[0], held) and not torch.equal(copies[0], w[0].bfloat16()) and torch.equal(copies[1], w[1].bfloat16())
    opt.copies[0] = copies[0]
    opt.step(g)
    assert all(torch.equal(c, x.bfloat16()) for c, x in zip(copies, w))


def test_weights_that_have_moved_to_another_device_are_refused(monkeypatch):
    """The states stay where they were made.  (One device is enough to see it: the states' device is said to be another.)"""
    import torch
    from paper_2311_14272_b200 import binding as B
    for kind in (list, tuple):
        w = torch.ones(8, 16, device="cuda")
        opt = B.AdamW([w])
        opt.step([torch.ones(8, 16, device="cuda")])
        held = w.clone(), opt.m.clone()
        opt.device = torch.device("cuda", 1)
        monkeypatch.setattr(B, "_current_device", lambda: 1)
        with pytest.raises(AssertionError):
            opt.step(kind([torch.ones(8, 16, device="cuda")]))
        monkeypatch.undo()
        torch.cuda.synchronize()
        assert torch.equal(w, held[0]) and torch.equal(opt.m, held[1]) and opt.step_count == 1


@pytest.mark.parametrize("bits", [8, 32])
def test_states_that_are_assigned_are_the_next_steps(bits):
    """As a checkpoint is read: the table of a step holds the buffers' addresses, so what is assigned goes into them."""
    import torch
    from paper_2311_14272_b200 import binding as B
    g = torch.linspace(1, 2, 640, device="cuda")
    first = B.AdamW([torch.linspace(-1, 1, 640, device="cuda")], state_bits=bits, seed=2, capturable=True, lr=1e-2)
    first.step([g])
    names = ["m", "v", "d_step", "d_lr"] + (["m_exp", "v_exp"] if bits == 8 else [])
    saved = {name: getattr(first, name).clone() for name in names}
    second = B.AdamW([first.weights[0].clone()], state_bits=bits, seed=2, capturable=True)
    for name in names:
        where = getattr(second, name).data_ptr()
        setattr(second, name, saved[name])
        assert getattr(second, name).data_ptr() == where and torch.equal(getattr(second, name), saved[name])
    for opt in (first, second):
        opt.step([g])
    assert torch.equal(first.weights[0], second.weights[0]) and all(torch.equal(getattr(first, name), getattr(second, name)) for name in names)
    for bad in (saved["m"][:-1], saved["m"].double()):
        with pytest.raises(AssertionError):
            second.m = bad
    if bits == 32:
        with pytest.raises(AssertionError):
            second.m_exp = saved["m"]
