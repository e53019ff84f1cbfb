"""Calls on another stream than the current one: what they allocate is the call's stream's, so that nothing that is still queued on the current one
reads or writes it."""
import pytest

pytestmark = pytest.mark.gpu


def test_memory_is_allocated_for_the_stream_of_a_call():
    import torch
    from paper_2311_14272_b200 import binding as B
    side = torch.cuda.Stream()
    for current in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(current):
            here = torch.cuda.current_stream().cuda_stream
            for stream, want in ((None, here), (0, 0), (side, side.cuda_stream), (side.cuda_stream, side.cuda_stream), (torch.cuda.default_stream(), 0)):
                with B._allocating_for(stream):
                    assert torch.cuda.current_stream().cuda_stream == want == B._stream(here if stream is None else stream)
            assert torch.cuda.current_stream().cuda_stream == here


def spoil_later(torch, shape, dtype):
    """Frees a tensor of that shape that the current stream goes on writing for a while (about 50 ms)."""
    torch.cuda._sleep(100_000_000)
    torch.full(shape, 77, dtype=dtype, device="cuda")


@pytest.mark.parametrize("compiled", [True, False])
@pytest.mark.parametrize("form", ["stream", "address"])
def test_8_bit_calls_do_not_write_what_the_current_stream_still_does(form, compiled, monkeypatch):
    import torch
    from paper_2311_14272_b200 import binding as B
    rows, k, ncols = 512, 1024, 96
    gen = torch.Generator("cuda").manual_seed(1)
    w = torch.randn(rows, k, device="cuda", generator=gen).bfloat16()
    x = torch.randn(ncols, k, device="cuda", generator=gen).bfloat16()

    def made():
        L = B.HybridLayer(rows, k, 4, 4, 128, 128, 1.0).build_mask(w.float().abs())
        opt = B.AdamW([w.float()], state_bits=8)
        opt.step([w.float()])
        return L, opt
    L, opt = made()
    L.encode8(w)
    act = L.quantize8(x, tokens=True)
    want = [L.decode8(), L.spmm8(x, tokens=True), L.spmm8(act, tokens=True), L.spmm8(x, tokens=True, y_dtype=1), *opt.moments()]
    L, opt = made()
    if not compiled:
        monkeypatch.setattr(B, "_network", False)
        L._gpu = None
    side = torch.cuda.Stream()
    stream = side if form == "stream" else side.cuda_stream
    torch.cuda.synchronize()
    size = B.crisp_encode8_sizes(L.mask)
    spoil_later(torch, (size,), torch.uint8)
    L.encode8(w, stream=stream)
    side.synchronize()
    got = []
    for call, shape, dtype in ((lambda: [L.decode8(stream=stream)], (rows, k), torch.bfloat16),
                               (lambda: [L.spmm8(x, tokens=True, stream=stream)], (ncols, rows), torch.bfloat16),
                               (lambda: [L.spmm8(L.quantize8(x, tokens=True, stream=stream), tokens=True, stream=stream)], (ncols, rows), torch.bfloat16),
                               (lambda: [L.spmm8(x, tokens=True, y_dtype=1, stream=stream)], (ncols, rows), torch.float32),
                               (lambda: opt.moments(stream=stream), (opt.elements,), torch.bfloat16)):
        spoil_later(torch, shape, dtype)
        spoil_later(torch, shape, dtype)
        got += call()
        side.synchronize()
        torch.cuda.synchronize()
    torch.cuda.synchronize()
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("compiled", [True, False])
@pytest.mark.parametrize("form", ["stream", "address"])
def test_products_and_pruning_do_not_write_what_the_current_stream_still_does(form, compiled, monkeypatch):
    """Encode, decode, products, convolutions and an iteration of pruning (which takes an address as the others do)."""
    import torch
    from paper_2311_14272_b200 import binding as B
    rows, k, ncols = 256, 576, 96
    gen = torch.Generator("cuda").manual_seed(2)
    w = torch.randn(rows, k, device="cuda", generator=gen).bfloat16()
    x = torch.randn(k, ncols, device="cuda", generator=gen).bfloat16()
    act = torch.randn(2, 8, 8, 64, device="cuda", generator=gen).bfloat16()
    grads = [[torch.randn(rows, k, device="cuda", generator=gen)]]

    def made():
        return B.HybridLayer(rows, k, 2, 4, 64, 64, 0.5).build_mask(w.float().abs()), B.PruningNetwork([(rows, k)], 2, 4, 64, 64)
    L, net = made()
    L.encode(w)
    want = [L.decode(), L.spmm(x), L.spmm(x, y_dtype=1), L.spmm_conv(act, 3, 3, 1), L.spmm_conv(act, 3, 3, 1, nhwc_out=True)]
    kept = net.step([w], grads, 0.7)
    want.append(net.layers[0].decode())
    sizes = [L.canonical_buf.numel(), L.exec_buf.numel()]
    L, net = made()
    if not compiled:
        monkeypatch.setattr(B, "_network", False)
        L._gpu = net.layers[0]._gpu = None
    side = torch.cuda.Stream()
    stream = side if form == "stream" else side.cuda_stream
    torch.cuda.synchronize()
    for size in sizes:
        spoil_later(torch, (size,), torch.uint8)
    L.encode(w, stream=stream)
    side.synchronize()
    got = []
    for call, shape, dtype in ((lambda: L.decode(stream=stream), (rows, k), torch.bfloat16),
                               (lambda: L.spmm(x, stream=stream), (rows, ncols), torch.bfloat16),
                               (lambda: L.spmm(x, y_dtype=1, stream=stream), (rows, ncols), torch.float32),
                               (lambda: L.spmm_conv(act, 3, 3, 1, stream=stream), (rows, 128), torch.bfloat16),
                               (lambda: L.spmm_conv(act, 3, 3, 1, stream=stream, nhwc_out=True), (2, 8, 8, rows), torch.bfloat16)):
        spoil_later(torch, shape, dtype)
        got.append(call())
        side.synchronize()
        torch.cuda.synchronize()
    assert net.step([w], grads, 0.7, stream=stream) == kept
    got.append(net.layers[0].decode(stream=stream))
    torch.cuda.synchronize()
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
    net.close()
