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
