"""Outputs that the binding makes for a call on another stream than the current one: their memory
belongs to the stream that fills it, and is not handed out again while readers on the current one
are at work."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2609_31224_gb300 import KVCache  # noqa: E402

pytestmark = pytest.mark.gpu

TRANSCRIPT, N = 2, 700
BUSY = 200_000_000  # cycles: about 0.1 s


def filled():
    """A cache with one session of N transcript positions, and their V."""
    cache = KVCache(n_sessions=1, layers=2, q_heads=8, kv_heads=2, head_dim=64, budget=-1, window=1,
                    dtype="f32", n_pages=64, max_pages_per_session=64, max_positions=1024,
                    max_seq_per_call=1, max_tokens_per_call=1024)
    v = torch.randn(2, N, 2, 64, device="cuda")
    cache.append_chunk([0], [0, N], torch.full((N,), TRANSCRIPT, dtype=torch.uint8, device="cuda"),
                       torch.randn_like(v), v)
    torch.cuda.synchronize()
    return cache, v


def stream_of(x):
    """The stream that the allocator keeps a tensor's memory for."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= x.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no segment")


def outputs(cache, call, stream):
    if call == "read":
        return cache.read_kv([0], [0], np.array([0, N]), stream=stream)
    pos, k, v, count = cache.export_transcript(0, N, stream=stream)
    return k, v, pos, count


CALLS = ["read", "transcript"]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("form", ["stream", "handle"])
def test_outputs_belong_to_the_stream_that_fills_them(call, form):
    cache, v = filled()
    side = torch.cuda.Stream()
    at = side if form == "stream" else side.cuda_stream
    outs = outputs(cache, call, at)
    side.synchronize()
    assert torch.equal(outs[1], v)
    for x in outs:
        assert stream_of(x) == side.cuda_stream
    for stream in (None, torch.cuda.current_stream(), torch.cuda.current_stream().cuda_stream):
        for x in outputs(cache, call, stream):
            assert stream_of(x) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):       # the default stream's handle is 0
        outs = outputs(cache, call, 0)
    torch.cuda.synchronize()
    assert torch.equal(outs[1], v)
    for x in outs:
        assert stream_of(x) == 0


@pytest.mark.parametrize("call", CALLS)
def test_a_dropped_output_waits_for_its_readers(call):
    """The current stream reads an output that was filled on another one; it is dropped before the
    read has run, and the other stream asks for memory of that size."""
    cache, v = filled()
    side = torch.cuda.Stream()
    outs = outputs(cache, call, side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(BUSY)
    got = outs[1].clone()
    places = {x.data_ptr() for x in outs}
    del outs
    with torch.cuda.stream(side):
        taken = [torch.full_like(v, 7.0) for _ in range(8)]
    assert not places & {y.data_ptr() for y in taken}
    torch.cuda.synchronize()
    assert torch.equal(got, v)


@pytest.mark.parametrize("call", CALLS)
def test_memory_still_in_use_on_the_current_stream_is_not_taken(call):
    """A kernel waits on the current stream to write a tensor that has been dropped already: an output
    for another stream is not made in its memory."""
    cache, v = filled()
    side = torch.cuda.Stream()
    late = [torch.empty_like(v) for _ in range(8)]
    torch.cuda._sleep(BUSY)
    for x in late:
        x.fill_(7.0)
    del late, x
    outs = outputs(cache, call, side)
    side.synchronize()
    assert torch.equal(outs[1], v)
    torch.cuda.synchronize()
    assert torch.equal(outs[1], v)


def test_a_transcript_is_not_cleared_behind_its_export():
    """The current stream is busy: what clears the outputs runs in front of the export all the same."""
    cache, v = filled()
    side = torch.cuda.Stream()
    torch.cuda._sleep(BUSY)
    pos, k, got, count = cache.export_transcript(0, N, stream=side)
    torch.cuda.synchronize()
    assert int(count) == N and pos.tolist() == list(range(N)) and torch.equal(got, v)
