"""A graph of a decode step (positions, then each layer's fused write and attention) replayed past the
pool's last page: the append records its error on the device, and what was captured behind it changes
nothing, whichever shape its decode was captured in."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2609_31224_gb300 import KVCache  # noqa: E402

pytestmark = pytest.mark.gpu

TEXT = 3


# A captured launch is shaped for the pages that a session comes to hold: 12 give the 4-warp pair
# split, 80 the 16-warp one; 150 sessions of 4 pages stream-K.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,room,pool,steps", [(2, 12, 10, 50), (2, 80, 10, 50), (150, 4, 310, 8)])
def test_nothing_behind_a_failed_append_is_written(dtype, n, room, pool, steps):
    d = 128 if dtype == "bf16" else 64
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    heads, layers = 4, 2
    cache = KVCache(n_sessions=n, layers=layers, q_heads=4 * heads, kv_heads=heads, head_dim=d,
                    budget=-1, window=1, dtype=dtype, n_pages=pool, max_pages_per_session=room,
                    max_positions=16 * room, max_seq_per_call=n, max_tokens_per_call=64 * n)
    every = list(range(n))
    # Two sessions: 30 and 15 positions; 150: 21 of 24 and 129 of 15.
    lens = [30, 15] if n == 2 else [24] * 21 + [15] * 129
    cu = np.concatenate([[0], np.cumsum(lens)])
    x = torch.randn(layers, int(cu[-1]), heads, d, device="cuda", dtype=td)
    cache.append_chunk(every, cu, torch.full((int(cu[-1]),), TEXT, dtype=torch.uint8, device="cuda"),
                       x, x)
    k, v = (torch.empty(layers, n, heads, d, dtype=td, device="cuda") for _ in range(2))
    q = torch.randn(n, 4 * heads, d, device="cuda", dtype=td)
    out = torch.zeros(layers, n, 4 * heads, d, dtype=td, device="cuda")
    types = torch.full((n,), TEXT, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    one = list(range(n + 1))
    look = 100                                       # rows of each session that are compared

    def rows():
        got = cache.read_kv(every, [0] * n, [look * i for i in range(n + 1)], stream=stream)
        return [y.clone() for y in got]

    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            cache.append_chunk(every, one, types, None, None, stream=stream)
            for layer in range(layers):
                cache.attn_decode_kv_raw(layer, k[layer].data_ptr(), v[layer].data_ptr(),
                                         q.data_ptr(), out[layer].data_ptr(), stream.cuda_stream)
        for step in range(steps + 5):
            before = rows()
            k.fill_(step + 1)
            v.fill_(-step - 1)
            out.fill_(7.0)
            graph.replay()
            stream.synchronize()
            if cache.device_status()[1] != 0:
                break
            assert (out != 7.0).any()
        after = rows()
        stream.synchronize()
    # Two sessions: after 50 steps 80 and 65 positions take five pages each, the next needs an
    # eleventh.  150: 21 sessions of 24 positions reach 32 in 8 steps, the others hold two pages from their
    # second step on; the next asks for 21 pages more than the 300 that are in use.
    assert step == steps, step
    for a, b in zip(before, after):
        assert torch.equal(a, b)
    assert (out == 7.0).all()
