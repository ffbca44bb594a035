"""Attention over prompts captured behind one append and replayed behind others: each replay answers the
append that is the last one then, of other lengths, other numbers of sessions and other histories.

A launch cuts its items' keys into parts by the append that the host knows of; the partial results of a
replay's items have to fit in the same scratch.  Tolerances as in test_gpu_prompt.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def holds(cache, sessions, lens, q, out):
    """out[layer] against 64 bits, and the rows behind the last session as they were (7)."""
    from tests import prompt_reference as R
    at = 0
    for s, t in zip(sessions, lens):
        k, v = R.held(cache, s)
        for layer in range(cache.cfg.layers):
            want = R.attention(cache, s, q[layer, at:at + t], k[layer], v[layer])[0]
            got = out[layer, at:at + t].double()
            rel = 6e-3 if q.dtype == torch.bfloat16 else 1e-5
            assert (got - want).norm() <= rel * want.norm(), (s, t, layer)
        at += t
    assert bool((out[:, at:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [1, 4])
@pytest.mark.parametrize("first, others", [
    ([64], [[2000], [33], [700], [1]]),
    ([40, 90], [[1500, 800], [1, 1], [64, 65], [900]]),
    ([2000], [[50], [1500, 90]])])
def test_replayed_behind_other_chunks(dtype, heads, first, others):
    from tests import prompt_reference as R
    rng = np.random.default_rng([heads, first[0]])
    most = max(sum(x) for x in [first] + others)
    cache = R.make_cache(2, dtype=dtype, heads=heads, layers=2, pages=600, positions=9000)
    R.feed(cache, [0, 1], [3000, 77], rng)
    R.feed(cache, range(len(first)), first, rng)
    q = R.queries(cache, most, rng)
    out = torch.full((2, most + 3, *q.shape[2:]), 7.0, dtype=q.dtype, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        for layer in range(2):
            cache.attn_prompt(layer, q[layer], out[layer])
    for lens in [first] + others:
        if lens is not first:
            R.feed(cache, range(len(lens)), lens, rng)
        for _ in range(2):
            out.fill_(7.0)
            graph.replay()
        torch.cuda.synchronize()
        assert cache.device_status()[1] == 0
        holds(cache, range(len(lens)), lens, q, out)


@pytest.mark.parametrize("dtype, kv_bits", [("bf16", None), ("f32", None), ("bf16", 4), ("f32", 4)])
@pytest.mark.parametrize("n, tokens", [(1, 17), (1, 32), (3, 17), (40, 20)])
def test_short_chunks_replayed_behind_long_ones_are_refused(dtype, kv_bits, n, tokens):
    """The kernels of chunks of up to 32 tokens do nothing behind longer ones, and the error word says so."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(n)
    cache = R.make_cache(n, dtype=dtype, kv_bits=kv_bits, layers=1, pages=80)
    every = list(range(n))
    R.feed(cache, every, [50] * n, rng)
    R.feed(cache, every, [tokens] * n, rng)
    q = R.queries(cache, 4000, rng)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        cache.attn_prompt(0, q[0], out[0])
    graph.replay()
    R.feed(cache, every, [2] * n, rng)
    graph.replay()
    torch.cuda.synchronize()
    assert cache.device_status()[1] == 0 and bool((out[0, :tokens * n] != 7.0).any())
    R.feed(cache, every, [33] + [3] * (n - 1), rng)
    out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert cache.device_status()[1] == 32
    assert bool((out == 7.0).all())
