"""Attention weights captured behind one append and replayed behind others: what a replay adds is drawn by
the queries of the append that is the last one then.  Tolerances as in test_gpu_weights.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

REL = 6e-5


def workspace(cache):
    """Scratch with a guard behind it, and the check that the guard is as it was."""
    need = cache.make_weights_workspace().numel()
    room = torch.full((need + (1 << 22),), 0x5A, dtype=torch.uint8, device="cuda")
    return room[:need], lambda: bool((room[need:] == 0x5A).all())


def holds(cache, sessions, lens, q, w):
    """w, from zeros, against 64 bits; what is not resident in these sessions, and others, untouched."""
    from tests import prompt_reference as R
    at = 0
    touched = torch.zeros_like(w, dtype=torch.bool)
    for s, t in zip(sessions, lens):
        k, v = R.held(cache, s)
        pos = torch.as_tensor(cache.export_state(s)["pos"], device="cuda")
        want = sum(R.attention(cache, s, q[layer, at:at + t], k[layer], v[layer])[1]
                   for layer in range(cache.cfg.layers))
        assert torch.allclose(w[s, pos].double(), want, rtol=REL, atol=1e-12), (s, t)
        touched[s, pos] = True
        at += t
    assert bool((w[~touched] == 0.0).all())


def replays(cache, first, others, rng):
    from tests import prompt_reference as R
    most = max(sum(x[1]) for x in [first] + others)
    q = R.queries(cache, most, rng)
    w = cache.make_weights()
    work, whole = workspace(cache)
    R.feed(cache, *first, rng)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        for layer in range(cache.cfg.layers):
            cache.attn_weights(layer, q[layer], w, work)
    for sessions, lens in [first] + others:
        if (sessions, lens) != first:
            R.feed(cache, sessions, lens, rng)
        w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert cache.device_status()[1] == 0
        holds(cache, sessions, lens, q, w)
        assert whole()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2])
def test_a_short_chunk_replayed_behind_long_ones(dtype, n):
    """The row statistics of a long chunk in as many parts as the short one's would not fit."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(n)
    cache = R.make_cache(n, dtype=dtype, heads=4, layers=1, pages=1000, positions=14000, tokens=7100)
    every = list(range(n))
    R.feed(cache, every, [7000] + [50] * (n - 1), rng)
    replays(cache, (every, [20] * n), [(every, [4000] + [33] * (n - 1)), (every, [2] * n),
                                       (every, [900] + [1] * (n - 1))], rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [7, 70])
def test_replayed_behind_other_sessions(dtype, tokens):
    """Fewer sessions (nothing of those before them counts), more, and in another order."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(tokens)
    cache = R.make_cache(6, dtype=dtype, heads=2, layers=2, pages=64, positions=1000)
    R.feed(cache, range(6), [300, 17, 150, 1, 64, 90], rng)
    replays(cache, ([4, 1, 0], [tokens] * 3), [
        ([2], [tokens]), ([5, 3, 0, 1, 2, 4], [tokens] * 6), ([0, 1], [tokens] * 2),
        ([3, 4, 5, 0], [tokens] * 4)], rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_tokens_replayed_behind_other_sessions(dtype):
    from tests import prompt_reference as R
    rng = np.random.default_rng(1)
    cache = R.make_cache(6, dtype=dtype, heads=2, layers=2, pages=64, positions=1000)
    R.feed(cache, range(6), [300, 17, 150, 1, 64, 90], rng)
    replays(cache, ([4, 1, 0], [1] * 3), [([5, 0, 2], [1] * 3), ([0, 1, 2], [1] * 3)], rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sessions, lens", [([0, 1], [1, 2]), ([0], [40]), ([0], [2]), ([1], [1]),
                                            ([2, 1, 0], [1, 1, 1])])
def test_single_tokens_replayed_behind_other_chunks_are_refused(dtype, sessions, lens):
    """Captured for a token of each of two sessions, replayed behind others: the error word says so, and
    nothing is added."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(3)
    cache = R.make_cache(3, dtype=dtype)
    work, w = cache.make_weights_workspace(), cache.make_weights()
    R.feed(cache, [0, 1, 2], [100, 30, 500], rng)
    R.feed(cache, [0, 1], [1, 1], rng)
    q = R.queries(cache, 40, rng)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        cache.attn_weights(0, q[0], w, work)
    graph.replay()
    torch.cuda.synchronize()
    assert cache.device_status()[1] == 0 and bool((w != 0).any())
    R.feed(cache, sessions, lens, rng)
    before = w.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, before)
    assert cache.device_status()[1] == 32
