"""Attention weights drawn by each position (kvc_attn_weights) against 64 bits.

Tolerances.  binary32: a score is a sum of D products of numbers around 1, divided by sqrt(D): each of
its roundings is 2^-24 of a partial sum, together below D * 2^-24 * |s| < 1e-5 for |s| < 8 (and 2^-24 sqrt(D)
in the mean); a weight p has the relative error of its score and its row's sum, sums of weights no
more.  bfloat16 rows: q in two pieces keeps 16 bits, so that a score is off by up to
2^-17 * sum |q k| / sqrt(D) < 2^-17 * 0.8 * 0.8 * 128 / 11.3 = 6e-5 at worst, its row's sum by the mean of
such; with rounding of alike signs in no two products the error is 11 times smaller."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

REL = 6e-5


def check(cache, sessions, lens, rng, work, weights=None):
    from tests import prompt_reference as R
    total = int(np.sum(lens))
    q = R.queries(cache, total, rng)
    w = cache.make_weights() if weights is None else weights
    before = w.clone()
    for layer in range(cache.cfg.layers):
        cache.attn_weights(layer, q[layer], w, work)
    assert cache.device_status()[1] == 0
    at = 0
    touched = torch.zeros_like(w, dtype=torch.bool)
    for s, t in zip(sessions, lens):
        k, v = R.held(cache, s)
        pos = torch.as_tensor(cache.export_state(s)["pos"], device="cuda")
        want = before[s, pos].double()
        for layer in range(cache.cfg.layers):
            want += R.attention(cache, s, q[layer, at:at + t], k[layer], v[layer])[1]
        got = w[s, pos].double()
        assert torch.allclose(got, want, rtol=REL, atol=1e-12), (s, (got / want - 1).abs().max())
        touched[s, pos] = True
        at += t
    assert torch.equal(w[~touched], before[~touched])
    return w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [1, 2, 5])
@pytest.mark.parametrize("lens", [[1], [1, 1, 1], [2], [17, 3, 32], [1, 40], [129, 1, 300]])
def test_weights_of_chunks(dtype, heads, lens):
    from tests import prompt_reference as R
    rng = np.random.default_rng([heads, len(lens), lens[0]])
    n = len(lens)
    cache = R.make_cache(n, dtype=dtype, heads=heads)
    work = cache.make_weights_workspace()
    sessions = list(range(n))
    R.feed(cache, sessions, lens, rng)                       # no history
    w = check(cache, sessions, lens, rng, work)
    R.feed(cache, sessions, [131 + 50 * i for i in range(n)], rng)
    R.feed(cache, sessions, lens, rng)
    check(cache, sessions, lens, rng, work, w)               # added to what is there


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, history", [([1100, 600], 0), ([1057, 1, 300], 520), ([2113], 33)])
def test_weights_of_chunks_in_shares(dtype, lens, history):
    """Chunks whose tokens are shared out: shares that see some tiles of an item's keys alone, or none."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(lens[0])
    n = len(lens)
    cache = R.make_cache(n, dtype=dtype, heads=2, pages=300, positions=2304)
    work = cache.make_weights_workspace()
    if history:
        R.feed(cache, list(range(n)), [history] * n, rng)
    R.feed(cache, list(range(n)), lens, rng)
    check(cache, list(range(n)), lens, rng, work)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1, 1], [9, 31], [70, 5]])
def test_weights_over_evicted_sessions(dtype, lens):
    from tests import prompt_reference as R
    rng = np.random.default_rng(len(dtype) + lens[0])
    cache = R.make_cache(3, dtype=dtype, budget=100, window=2)
    work = cache.make_weights_workspace()
    R.feed(cache, [0, 1, 2], [333, 150, 17], rng)
    cache.evict([0, 1, 2])
    R.feed(cache, [2, 0], lens, rng)                         # another order than the ids
    check(cache, [2, 0], lens, rng, work)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1], [5], [100]])
def test_weights_repeat_bit_for_bit(dtype, lens):
    from tests import prompt_reference as R
    rng = np.random.default_rng(1)
    cache = R.make_cache(1, dtype=dtype)
    work = cache.make_weights_workspace()
    R.feed(cache, [0], [700], rng)
    R.feed(cache, [0], lens, rng)
    q = R.queries(cache, sum(lens), rng)
    got = []
    for fill in (0, 0xFF):
        work.fill_(fill)  # (what the scratch holds does not matter)
        w = cache.make_weights()
        cache.attn_weights(1, q[1], w, work)
        got.append(w)
    assert torch.equal(got[0], got[1])
    assert abs(float(got[0].double().sum()) - 8 * sum(lens)) < 1e-4 * 8 * sum(lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 20, 90])
def test_what_no_token_sees_does_not_count(dtype, t):
    """NaN in freed pages that are used again, and in keys behind a token, draw nothing from it."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(t)
    cache = R.make_cache(2, dtype=dtype, pages=16, n_pages=17)
    work = cache.make_weights_workspace()
    types = torch.zeros(250, dtype=torch.uint8, device="cuda")
    nan = torch.full((2, 250, 2, cache.cfg.head_dim), torch.nan, dtype=cache.torch_dtype, device="cuda")
    cache.append_chunk([1], [0, 250], types, nan, nan)
    cache.release([1])
    R.feed(cache, [0], [21], rng)
    k, v = R.rows(cache, t, rng), R.rows(cache, t, rng)
    if t > 1:
        k[:, -1] = torch.nan
    cache.append_chunk([0], [0, t], types[:t], k, v)
    q = R.queries(cache, t, rng)
    if t > 1:
        # The last token sees its own key: its row is NaN and so are all sums; without it nothing is.
        w = cache.make_weights()
        cache.attn_weights(0, q[0], w, work)
        assert torch.isnan(w[0, :21 + t]).all() and torch.equal(w[1], torch.zeros_like(w[1]))
    else:
        check(cache, [0], [t], rng, work)


def test_captured_and_replayed():
    from tests import prompt_reference as R
    rng = np.random.default_rng(8)
    cache = R.make_cache(2)
    work = cache.make_weights_workspace()
    R.feed(cache, [0, 1], [90, 300], rng)
    R.feed(cache, [0, 1], [1, 1], rng)
    q = R.queries(cache, 2, rng)
    want = cache.make_weights()
    cache.attn_weights(0, q[0], want, work)
    w = cache.make_weights()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        cache.attn_weights(0, q[0], w, work)
    for _ in range(2):
        w.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, before", [([5], [4500]), ([64], [4095]), ([2, 33], [40, 3001])])
def test_weights_of_short_chunks_behind_long_histories(dtype, lens, before):
    """Row statistics in parts of the keys, more of them than are read at once."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(lens[0])
    n = len(lens)
    cache = R.make_cache(n, dtype=dtype, heads=1, pages=300, positions=4608, tokens=8192)
    work = cache.make_weights_workspace()
    R.feed(cache, list(range(n)), before, rng)
    R.feed(cache, list(range(n)), lens, rng)
    check(cache, list(range(n)), lens, rng, work)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("most", [1, 40])
def test_weights_of_many_sessions(dtype, most):
    from tests import prompt_reference as R
    rng = np.random.default_rng(most)
    n = 150
    cache = R.make_cache(n, dtype=dtype, layers=1, heads=1, pages=12, tokens=8192)
    work = cache.make_weights_workspace()
    lens = [int(x) for x in rng.integers(1, most + 1, size=n)]
    R.feed(cache, list(range(n)), [int(x) for x in rng.integers(1, 100, size=n)], rng)
    order = [int(x) for x in rng.permutation(n)]
    R.feed(cache, order, lens, rng)
    check(cache, order, lens, rng, work)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_chunk_captured_and_replayed(dtype):
    """With a scratch of its own, while an eager call uses another: the same bits."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(3)
    cache = R.make_cache(2, dtype=dtype, pages=120)
    R.feed(cache, [0, 1], [1200, 30], rng)
    R.feed(cache, [0, 1], [40, 9], rng)
    q = R.queries(cache, 49, rng)
    want, w = cache.make_weights(), cache.make_weights()
    cache.attn_weights(1, q[1], want, cache.make_weights_workspace())
    work = cache.make_weights_workspace()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        cache.attn_weights(1, q[1], w, work)
    for _ in range(2):
        w.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, want)
