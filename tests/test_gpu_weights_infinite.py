"""Attention weights over keys that hold infinities, NaN in places that nobody sees, and large scores.

Keys of -infinity score -infinity against the queries here (as in test_gpu_prompt_infinite.py) and weigh
nothing; everything else weighs as if they were not there.  Tolerances as in test_gpu_weights.py: 6e-5 for
bfloat16 rows, 1e-5 for binary32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def slow_pair(x, a, b):
    d = x.shape[-1]
    x[..., d // 2 - 1] = a
    x[..., d - 1] = b
    return x


def feed(cache, sessions, lens, k, v):
    n = int(np.sum(lens))
    cache.append_chunk(sessions, np.concatenate([[0], np.cumsum(lens)]),
                       torch.zeros(n, dtype=torch.uint8, device="cuda"), k, v)


def holds(cache, sessions, lens, q, w):
    from tests import prompt_reference as R
    rel = 6e-5 if q.dtype == torch.bfloat16 else 1e-5
    at = 0
    touched = torch.zeros_like(w, dtype=torch.bool)
    for s, t in zip(sessions, lens):
        k, v = R.held(cache, s)
        pos = torch.as_tensor(cache.export_state(s)["pos"], device="cuda")
        want = R.attention(cache, s, q[0, at:at + t], k[0], torch.nan_to_num(v[0]))[1]
        got = w[s, pos].double()
        assert bool(torch.isfinite(want).all())
        assert torch.allclose(got, want, rtol=rel, atol=1e-12), (s, (got - want).abs().max())
        touched[s, pos] = True
        at += t
    assert bool((w[~touched] == 0.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lost", [1, 16, 40, 300, 2000])
@pytest.mark.parametrize("lens", [[1], [1, 1], [2, 30], [33], [100, 7], [700]])
def test_keys_of_minus_infinity_weigh_nothing(dtype, lost, lens):
    from tests import prompt_reference as R
    rng = np.random.default_rng([lost, lens[0]])
    cache = R.make_cache(2, dtype=dtype, layers=1, pages=300, positions=4000)
    n = lost + 1
    k, v = R.rows(cache, n + 90, rng), R.rows(cache, n + 90, rng)
    slow_pair(k[:, :n], -torch.inf, 0.0)
    feed(cache, [0, 1], [n, 90], k, v)
    w = cache.make_weights() + 1.0
    w[0, 0] = 0.0                         # position 0, whose key is NaN, goes
    cache.evict_weighted([0], [lost], w)
    total = sum(lens)
    k, v = R.rows(cache, total, rng), R.rows(cache, total, rng)
    for at in range(3, total, 41):        # and some in the chunk
        slow_pair(k[:, at], -torch.inf, 0.0)
    sessions = list(range(len(lens)))
    feed(cache, sessions, lens, k, v)
    q = slow_pair(R.queries(cache, total, rng), 1.0, 0.8)
    w = cache.make_weights()
    cache.attn_weights(0, q[0], w, cache.make_weights_workspace())
    assert cache.device_status()[1] == 0
    holds(cache, sessions, lens, q, w)
    assert bool((w[0, 1:n] == 0.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 20, 90, 500])
def test_freed_pages_of_nan_used_again(dtype, t):
    """Every slot of the pool held NaN before; the chunk and its history are finite."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(t)
    cache = R.make_cache(2, dtype=dtype, pages=64, n_pages=65, layers=1)
    nan = torch.full((1, 1000, 2, cache.cfg.head_dim), torch.nan, dtype=cache.torch_dtype, device="cuda")
    feed(cache, [1], [1000], nan, nan)
    cache.release([1])
    R.feed(cache, [0], [21], rng)
    R.feed(cache, [0], [t], rng)
    q = R.queries(cache, t, rng)
    w = cache.make_weights()
    cache.attn_weights(0, q[0], w, cache.make_weights_workspace())
    holds(cache, [0], [t], q, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t, at", [(20, 13), (90, 64), (500, 300)])
def test_a_key_that_takes_everything_takes_nothing_before_it(dtype, t, at):
    """A key whose score is 2^14 above the others' has weight 1 from its own token on and 0 before."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(t)
    cache = R.make_cache(1, dtype=dtype, layers=1)
    R.feed(cache, [0], [45], rng)
    k, v = R.rows(cache, t, rng), R.rows(cache, t, rng)
    slow_pair(k[:, at], 2.0 ** 18, 0.0)
    feed(cache, [0], [t], k, v)
    q = slow_pair(R.queries(cache, t, rng), 1.0, 0.8)
    w = cache.make_weights()
    cache.attn_weights(0, q[0], w, cache.make_weights_workspace())
    holds(cache, [0], [t], q, w)
    assert float(w[0, 45 + at]) == 8.0 * (t - at)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 20, 90])
def test_what_is_not_a_number_by_definition_stays_so(dtype, t):
    """A NaN or an infinity in one session's last query makes its sums NaN, and no other session's."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(t)
    cache = R.make_cache(3, dtype=dtype, layers=1)
    R.feed(cache, [0, 1, 2], [60, 75, 200], rng)
    R.feed(cache, [0, 1, 2], [t] * 3, rng)
    q = R.queries(cache, 3 * t, rng)
    q[0, t - 1, 5, 3] = torch.nan
    q[0, 3 * t - 1, 0, 0] = torch.inf
    w = cache.make_weights()
    cache.attn_weights(0, q[0], w, cache.make_weights_workspace())
    assert bool(torch.isnan(w[0, :60 + t]).all()) and bool(torch.isnan(w[2, :200 + t]).all())
    w[0], w[2] = 0.0, 0.0
    at = q[:, t:2 * t]
    holds(cache, [1], [t], at, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 20, 90])
@pytest.mark.parametrize("at", [0, 1, 37, 199])
def test_a_key_that_is_not_a_number(dtype, t, at):
    """Every row that sees it is NaN, wherever it stands; other sessions are not."""
    from tests import prompt_reference as R
    rng = np.random.default_rng([t, at])
    cache = R.make_cache(2, dtype=dtype, layers=1)
    k, v = R.rows(cache, 260, rng), R.rows(cache, 260, rng)
    k[0, at] = torch.nan
    feed(cache, [0, 1], [200, 60], k, v)
    R.feed(cache, [0, 1], [t] * 2, rng)
    q = R.queries(cache, 2 * t, rng)
    w = cache.make_weights()
    cache.attn_weights(0, q[0], w, cache.make_weights_workspace())
    assert bool(torch.isnan(w[0, :200 + t]).all())
    w[0] = 0.0
    holds(cache, [1], [t], q[:, t:], w)
