"""Prompts over keys that score -infinity, and over scores that are far apart: softmax as 64 bits have it.

A rotation mixes a key's dims in pairs (i, i + D / 2), which makes NaN of most infinities.  The slowest pair
turns by less than 0.6 over the positions here, so that a key (-infinity, 0) in it becomes (-infinity,
-infinity) from position 1 on, and a query (1, 0.8) there stays positive in both."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def slow_pair(x, a, b):
    d = x.shape[-1]
    x[..., d // 2 - 1] = a
    x[..., d - 1] = b
    return x


def rel_of(dtype):  # as derived in test_gpu_prompt.py
    return 6e-3 if dtype == "bf16" else 1e-5


def feed(cache, sessions, lens, k, v):
    n = int(np.sum(lens))
    cache.append_chunk(sessions, np.concatenate([[0], np.cumsum(lens)]),
                       torch.zeros(n, dtype=torch.uint8, device="cuda"), k, v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lost", [16, 31, 32, 33, 40, 130, 300, 3000])
@pytest.mark.parametrize("t", [33, 100])
def test_rows_whose_first_keys_score_minus_infinity(dtype, lost, t):
    from tests import prompt_reference as R
    rng = np.random.default_rng([lost, t])
    cache = R.make_cache(1, dtype=dtype, layers=1, pages=400, positions=5000)
    n = lost + 1
    k, v = R.rows(cache, n, rng), R.rows(cache, n, rng)
    feed(cache, [0], [n], slow_pair(k, -torch.inf, 0.0), v)
    w = cache.make_weights() + 1.0
    w[0, 0] = 0.0                         # position 0, whose key is NaN, goes
    cache.evict_weighted([0], [lost], w)
    k, v = R.rows(cache, t, rng), R.rows(cache, t, rng)
    k[0, t // 2] = slow_pair(k[0, t // 2], -torch.inf, 0.0)
    feed(cache, [0], [t], k, v)
    q = slow_pair(R.queries(cache, t, rng), 1.0, 0.8)
    out = torch.zeros_like(q)
    cache.attn_prompt(0, q[0], out[0])
    hk, hv = R.held(cache, 0)
    assert bool((hk[0, :lost, :, -1] == -torch.inf).all()) and not bool(torch.isnan(hk).any())
    want = R.attention(cache, 0, q[0], hk[0], hv[0])[0]
    assert bool(torch.isfinite(want).all()) and bool(torch.isfinite(out).all())
    d = (out[0].double() - want).norm(dim=-1) / want.norm(dim=-1)
    assert (out[0].double() - want).norm() <= rel_of(dtype) * want.norm() and float(d.max()) < 2.0 ** -5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", ["rising", "falling", "mixed"])
def test_scores_without_whole_numbers_between_them(dtype, sizes):
    """Scores of up to 2^90: each row takes the value of one key."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(len(sizes))
    cache = R.make_cache(1, dtype=dtype, layers=1, pages=40)
    t = 300
    size = 2.0 ** np.linspace(0.0, 90.0, t)
    size = {"rising": size, "falling": size[::-1], "mixed": rng.permutation(size)}[sizes]
    k, v = torch.zeros_like(R.rows(cache, t, rng)), R.rows(cache, t, rng)
    size = torch.as_tensor(size.copy(), device="cuda").float()[:, None]
    feed(cache, [0], [t], slow_pair(k, size, 0.0), v)
    q = slow_pair(R.queries(cache, t, rng), 1.0, 0.8)
    out = torch.zeros_like(q)
    cache.attn_prompt(0, q[0], out[0])
    hk, hv = R.held(cache, 0)
    want = R.attention(cache, 0, q[0], hk[0], hv[0])[0]
    # A row's largest score is 2^0.3 times its second and past 2^12 more than 500 above it, so that its
    # value is the key's own.  (Rows whose scores are all below that are left out: q rounded to bfloat16
    # moves them by whole numbers.)
    far = torch.cummax(size[:, 0], dim=0)[0] > 2.0 ** 13
    assert bool(torch.isfinite(out[0, far]).all()) and int(far.sum()) > 200
    assert (out[0, far].double() - want[far]).norm() <= rel_of(dtype) * want[far].norm()
