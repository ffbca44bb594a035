"""Attention weights with more KV heads than are formed at once, and binary32 held to binary32's bound.

binary32: a score is off by less than D * 2^-24 * |s| < 1e-5 for |s| < 2.6 (all its 64 roundings of one sign),
2^-24 * 8 * |s| < 4e-6 for |s| < 8 in the mean, its row's sum by no more: 1e-5.  bfloat16: 6e-5, as in
test_gpu_weights.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [8, 9, 16, 21, 64])
@pytest.mark.parametrize("lens", [[1], [1, 1, 1], [3, 1], [40]])
def test_many_heads(dtype, heads, lens):
    from tests import prompt_reference as R
    rng = np.random.default_rng([heads, len(lens)])
    n = len(lens)
    cache = R.make_cache(n, dtype=dtype, heads=heads, layers=1, pages=40, positions=600)
    work, w = cache.make_weights_workspace(), cache.make_weights()
    R.feed(cache, range(n), [311 - 100 * i for i in range(n)], rng)
    R.feed(cache, range(n), lens, rng)
    q = R.queries(cache, sum(lens), rng)
    cache.attn_weights(0, q[0], w, work)
    assert cache.device_status()[1] == 0
    at = 0
    for s, t in zip(range(n), lens):
        k, v = R.held(cache, s)
        want = R.attention(cache, s, q[0, at:at + t], k[0], v[0])[1]
        got = w[s, :len(want)].double()
        assert torch.allclose(got, want, rtol=6e-5 if dtype == "bf16" else 1e-5, atol=1e-12), s
        assert bool((w[s, len(want):] == 0).all())
        at += t
