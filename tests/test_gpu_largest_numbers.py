"""Prompts and attention weights over K and V with the element type's largest numbers, which are finite
and stay so: a key of them takes a row whole or not at all, a value of them comes through its weight.
Tolerances as in test_gpu_prompt.py and test_gpu_weights.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t, before", [(33, 20), (100, 300), (70, 3000)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("short", [0, 2.0 ** -13, 2.0 ** -11])
def test_largest_numbers(dtype, t, before, sign, short):
    from tests import prompt_reference as R
    rng = np.random.default_rng([t, before])
    cache = R.make_cache(1, dtype=dtype, layers=1, pages=300, positions=4000)
    R.feed(cache, [0], [before], rng)
    most = sign * torch.finfo(cache.torch_dtype).max * (1 - short)
    d = cache.cfg.head_dim
    k, v = R.rows(cache, t, rng), R.rows(cache, t, rng)
    k[0, t // 3, :, d // 2 - 1] = most            # turns little (test_gpu_prompt_infinite.py)
    k[0, t // 3, :, d - 1] = 0.0
    v[0, t // 2, :, 3] = most
    cache.append_chunk([0], [0, t], torch.zeros(t, dtype=torch.uint8, device="cuda"), k, v)
    q = R.queries(cache, t, rng)
    q[..., d // 2 - 1], q[..., d - 1] = 1.0, 0.8
    out, w = torch.zeros_like(q), cache.make_weights()
    cache.attn_prompt(0, q[0], out[0])
    cache.attn_weights(0, q[0], w, cache.make_weights_workspace())
    hk, hv = R.held(cache, 0)
    want, draws = R.attention(cache, 0, q[0], hk[0], hv[0])
    got, n = out[0].double(), before + t
    assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(want).all())
    rel, each = (6e-3, 6e-5) if dtype == "bf16" else (1e-5, 1e-5)
    # (The dims apart: one holds numbers of 10^38.)
    for dims in (slice(3, 4), [i for i in range(d) if i != 3]):
        assert (got[..., dims] - want[..., dims]).norm() <= rel * want[..., dims].norm()
    assert torch.allclose(w[0, :n].double(), draws, rtol=each, atol=1e-12)
