"""Host checks of the calls on whole prompts: refusals come before any launch."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_31224_gb300 import _lib as L  # noqa: E402
from paper_2609_31224_gb300 import build as B  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    B.build()
    return L.load_library()


def config(**kw):
    base = dict(n_sessions=4, layers=2, q_heads=8, kv_heads=2, head_dim=128, page_size=16, budget=64,
                window=2, dtype=L.KVC_BF16, rope_base=10000.0, n_pages=100, max_pages_per_session=50,
                max_positions=500, max_seq_per_call=4, max_tokens_per_call=300)
    base.update(kw)
    return L.Config(**base)


def test_null_context_is_rejected(lib):
    s = (ctypes.c_int32 * 1)(0)
    assert lib.kvc_attn_prompt(None, 0, None, None, None) == -1
    assert lib.kvc_attn_weights(None, 0, None, None, None, 0, None) == -1
    assert lib.kvc_evict_weighted(None, 1, s, s, None, 15, 0, 0, None, None, None) == -1
    assert lib.kvc_last_error()


def test_workspace_follows_the_configuration(lib):
    n = ctypes.c_size_t()
    assert lib.kvc_weights_workspace(ctypes.byref(config()), ctypes.byref(n)) == 0
    # scores or sums by slot and query head, and a number by token and query head, at least
    assert n.value >= 100 * 16 * 8 * 4 + 300 * 8 * 4
    assert lib.kvc_weights_workspace(ctypes.byref(config()), None) == -1
    assert lib.kvc_weights_workspace(ctypes.byref(config(head_dim=64)), ctypes.byref(n)) == -1


class Fake(L.KVCache):
    """A cache without a device: arguments are checked before the library is called."""

    def __init__(self):
        self.cfg = config()
        self.pool = torch.zeros(1)
        self.ctx = None
        self.lib = None


@pytest.mark.parametrize("bad", [
    dict(weights=torch.zeros(4, 499)), dict(weights=torch.zeros(3, 500)),
    dict(weights=torch.zeros(4, 500, dtype=torch.float64)),
    dict(weights=torch.zeros(500, 4).T),
    dict(kept=torch.zeros(1, 500, dtype=torch.bool)), dict(kept=torch.zeros(2, 500, dtype=torch.uint8)),
    dict(resident_out=torch.zeros(2, dtype=torch.int32)), dict(resident_out=torch.zeros(1, dtype=torch.int64)),
    dict(keep=[1]),
])
def test_evict_weighted_checks_its_tensors(bad):
    kw = dict(sessions=[0, 1], keep=[3, 3], weights=torch.zeros(4, 500))
    kw.update(bad)
    with pytest.raises(ValueError):
        Fake().evict_weighted(**kw)


def test_attn_weights_checks_its_tensors():
    with pytest.raises(ValueError):
        Fake().attn_weights(0, torch.zeros(1), torch.zeros(4, 400), torch.zeros(8, dtype=torch.uint8))


@pytest.mark.gpu
def test_refusals_with_a_context():
    from tests import prompt_reference as R
    rng = np.random.default_rng(0)
    cache = R.make_cache(2)
    w, work = cache.make_weights(), cache.make_weights_workspace()
    q = torch.zeros((40, 8, 128), dtype=torch.bfloat16, device="cuda")

    def refused(code, call, *args, **kw):
        launches = cache.launches()
        with pytest.raises(L.KvcError) as e:
            call(*args, **kw)
        assert e.value.code == code and cache.launches() == launches

    refused(-4, cache.attn_prompt, 0, q, q)                      # no append yet
    refused(-4, cache.attn_weights, 0, q, w, work)
    R.feed(cache, [0], [40], rng)
    refused(-1, cache.attn_prompt, 2, q, q)                      # no such layer
    refused(-1, cache.attn_weights, -1, q, w, work)
    refused(-1, cache.attn_weights, 0, q, w, work[:-256])        # too little scratch
    refused(-1, cache.attn_weights, 0, q, w, work[1:])
    refused(-1, cache.evict_weighted, [0, 0], [1, 1], w)         # the same session twice
    refused(-1, cache.evict_weighted, [2], [1], w)
    refused(-1, cache.evict_weighted, [0], [-1], w)
    refused(-1, cache.evict_weighted, [0], [1], w, kinds=16)
    refused(-1, cache.evict_weighted, [0], [1], w, sink=-1)
    refused(-1, cache.evict_weighted, [0], [1], w, recent=-1)
    cache.evict_weighted([0], [10], w)
    refused(-4, cache.attn_prompt, 0, q, q)                      # the chunk's queries are gone
    refused(-4, cache.attn_weights, 0, q, w, work)
    small = R.make_cache(1, kv_bits=4)
    R.feed(small, [0], [40], rng)
    cache = small
    refused(-1, small.attn_prompt, 0, q, q)                      # rows in 4 bits, a long chunk
    refused(-1, small.attn_weights, 0, q, small.make_weights(), small.make_weights_workspace())
