"""What KVCache.read_kv refuses before it hands addresses to the library (no GPU needed: the library
is a stand-in that must not be called)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_31224_gb300 import _lib as L  # noqa: E402


class Called(Exception):
    pass


class Library:
    def kvc_read_kv(self, *args):
        raise Called


@pytest.fixture
def cache():
    c = object.__new__(L.KVCache)  # a context of two layers whose pool is on the CPU
    c.lib, c.ctx, c.torch_dtype = Library(), None, torch.bfloat16
    c.cfg = L.Config(layers=2, q_heads=8, kv_heads=2, head_dim=128)
    c.pool = torch.empty(0, dtype=torch.uint8)
    return c


def rows(n=3, **kw):
    return torch.empty((2, n, 2, 128), **{"dtype": torch.bfloat16, **kw})


def test_fitting_outputs_reach_the_library(cache):
    for kw in (dict(), dict(k=rows(), v=rows()), dict(resident_out=torch.zeros(2, dtype=torch.int64)),
               dict(resident_out=torch.zeros(5, dtype=torch.int64))):
        with pytest.raises(Called):
            cache.read_kv([0, 1], [0, 0], [0, 1, 3], stream=0, **kw)


@pytest.mark.parametrize("kw,word", [
    (dict(k=rows(device="meta")), "on cpu"),
    (dict(v=rows(device="meta")), "on cpu"),
    (dict(k=rows(4)), "shape"),
    (dict(v=rows(dtype=torch.float32)), "bfloat16"),
    (dict(k=rows(6)[:, ::2]), "contiguous"),
    (dict(resident_out=torch.zeros(2, dtype=torch.int32)), "resident_out"),
    (dict(resident_out=torch.zeros(1, dtype=torch.int64)), "resident_out"),
    (dict(resident_out=torch.zeros(4, dtype=torch.int64)[::2]), "resident_out"),
    (dict(resident_out=torch.zeros(2, dtype=torch.int64, device="meta")), "resident_out"),
])
def test_unfit_outputs_are_refused(cache, kw, word):
    with pytest.raises(ValueError, match=word):
        cache.read_kv([0, 1], [0, 0], np.array([0, 1, 3], np.int32), stream=0, **kw)
