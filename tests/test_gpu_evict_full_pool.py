"""A call of kvc_evict_weighted whose pages the pool does not have: the error word says so, and nothing of
any session of the call changes, the ones that needed no page included."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, kv_bits", [("bf16", None), ("f32", None), ("bf16", 4), ("f32", 4)])
@pytest.mark.parametrize("order", [[0, 1], [1, 0]])
def test_nothing_changes(dtype, kv_bits, order):
    from tests import prompt_reference as R
    rng = np.random.default_rng(6)
    cache = R.make_cache(2, dtype=dtype, kv_bits=kv_bits, heads=2, pages=8, n_pages=4, positions=200, tokens=200)
    w = torch.ones((2, 200), device="cuda")
    w[0, 17] = 0.0          # of 30 positions the 18th goes: 17 before it need a second page of their own
    R.feed(cache, [0, 1], [30, 30], rng)
    torch.cuda.synchronize()

    def all_of_it():
        n = torch.zeros(2, dtype=torch.int64, device="cuda")
        k, v = cache.read_kv([0, 1], [0, 0], [0, 30, 60], resident_out=n)
        torch.cuda.synchronize()
        return k.clone(), v.clone(), n.clone()

    before = all_of_it()
    states = [cache.export_state(s) for s in (0, 1)]
    resident = torch.full((2,), -7, dtype=torch.int64, device="cuda")
    kept = torch.zeros((2, 200), dtype=torch.bool, device="cuda")
    kept[:, ::3] = True
    marks = kept.clone()
    cache.evict_weighted(order, [29 if s == 0 else 12 for s in order], w, resident_out=resident, kept=kept)
    assert cache.device_status() == (0, 1)
    for x, y in zip(before, all_of_it()):
        assert torch.equal(x, y)
    assert resident.tolist() == [-7, -7] and torch.equal(kept, marks)
    # The tags, through a call that takes one: what goes by the same weights where no page is wanted.
    # (Session 1 alone: 12 of its 30 stay, the newest, in the page that is there.)
    cache.evict_weighted([1], [12], w, resident_out=resident[:1], kept=kept[:1])
    torch.cuda.synchronize()
    assert int(resident[0]) == 12
    assert torch.equal(kept[0, :30].cpu(), torch.arange(30) >= 18)
    k, v = cache.read_kv([1], [0], [0, 12])
    assert torch.equal(k, before[0][:, 48:60]) and torch.equal(v, before[1][:, 48:60])
    assert [s["resident"] for s in states] == [30, 30]
