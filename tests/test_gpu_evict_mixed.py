"""kvc_evict on sessions that kvc_evict_weighted has thinned out: its rule holds over all that is resident,
whichever region of the cache holds it.  What stays, its rows and its pages, exactly."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HEADS = 2


def make(n, policy, *, dtype="bf16", kv_bits=None, budget=150, window=2, sink=5, recent=90, layers=2):
    from paper_2609_31224_gb300 import KVCache
    return KVCache(n_sessions=n, layers=layers, q_heads=4 * HEADS, kv_heads=HEADS,
                   head_dim=128 if dtype == "bf16" else 64, budget=budget, window=window, dtype=dtype,
                   n_pages=n * 80, max_pages_per_session=80, max_positions=2500, max_seq_per_call=n,
                   max_tokens_per_call=n * 400, rope_base=10000.0, kv_bits=kv_bits, policy=("unit", "position", "sink_recent")[policy],
                   sink=sink, recent=recent)


def rule_leaves(state, cfg):
    """Indexes (retained order) that a plain reading of the policy leaves."""
    pos, typ, unit = (np.array(state[x], np.int64) for x in ("pos", "type", "unit"))
    if cfg.policy == 2:
        return np.flatnonzero((pos < cfg.sink) | (pos >= state["pos_next"] - cfg.recent)).tolist()
    stays = np.ones(len(pos), bool)
    may = (typ <= 1) & (unit >= 0) & (unit <= state["unit_cur"] - cfg.window)
    while stays.sum() > cfg.budget >= 0 and (stays & may).any():
        oldest = np.flatnonzero(stays & may)[0]
        goes = stays & may & (unit == unit[oldest]) if cfg.policy == 0 else np.arange(len(pos)) == oldest
        stays &= ~goes
    return np.flatnonzero(stays).tolist()


def evict(cache, sessions, run=None):
    """One call, held against the rule; free pages against what the sessions hold."""
    from tests import prompt_reference as R
    c = cache.cfg
    before = [cache.export_state(s) for s in range(c.n_sessions)]
    rows = [R.held(cache, s) if before[s]["resident"] else None for s in range(c.n_sessions)]
    resident = torch.full((len(sessions),), -1, dtype=torch.int64, device="cuda")
    if run is None:
        cache.evict(sessions, resident)
    else:
        run()
    resident = resident.tolist()
    used = []
    for s in range(c.n_sessions):
        b, after = before[s], cache.export_state(s)
        left = rule_leaves(b, c) if s in sessions else list(range(b["resident"]))
        for x in ("pos", "type", "unit"):
            assert after[x] == [b[x][j] for j in left], (s, x)
        if s in sessions and run is None:
            assert resident[list(sessions).index(s)] == len(left)
        assert after["n_evicted"] == b["n_evicted"] + b["resident"] - len(left)
        assert (after["live_head"] + after["n_live"]) % 16 == (b["live_head"] + b["n_live"]) % 16
        if left:
            for x, y in zip(rows[s], R.held(cache, s)):
                assert torch.equal(x[:, left], y)
        used += after["hist_pages"] + after["live_pages"]
    assert len(used) == len(set(used))
    assert cache.device_status() == (c.n_pages - len(used), 0)


@pytest.mark.parametrize("policy", [0, 1, 2])
@pytest.mark.parametrize("dtype, kv_bits", [("bf16", None), ("f32", None), ("bf16", 4)])
@pytest.mark.parametrize("seed", range(4))
def test_turns(policy, dtype, kv_bits, seed):
    from tests import prompt_reference as R
    from tests.test_gpu_evict_weighted import draw, step
    rng = np.random.default_rng([seed, policy])
    n = 3
    cache = make(n, policy, dtype=dtype, kv_bits=kv_bits, budget=int(rng.integers(40, 200)),
                 window=int(rng.integers(0, 4)), recent=int(rng.integers(1, 150)))
    w = draw(rng, (n, cache.cfg.max_positions))
    for turn in range(5):
        order = rng.permutation(n)
        lens = rng.integers(1, 260, size=n)
        # (A few positions in front of the first unit, which no rule but the third one takes.)
        types = [np.concatenate([np.full(min(3, t) if turn == 0 else 0, 3, np.uint8),
                                 R.stream_types(int(t), rng)])[:t] for t in lens]
        R.feed(cache, order, lens, rng, types=types)
        some = order[:int(rng.integers(1, n + 1))]
        if turn != 1:
            step(cache, some, rng.integers(60, 300, size=len(some)), w, kinds=int(rng.choice([0xF, 0x3, 0x4])),
                 recent=int(rng.choice([0, 1, 40])))
        evict(cache, rng.permutation(n)[:int(rng.integers(1, n + 1))])
    # Released sessions start anew, by the old way or the new one.
    cache.release([0])
    R.feed(cache, [0], [200], rng)
    evict(cache, [0])
    evict(cache, [0, 1, 2])


@pytest.mark.parametrize("policy", [0, 1, 2])
def test_a_budget_is_met(policy):
    """What eviction by weight left of old units goes when the budget asks for it."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(policy)
    cache = make(1, policy, budget=60, recent=60, sink=0)
    w = np.zeros((1, 2500), np.float32)
    w[0, :300] = 1.0
    R.feed(cache, [0], [400], rng, types=[np.where(np.arange(400) % 10 == 0, 0x80, 0).astype(np.uint8)])
    cache.evict_weighted([0], [250], torch.as_tensor(w, device="cuda"))
    evict(cache, [0])
    assert cache.resident_size(0) <= 60


def test_captured_and_replayed():
    from tests import prompt_reference as R
    from tests.test_gpu_evict_weighted import draw
    rng = np.random.default_rng(2)
    cache = make(2, 0, budget=80)
    w = torch.as_tensor(draw(rng, (2, 2500)), device="cuda")
    R.feed(cache, [0, 1], [300, 350], rng)
    cache.evict_weighted([1], [250], w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        cache.evict([0, 1])
    evict(cache, [0, 1], run=graph.replay)
    R.feed(cache, [0, 1], [100, 50], rng)
    cache.evict_weighted([0], [120], w)          # one that was not thinned out at the capture
    evict(cache, [0, 1], run=graph.replay)


def test_many_sessions():
    from tests import prompt_reference as R
    from tests.test_gpu_evict_weighted import draw
    rng = np.random.default_rng(5)
    n = 50
    cache = make(n, 0, budget=70, layers=1)
    w = torch.as_tensor(draw(rng, (n, 2500)), device="cuda")
    R.feed(cache, range(n), rng.integers(1, 300, size=n), rng)
    cache.evict_weighted([3, 7, 44], [100, 30, 80], w)
    evict(cache, rng.permutation(n))
    R.feed(cache, range(n), rng.integers(1, 90, size=n), rng)
    evict(cache, rng.permutation(n)[:41])
