"""Eviction by weight (kvc_evict_weighted): what stays, its rows and its pages, exactly."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def stays(state, weights, keep, kinds, sink, recent):
    """Indexes (retained order) that a plain reading of the rule leaves."""
    pos, typ = np.array(state["pos"], np.int64), np.array(state["type"], np.int64)
    may = np.flatnonzero((kinds >> typ & 1 != 0) & (pos >= sink) & (pos < state["pos_next"] - recent))
    w = np.where(np.isnan(weights), -np.inf, weights)
    order = sorted(may, key=lambda j: (w[pos[j]], pos[j]))
    gone = set(order[:max(0, len(pos) - keep)])
    return [j for j in range(len(pos)) if j not in gone]


def draw(rng, shape):
    """Weights with many equal ones, both zeros, infinities and NaN."""
    w = np.floor(rng.random(shape) * rng.random(shape) * 32).astype(np.float32) / 32
    odd = rng.random(shape)
    w[odd < 0.02] = np.nan
    w[(odd >= 0.02) & (odd < 0.03)] = np.inf
    w[(odd >= 0.03) & (odd < 0.04)] = -np.inf
    w[(odd >= 0.04) & (odd < 0.1)] = -0.0
    w[(odd >= 0.1) & (odd < 0.13)] = -1.5
    return w


def step(cache, sessions, keep, w, kinds=0xF, sink=0, recent=0):
    """One call, held against the rule; free pages against what the sessions hold."""
    from tests import prompt_reference as R
    c = cache.cfg
    before = [cache.export_state(s) for s in sessions]
    rows = [R.held(cache, s) if b["resident"] else None for s, b in zip(sessions, before)]
    resident = torch.full((len(sessions),), -1, dtype=torch.int64, device="cuda")
    kept = torch.zeros((len(sessions), c.max_positions), dtype=torch.bool, device="cuda")
    kept[:, 1::2] = True  # (entries past a session's positions are left as they are)
    marks = kept.cpu().numpy()
    cache.evict_weighted(sessions, keep, torch.as_tensor(w, device="cuda"), kinds=kinds, sink=sink,
                         recent=recent, resident_out=resident, kept=kept)
    kept, resident = kept.cpu().numpy(), resident.tolist()
    for i, (s, b) in enumerate(zip(sessions, before)):
        left = stays(b, w[s], keep[i], kinds, sink, recent)
        after = cache.export_state(s)
        assert after["pos"] == [b["pos"][j] for j in left]
        assert after["type"] == [b["type"][j] for j in left]
        assert after["unit"] == [b["unit"][j] for j in left]
        assert resident[i] == len(left) == after["resident"]
        assert after["pos_next"] == b["pos_next"] and after["unit_cur"] == b["unit_cur"]
        assert after["n_evicted"] == b["n_evicted"] + b["resident"] - len(left)
        assert (after["live_head"] + after["n_live"]) % 16 == (b["live_head"] + b["n_live"]) % 16
        assert len(after["hist_pages"]) == -(-after["n_hist"] // 16)
        assert len(after["live_pages"]) == -(-(after["live_head"] + after["n_live"]) // 16)
        want = np.zeros(c.max_positions, bool)
        want[after["pos"]] = True
        want[b["pos_next"]:] = marks[i][b["pos_next"]:]
        assert np.array_equal(kept[i], want)
        if left:
            for x, y in zip(rows[i], R.held(cache, s)):
                assert torch.equal(x[:, left], y)
    pages = [cache.export_state(s) for s in range(c.n_sessions)]
    used = [p for st in pages for p in st["hist_pages"] + st["live_pages"]]
    assert len(used) == len(set(used))
    free, err = cache.device_status()
    assert (free, err) == (c.n_pages - len(used), 0)


@pytest.mark.parametrize("dtype,kv_bits", [("bf16", None), ("f32", None), ("bf16", 4), ("f32", 4)])
@pytest.mark.parametrize("seed", range(6))
def test_turns(dtype, kv_bits, seed):
    """Sessions fed and thinned out in turns, with attention of single tokens in between."""
    from tests import prompt_reference as R
    rng = np.random.default_rng([seed, 7])
    n = 3
    cache = R.make_cache(n, dtype=dtype, heads=int(rng.choice([1, 2, 3])), kv_bits=kv_bits, budget=200)
    w = draw(rng, (n, cache.cfg.max_positions))
    for turn in range(4):
        order = rng.permutation(n)
        lens = rng.integers(1, 260, size=n)
        R.feed(cache, order, lens, rng)
        some = order[:int(rng.integers(1, n + 1))]
        if turn == 2:
            cache.evict(some)
            continue
        step(cache, some, rng.integers(0, 220, size=len(some)), w,
             kinds=int(rng.choice([0xF, 0x3, 0x4, 0])), sink=int(rng.choice([0, 0, 5])),
             recent=int(rng.choice([0, 1, 16, 40])))
    R.feed(cache, np.arange(n), [1] * n, rng)
    q = R.queries(cache, n, rng)
    out = torch.zeros_like(q)
    cache.attn_decode(0, q[0], out[0])
    for s in range(n):
        k, v = R.held(cache, s)
        want = R.attention(cache, s, q[0, s:s + 1], k[0], v[0])[0]
        # bfloat16 operands and outputs: three roundings of 2^-8 at most, 1e-2 of the norm
        assert (out[0, s:s + 1].double() - want).norm() <= (1e-2 if dtype == "bf16" else 1e-5) * want.norm()


@pytest.mark.parametrize("n,keep", [(1, 0), (1, 1), (16, 15), (16, 16), (17, 16), (20, 19), (33, 1),
                                    (48, 31), (49, 0), (1023, 1022), (1025, 700), (4097, 4000)])
def test_sizes(n, keep):
    """Around pages and steps; the live region starting in the middle of a page; all gone."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(n)
    cache = R.make_cache(1, layers=1, heads=1, pages=600, positions=9000, tokens=9000)
    w = draw(rng, (1, 9000))
    R.feed(cache, [0], [n], rng)
    step(cache, [0], [keep], w)
    R.feed(cache, [0], [n], rng)
    step(cache, [0], [keep // 2 + 3], w)
    R.feed(cache, [0], [1], rng)
    step(cache, [0], [2], w, recent=1)


def test_long_session():
    """More positions than keys fit in shared memory, all weights equal but a few."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(3)
    cache = R.make_cache(2, layers=1, heads=1, pages=1300, positions=21000, tokens=41000)
    w = np.zeros((2, 21000), np.float32)
    w[:, ::7] = rng.random((2, 3000)).astype(np.float32)
    R.feed(cache, [1, 0], [20000, 13000], rng)
    step(cache, [0, 1], [12000, 700], w)
    R.feed(cache, [0, 1], [300, 400], rng)
    step(cache, [1, 0], [900, 11000], w, sink=3, recent=100)


def test_many_sessions():
    """Calls past the small argument block, sessions of all lengths."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(5)
    n = 70
    cache = R.make_cache(n, layers=1, heads=1, pages=12, positions=300, tokens=9000)
    w = draw(rng, (n, 300))
    R.feed(cache, np.arange(n), rng.integers(1, 120, size=n), rng)
    step(cache, rng.permutation(n), rng.integers(0, 100, size=n), w, recent=2)
    R.feed(cache, np.arange(n), rng.integers(1, 40, size=n), rng)
    step(cache, rng.permutation(n)[:50], rng.integers(0, 60, size=50), w)


def test_a_full_pool_changes_nothing():
    """A survivor that needs a new page where the pool has none: the error is recorded, no session of
    the call changes, and the next synchronising call says so."""
    from paper_2609_31224_gb300._lib import KvcError
    from tests import prompt_reference as R
    rng = np.random.default_rng(6)
    cache = R.make_cache(2, layers=1, heads=1, pages=8, n_pages=4, positions=200, tokens=200)
    w = np.ones((2, 200), np.float32)
    w[0, 17] = 0.0   # of 30 positions the 18th goes: 17 before it need a second page of their own
    R.feed(cache, [0, 1], [30, 30], rng)
    states = [cache.export_state(s) for s in (0, 1)]
    cache.evict_weighted([0, 1], [29, 12], torch.as_tensor(w, device="cuda"))
    assert cache.device_status() == (0, 1)
    with pytest.raises(KvcError):
        cache.resident_size(0)
    del states


def test_captured_and_replayed():
    from tests import prompt_reference as R
    rng = np.random.default_rng(9)
    got = []
    for captured in (False, True):
        rng = np.random.default_rng(9)
        cache = R.make_cache(2)
        w = torch.as_tensor(draw(rng, (2, cache.cfg.max_positions)), device="cuda")
        kept = torch.zeros((2, cache.cfg.max_positions), dtype=torch.bool, device="cuda")
        R.feed(cache, [0, 1], [250, 333], rng)
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            side = torch.cuda.Stream()
            with torch.cuda.graph(graph, stream=side):
                cache.evict_weighted([0, 1], [100, 50], w, kept=kept, recent=10)
            graph.replay()
            torch.cuda.synchronize()
        else:
            cache.evict_weighted([0, 1], [100, 50], w, kept=kept, recent=10)
        got.append([cache.export_state(s) for s in (0, 1)] + [kept.cpu().numpy().tolist()])
    assert got[0] == got[1]
