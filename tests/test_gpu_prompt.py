"""Attention over chunks of any length (kvc_attn_prompt) against 64 bits.

Tolerances.  binary32: as for the weights (1e-5 of the norm), sums of p v no more.  bfloat16: q, P and
the output are rounded once each, by 2^-8 at most and 2^-8 / sqrt(3) = 2.3e-3 of their binade in the
mean, 1.7e-3 of a value; a score moves with its row's q by as much of its size (about 1), so that the
norm of an output row is off by about sqrt(3) * 1.7e-3 = 2.9e-3 and held to 6e-3, a single value to
2^-6 of the row's largest."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check(cache, sessions, lens, rng, q=None, layers=None):
    from tests import prompt_reference as R
    total = int(np.sum(lens))
    q = R.queries(cache, total, rng) if q is None else q
    guard = 3  # rows behind the last session, left as they were
    out = torch.full((cache.cfg.layers, total + guard, *q.shape[2:]), 7.0, dtype=q.dtype, device="cuda")
    for layer in range(cache.cfg.layers):
        cache.attn_prompt(layer, q[layer], out[layer])
    assert cache.device_status()[1] == 0
    assert bool((out[:, total:] == 7.0).all())
    at = 0
    for s, t in zip(sessions, lens):
        k, v = R.held(cache, s)
        for layer in range(cache.cfg.layers):
            want = R.attention(cache, s, q[layer, at:at + t], k[layer], v[layer])[0]
            got = out[layer, at:at + t].double()
            fine = torch.isfinite(want)
            assert torch.equal(fine, torch.isfinite(got)), (s, layer)
            assert torch.equal(torch.isnan(want), torch.isnan(got))
            d, w = torch.where(fine, got - want, 0.0), torch.where(fine, want, 0.0)
            rel, top = (6e-3, 2.0 ** -6) if q.dtype == torch.bfloat16 else (1e-5, 1e-4)
            assert d.norm() <= rel * w.norm(), (s, layer, float(d.norm() / w.norm()))
            big = w.abs().amax(dim=-1, keepdim=True)
            assert bool((d.abs() <= top * big).all()), (s, layer, float((d.abs() / big).max()))
        at += t
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [1, 3])
@pytest.mark.parametrize("lens", [[33], [64], [65], [128], [129], [257], [1000], [1, 200, 17, 63],
                                  [600, 2, 31, 97, 1]])
def test_prompts_without_history(dtype, heads, lens):
    from tests import prompt_reference as R
    rng = np.random.default_rng([heads, lens[0], len(lens)])
    cache = R.make_cache(len(lens), dtype=dtype, heads=heads, pages=80)
    R.feed(cache, range(len(lens)), lens, rng)
    check(cache, range(len(lens)), lens, rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[40, 1], [33, 300], [200, 130], [1, 1], [5, 20]])
@pytest.mark.parametrize("before", [[1, 15], [97, 16], [700, 333], [1500, 4]])
def test_prompts_behind_evicted_histories(dtype, lens, before):
    from tests import prompt_reference as R
    rng = np.random.default_rng([lens[0], before[0]])
    cache = R.make_cache(3, dtype=dtype, budget=90, window=2, pages=150)
    R.feed(cache, [0, 1, 2], before + [50], rng)
    cache.evict([0, 1, 2])
    R.feed(cache, [0, 1], [7, 3], rng)
    R.feed(cache, [1, 0], lens, rng)                 # another order than the ids
    check(cache, [1, 0], lens, rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [1, 4])
@pytest.mark.parametrize("lens, before, evicts", [
    ([33], [5000], False), ([64], [4097], True), ([65], [1531], True), ([100, 40], [3000, 17], True),
    ([40, 33, 70], [900, 2600, 16], False), ([300], [2047], True), ([130, 1], [1, 4000], True)])
def test_short_chunks_behind_long_histories(dtype, heads, lens, before, evicts):
    """Too few rows for all SMs: an item's keys are cut into parts, some of them empty."""
    from tests import prompt_reference as R
    rng = np.random.default_rng([heads, lens[0], before[0]])
    n = len(lens)
    cache = R.make_cache(n, dtype=dtype, heads=heads, budget=max(before) - 300 if evicts else -1, pages=360,
                         positions=8192, tokens=8192)
    R.feed(cache, range(n), before, rng)
    if evicts:
        cache.evict(list(range(n)))
        R.feed(cache, range(n), [9] * n, rng)
        cache.evict(list(range(n)))
    R.feed(cache, range(n), lens, rng)
    a = check(cache, range(n), lens, rng, q=(q := R.queries(cache, sum(lens), rng)))
    assert torch.equal(a, check(cache, range(n), lens, rng, q=q))    # bit for bit


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_behind_a_token_in_parts(dtype):
    """V that is not finite in a chunk's own keys reaches the tokens at and behind it alone."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(5)
    cache = R.make_cache(1, dtype=dtype, heads=2, pages=360, positions=8192)
    R.feed(cache, [0], [4000], rng)
    k, v = R.rows(cache, 70, rng), R.rows(cache, 70, rng)
    v[:, 37] = torch.nan
    v[:, 69] = torch.inf
    cache.append_chunk([0], [0, 70], torch.zeros(70, dtype=torch.uint8, device="cuda"), k, v)
    check(cache, [0], [70], rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart_in_parts(dtype):
    """Parts whose scores differ by so much that all but one of them weigh nothing, and the other way round."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(9)
    cache = R.make_cache(1, dtype=dtype, layers=1, heads=1, pages=200, positions=4096)
    t = 3000
    k, v = R.rows(cache, t, rng), R.rows(cache, t, rng)
    size = torch.ones(t, device="cuda")
    size[:900], size[2000:2600] = 0.0, 20.0
    k = (k.float() * size[None, :, None, None]).to(k.dtype)
    cache.append_chunk([0], [0, t], torch.zeros(t, dtype=torch.uint8, device="cuda"), k, v)
    R.feed(cache, [0], [50], rng)
    q = R.queries(cache, 50, rng)
    if dtype == "bf16":
        q = (q.float() / 10).to(q.dtype)
    out = torch.zeros_like(q)
    cache.attn_prompt(0, q[0], out[0])
    hk, hv = R.held(cache, 0)
    want = R.attention(cache, 0, q[0], hk[0], hv[0])[0]
    d = (out[0].double() - want).norm() / want.norm()
    # scores of size up to 2 * 5 (bfloat16) or 20 * 5 (binary32): errors grow with them
    assert d < (10 * 3e-3 if dtype == "bf16" else 100 * 1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sessions_of_long_chunks(dtype):
    from tests import prompt_reference as R
    rng = np.random.default_rng(4)
    n = 130
    cache = R.make_cache(n, dtype=dtype, layers=1, heads=1, pages=16, tokens=16384)
    lens = [int(x) for x in rng.integers(1, 80, size=n)]
    R.feed(cache, range(n), [int(x) for x in rng.integers(1, 100, size=n)], rng)
    order = [int(x) for x in rng.permutation(n)]
    R.feed(cache, order, lens, rng)
    check(cache, order, lens, rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_items_a_cta(dtype):
    """Items of one and two tiles and of one to three steps behind one another, time and again: the same bits."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(14)
    n = 200
    cache = R.make_cache(n, dtype=dtype, layers=1, heads=8, pages=24, tokens=32768)
    lens = [int(x) for x in rng.integers(1, 150, size=n)]
    R.feed(cache, range(n), [int(x) for x in rng.integers(1, 200, size=n)], rng)
    R.feed(cache, range(n), lens, rng)
    q = R.queries(cache, sum(lens), rng)
    want = check(cache, range(n), lens, rng, q=q)[0, :sum(lens)]
    out = torch.zeros_like(q[0])
    work, w = cache.make_weights_workspace(), [cache.make_weights() for _ in range(2)]
    for _ in range(30):
        out.zero_()
        cache.attn_prompt(0, q[0], out)
        assert torch.equal(out, want)
        for x in w:
            x.zero_()
            cache.attn_weights(0, q[0], x, work)
        assert torch.equal(w[0], w[1])
    assert cache.device_status()[1] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_of_one_session_among_many(dtype):
    from tests import prompt_reference as R
    rng = np.random.default_rng(2)
    n = 40
    cache = R.make_cache(n, dtype=dtype, layers=1, heads=1, pages=40, tokens=2000)
    lens = [1] * n
    lens[17] = 555
    R.feed(cache, range(n), [int(x) for x in rng.integers(1, 40, size=n)], rng)
    R.feed(cache, range(n), lens, rng)
    check(cache, range(n), lens, rng)


def test_a_long_prompt():
    from tests import prompt_reference as R
    rng = np.random.default_rng(4)
    cache = R.make_cache(1, layers=1, heads=2, pages=400, positions=6000, tokens=6000)
    R.feed(cache, [0], [517], rng)
    R.feed(cache, [0], [4500], rng)
    check(cache, [0], [4500], rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [30.0, 1e-3])
def test_scores_far_apart(dtype, size):
    """Rows whose maximum moves late and by much, and nearly uniform rows."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(6)
    cache = R.make_cache(1, dtype=dtype, layers=1, heads=1, pages=60)
    t = 500
    k, v = R.rows(cache, t, rng), R.rows(cache, t, rng)
    ramp = torch.linspace(0.0, 1.0, t, device="cuda", dtype=torch.float32)[None, :, None, None]
    k = (k.float() * ramp).to(k.dtype)
    cache.append_chunk([0], [0, t], torch.zeros(t, dtype=torch.uint8, device="cuda"), k, v)
    q = R.queries(cache, t, rng)
    q = (q.float() * size).to(q.dtype)
    if dtype == "bf16" and size > 1:  # (roundings of q would move larger scores by whole numbers)
        q = (q.float() / 15).to(q.dtype)
    out = torch.zeros_like(q)
    cache.attn_prompt(0, q[0], out[0])
    hk, hv = R.held(cache, 0)
    want = R.attention(cache, 0, q[0], hk[0], hv[0])[0]
    d = (out[0].double() - want).norm() / want.norm()
    # scores of size up to 2 * 8 (bfloat16) or 30 * 8 (binary32): errors grow with them
    assert d < (16 * 3e-3 if dtype == "bf16" else 240 * 1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [50, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_token_does_not_see_does_not_reach_it(dtype, t, bad):
    """Values that are not finite: in freed pages that are used again nobody sees them; in the chunk
    the tokens before them do not."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(t)
    cache = R.make_cache(2, dtype=dtype, pages=40, n_pages=41, layers=1)
    n = 600
    types = torch.zeros(n, dtype=torch.uint8, device="cuda")
    odd = torch.full((1, n, 2, cache.cfg.head_dim), bad, dtype=cache.torch_dtype, device="cuda")
    cache.append_chunk([1], [0, n], types, odd, odd)
    cache.release([1])
    R.feed(cache, [0], [21], rng)
    k, v = R.rows(cache, t, rng), R.rows(cache, t, rng)
    for at in (t // 3, t - 2):
        v[0, at, 0, 5] = bad
        v[0, at, 1] = bad
    cache.append_chunk([0], [0, t], types[:t], k, v)
    out = check(cache, [0], [t], rng)
    assert bool(torch.isfinite(out[0, :t // 3].float()).all())
    # and keys: rows that see one are NaN, the others as if it were not there
    cache.release([0])
    k[0, t - 2] = float("nan")
    cache.append_chunk([0], [0, t], types[:t], k, R.rows(cache, t, rng))
    q = R.queries(cache, t, rng)
    cache.attn_prompt(0, q[0], out[0])
    hk, hv = R.held(cache, 0)
    want = R.attention(cache, 0, q[0], hk[0], hv[0])[0][:t - 2]
    got = out[0, :t - 2].double()
    assert bool(torch.isfinite(got).all())
    assert (got - want).norm() <= (6e-3 if dtype == "bf16" else 1e-5) * want.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_another_stream_and_a_graph(dtype):
    """On a stream of its own, captured and replayed: the same bits each time."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(12)
    lens = [150, 70]
    cache = R.make_cache(2, dtype=dtype)
    R.feed(cache, [0, 1], [100, 10], rng)
    R.feed(cache, [0, 1], lens, rng)
    q = R.queries(cache, 220, rng)
    outs = [torch.zeros_like(q) for _ in range(3)]
    cache.attn_prompt(0, q[0], outs[0][0])
    cache.attn_prompt(1, q[1], outs[0][1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for layer in (1, 0):
        cache.attn_prompt(layer, q[layer], outs[1][layer], stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for layer in range(2):
            cache.attn_prompt(layer, q[layer], outs[2][layer])
    graph.replay()
    outs[2].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_is_read_weighed_thinned_out_and_answered(dtype):
    """A run of the calls as a program makes them: prompt, attention, weights, eviction by them, then
    tokens one by one, whose weights are added, and another eviction."""
    from tests import prompt_reference as R
    rng = np.random.default_rng(20)
    lens = [400, 260]
    cache = R.make_cache(2, dtype=dtype)
    w, work = cache.make_weights(), cache.make_weights_workspace()
    c = cache.cfg
    types = [R.stream_types(t, rng) for t in lens]
    cache.append_chunk([0, 1], [0, 400, 660], torch.as_tensor(np.concatenate(types), device="cuda"),
                       None, None)
    q = R.queries(cache, 660, rng)
    k, v = R.rows(cache, 660, rng), R.rows(cache, 660, rng)
    out = torch.zeros_like(q)
    for layer in range(c.layers):  # a model's order: a layer's rows, then its attention
        cache.append_kv_layer(layer, k[layer], v[layer])
        cache.attn_prompt(layer, q[layer], out[layer])
        cache.attn_weights(layer, q[layer], w, work)
    want = torch.zeros((2, c.max_positions), dtype=torch.float64, device="cuda")
    for s, a, b in ((0, 0, 400), (1, 400, 660)):
        hk, hv = R.held(cache, s)
        for layer in range(c.layers):
            o, x = R.attention(cache, s, q[layer, a:b], hk[layer], hv[layer])
            assert (out[layer, a:b].double() - o).norm() <= (6e-3 if dtype == "bf16" else 1e-5) * o.norm()
            want[s, :b - a] += x
    assert torch.allclose(w.double(), want, rtol=6e-5, atol=1e-12)
    resident = torch.zeros(2, dtype=torch.int64, device="cuda")
    cache.evict_weighted([0, 1], [120, 130], w, sink=4, recent=32, resident_out=resident)
    assert resident.tolist() == [120, 130]
    for _ in range(3):
        R.feed(cache, [0, 1], [1, 1], rng)
        q1 = R.queries(cache, 2, rng)
        o1 = torch.zeros_like(q1)
        before = w.clone()
        for layer in range(c.layers):
            cache.attn_prompt(layer, q1[layer], o1[layer])
            cache.attn_weights(layer, q1[layer], w, work)
        for s in (0, 1):
            hk, hv = R.held(cache, s)
            pos = torch.as_tensor(cache.export_state(s)["pos"], device="cuda")
            add = torch.zeros(len(pos), dtype=torch.float64, device="cuda")
            for layer in range(c.layers):
                o, x = R.attention(cache, s, q1[layer, s:s + 1], hk[layer], hv[layer])
                assert (o1[layer, s:s + 1].double() - o).norm() <= (1e-2 if dtype == "bf16" else 1e-5) * o.norm()
                add += x
            assert torch.allclose(w[s, pos].double(), before[s, pos].double() + add, rtol=6e-5, atol=1e-12)
        cache.append_chunk([0], [0, 1], torch.zeros(1, dtype=torch.uint8, device="cuda"),
                           R.rows(cache, 1, rng), R.rows(cache, 1, rng))
    cache.evict_weighted([0, 1], [50, 60], w, recent=8, resident_out=resident)
    assert resident.tolist() == [50, 60] and cache.device_status()[1] == 0
