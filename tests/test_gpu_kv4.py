"""The cache held in 4 bits (KVC_KV4) against a plain reference in 64 bits: what is held bit for bit,
attention within the rounding of its operands, and the places where either can go wrong.

Attention tolerances.  The reference takes the very numbers that the codes stand for, so what is
left is the rounding of q, P and the output.  bfloat16 (8 significant bits): the output's rounding is
at most 2^-8 of each element, 2^-8 / sqrt(3) of the norm; q and P are rounded to 11 bits, which moves
a weight by about 2^-12 times its logit's scale (inputs N(0, 1): logits of N(0, 1)) and each term by
2^-12, at random: under 2^-11 of the row's root mean square in total, 4 standard deviations 2^-9 of
it.  binary32: q and P keep 22 bits (an error of 2^-23 each against values up to 1, logits up to
about 6), sums of up to 10^3 truncated products in binary32 lose up to 2^-24 of the running sum a
step over 64 pages of a warp: 2^-18 of the root mean square is the largest of it that can add up,
the norm stays under 2^-19.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import kv4_reference as R  # noqa: E402
from harness import Lockstep  # noqa: E402
from paper_2609_31224_gb300 import KVCache, KvcError  # noqa: E402
from synth import gpu as synth_gpu  # noqa: E402
from synth import script as S  # noqa: E402
from synth.driver import Driver  # noqa: E402

pytestmark = pytest.mark.gpu

DIM = {"bf16": 128, "f32": 64}
TD = {"bf16": torch.bfloat16, "f32": torch.float32}
ACOUSTIC, DELIM, TRANSCRIPT, TEXT, BEGIN = 0, 1, 2, 3, 0x80


def assert_attention(got, ref, dtype, what=""):
    got, ref = got.astype(np.float64), ref.astype(np.float64)
    assert np.isfinite(got).all(), what
    rms = np.sqrt(np.mean(ref ** 2, axis=-1, keepdims=True))
    each, unit = (2.0 ** -8, 2.0 ** -9) if dtype == "bf16" else (2.0 ** -23, 2.0 ** -18)
    norm = 2.0 ** -8 * 0.75 if dtype == "bf16" else 2.0 ** -19
    err = np.abs(got - ref)
    assert (err <= each * np.abs(ref) + unit * rms).all(), (what, (err / rms).max())
    assert np.linalg.norm(got - ref) <= norm * np.linalg.norm(ref), \
        (what, np.linalg.norm(got - ref) / np.linalg.norm(ref))


class Pair:
    """A cache held in 4 bits and the reference's copy of what it holds."""

    def __init__(self, dtype, heads, n, layers=2, budget=-1, window=1, n_pages=600, most=9000,
                 tokens=20000, seed=0, **kw):
        self.dtype, self.heads, self.layers, self.d = dtype, heads, layers, DIM[dtype]
        self.rng = np.random.default_rng(seed)
        self.cache = KVCache(n_sessions=n, layers=layers, q_heads=4 * heads, kv_heads=heads,
                             head_dim=self.d, budget=budget, window=window, dtype=dtype,
                             rope_base=R.BASE, n_pages=n_pages,
                             max_pages_per_session=most // 16 + 8, max_positions=2 * most,
                             max_seq_per_call=n, max_tokens_per_call=tokens, kv_bits=4, **kw)
        e = np.zeros((0, layers, heads, self.d), np.float32)
        self.k, self.v, self.pos = [e] * n, [e] * n, [np.zeros(0, int) for _ in range(n)]
        self.fed = [0] * n

    def normal(self, *shape):
        return R.in_type(self.rng.standard_normal(shape).astype(np.float32), self.dtype)

    def device(self, x):
        return torch.as_tensor(x).to("cuda", TD[self.dtype]).contiguous()

    def append(self, sessions, lens, types=None, kv=None, per_layer=False, hold=True):
        """kv: (k, v) [total, layers, heads, D] float32 in the element type.  hold=False with
        per_layer: positions only, the rows are the caller's to write."""
        cu = np.concatenate([[0], np.cumsum(lens)])
        total = int(cu[-1])
        types = np.full(total, TEXT, np.uint8) if types is None else np.asarray(types, np.uint8)
        k, v = kv if kv is not None else (self.normal(total, self.layers, self.heads, self.d),
                                          self.normal(total, self.layers, self.heads, self.d))
        dk, dv = (self.device(x.transpose(1, 0, 2, 3)) for x in (k, v))
        self.cache.append_chunk(sessions, cu, torch.as_tensor(types, device="cuda"),
                                None if per_layer else dk, None if per_layer else dv)
        if per_layer and hold:
            for layer in range(self.layers):
                self.cache.append_kv_layer(layer, dk[layer], dv[layer])
        for i, s in enumerate(sessions):
            pos = np.arange(self.fed[s], self.fed[s] + lens[i])
            a, b = cu[i], cu[i + 1]
            flat = k[a:b].reshape(lens[i], -1, self.d)
            hk = R.held(R.rotate32(flat, pos)).reshape(k[a:b].shape)
            self.k[s] = np.concatenate([self.k[s], hk])
            self.v[s] = np.concatenate([self.v[s], R.held(v[a:b])])
            self.pos[s] = np.concatenate([self.pos[s], pos])
            self.fed[s] += lens[i]
        return dk, dv

    def keep(self, s, kept):
        """An eviction left these positions."""
        at = np.searchsorted(self.pos[s], kept)
        assert (self.pos[s][at] == kept).all()
        self.k[s], self.v[s], self.pos[s] = self.k[s][at], self.v[s][at], self.pos[s][at]

    def read(self, sessions, first, lens, **kw):
        cu = np.concatenate([[0], np.cumsum(lens)])
        k, v = self.cache.read_kv(sessions, first, cu, **kw)
        return k.float().cpu().numpy(), v.float().cpu().numpy()

    def check_rows(self, sessions):
        """Every resident row of the sessions, bit for bit."""
        lens = [len(self.pos[s]) for s in sessions]
        k, v = self.read(sessions, [0] * len(sessions), lens)
        for got, mine in ((k, self.k), (v, self.v)):
            want = np.concatenate([mine[s] for s in sessions]).transpose(1, 0, 2, 3)
            np.testing.assert_array_equal(got, R.in_type(want, self.dtype))

    def queries(self, lens):
        return self.normal(sum(lens), self.layers, 4 * self.heads, self.d)

    def attend(self, sessions, lens, q, layer, kind, kv=None, stream=None):
        dq = self.device(q[:, layer])
        out = torch.full_like(dq, float("nan"))
        c = self.cache
        if kv is not None:
            fn = c.attn_decode_kv_raw if kind == "decode" else c.attn_prefill_kv_raw
            fn(layer, kv[0][layer].data_ptr(), kv[1][layer].data_ptr(), dq.data_ptr(),
               out.data_ptr(), torch.cuda.current_stream().cuda_stream)
        else:
            (c.attn_decode if kind == "decode" else c.attn_prefill_chunk)(layer, dq, out,
                                                                          stream=stream)
        return out

    def reference(self, sessions, lens, q, layer):
        outs, a = [], 0
        for s, t in zip(sessions, lens):
            n = len(self.pos[s])
            outs.append(R.attention(q[a:a + t, layer], self.pos[s][n - t:], self.k[s][:, layer],
                                    self.v[s][:, layer], np.arange(n - t + 1, n + 1)))
            a += t
        return np.concatenate(outs)

    def check_attention(self, sessions, lens, kind, kv=None, layers=None):
        q = self.queries(lens)
        for layer in range(self.layers) if layers is None else layers:
            out = self.attend(sessions, lens, q, layer, kind, kv)
            assert_attention(out.float().cpu().numpy(), self.reference(sessions, lens, q, layer),
                             self.dtype, f"{kind} layer {layer}")
        assert self.cache.device_status()[1] == 0


# -- what is held ------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [1, 3, 8])
@pytest.mark.parametrize("lens", [[1], [2, 15], [16, 1, 17], [33, 100, 7], [300, 1, 1, 5]])
@pytest.mark.parametrize("per_layer", [False, True])
def test_rows_are_held_as_defined(dtype, heads, lens, per_layer):
    p = Pair(dtype, heads, len(lens), layers=3)
    every = list(range(len(lens)))
    p.append(every, [3 + i for i in every], per_layer=per_layer)  # slots start inside a page
    p.append(every, lens, per_layer=per_layer)
    p.append(every, [1] * len(lens), per_layer=per_layer)
    p.check_rows(every)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_special_groups(dtype):
    """Zeros, values below and around the finest scale, ties, values beyond what is held, infinities
    and NaN: in their group only."""
    p = Pair(dtype, 2, 1, layers=1)
    n = 64
    k, v = p.normal(n, 1, 2, p.d), p.normal(n, 1, 2, p.d)
    with np.errstate(over="ignore"):
        mag = (10.0 ** p.rng.uniform(-8, 8, (n, 1, 2, 1))).astype(np.float32)
        k, v = R.in_type(k * mag, dtype), R.in_type(v * mag[::-1], dtype)
    v[0] = 0
    v[1, :, :, :32] = 0
    v[2] = np.float32(3.0 * 2.0 ** -20)
    v[3] = np.float32(3.5 * 2.0 ** -20)
    v[4] = np.tile(np.arange(-7, 8.5, 0.5, np.float32)[:31].tolist() + [7.0], p.d // 32)  # ties
    v[5, ..., 3], v[6, ..., 40], v[7, ..., 5] = np.inf, -np.inf, np.nan
    k[8, ..., 1], k[9, ..., p.d // 2] = np.nan, np.inf
    v[10] = 65408
    v[11] = -3e38
    p.append([0], [n], kv=(k, v))
    p.check_rows([0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read_back(dtype):
    """Any part of any session, in any order, any layers; zeros past the end; resident counts."""
    p = Pair(dtype, 2, 4, layers=3)
    p.append([0, 1, 2, 3], [40, 1, 17, 130])
    sess, first, lens = [3, 0, 2, 1], [100, 39, 5, 0], [50, 1, 0, 3]
    res = torch.zeros(4, dtype=torch.int64, device="cuda")
    k, v = p.read(sess, first, lens, layer0=1, n_layers=2, resident_out=res)
    assert res.tolist() == [130, 40, 17, 1]
    at = 0
    for s, f, n in zip(sess, first, lens):
        have = min(n, len(p.pos[s]) - f)
        for got, mine in ((k, p.k), (v, p.v)):
            want = R.in_type(mine[s][f:f + n, 1:].transpose(1, 0, 2, 3), dtype)
            np.testing.assert_array_equal(got[:, at:at + have], want)
            assert (got[:, at + have:at + n] == 0).all()
        at += n
    ek, ev = p.cache.export_kv(3, 2)                       # the host's own read-back
    k, v = p.read([3], [0], [130], layer0=2, n_layers=1)
    np.testing.assert_array_equal(ek, k[0])
    np.testing.assert_array_equal(ev, v[0])
    counts = torch.zeros(4, dtype=torch.int64, device="cuda")
    p.cache.read_kv(sess, [0] * 4, [0] * 5, resident_out=counts)
    assert counts.tolist() == [130, 40, 17, 1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read_back_of_a_cache_in_its_own_type(dtype):
    d = DIM[dtype]
    cache = KVCache(n_sessions=40, layers=2, q_heads=8, kv_heads=2, head_dim=d, budget=20, window=0,
                    dtype=dtype, n_pages=400, max_pages_per_session=20, max_positions=400,
                    max_seq_per_call=40, max_tokens_per_call=4000)
    every = list(range(40))
    lens = [1 + 3 * i % 50 for i in every]
    cu = np.concatenate([[0], np.cumsum(lens)])
    k = torch.randn(2, cu[-1], 2, d, device="cuda", dtype=TD[dtype])
    types = np.concatenate([[BEGIN] + [ACOUSTIC if j % 3 else TEXT for j in range(n - 1)]
                            for n in lens]).astype(np.uint8)
    cache.append_chunk(every, cu, torch.as_tensor(types, device="cuda"), k, k)
    cache.evict(every)
    kept = [cache.resident_size(s) for s in every]
    assert min(kept) < max(kept) and sum(kept) < cu[-1]
    rows = np.concatenate([[0], np.cumsum(kept)])
    rk, rv = cache.read_kv(every, [0] * 40, rows)
    for s in every:
        for layer in range(2):
            ek, ev = cache.export_kv(s, layer)
            np.testing.assert_array_equal(rk[layer, rows[s]:rows[s + 1]].float().cpu().numpy(), ek)
            np.testing.assert_array_equal(rv[layer, rows[s]:rows[s + 1]].float().cpu().numpy(), ev)


# -- attention ---------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [1, 3, 8])
@pytest.mark.parametrize("lens", [[0], [1], [14], [15], [16], [31, 0, 200], [5, 64, 1000, 17, 330]])
@pytest.mark.parametrize("fused", [False, True])
def test_decode(dtype, heads, lens, fused):
    p = Pair(dtype, heads, len(lens))
    every = list(range(len(lens)))
    if any(lens):
        p.append([s for s in every if lens[s]], [n for n in lens if n])
    kv = p.append(every, [1] * len(every), per_layer=fused, hold=not fused)
    p.check_attention(every, [1] * len(every), "decode", kv if fused else None)
    p.check_rows(every)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,chunk", [
    (2, [0], [1]), (2, [3], [2]), (2, [0, 7], [3, 1]), (1, [0], [17]), (2, [40], [17]),
    (8, [15, 0, 300], [17, 17, 17]), (3, [1, 130], [6, 12]), (2, [16, 31, 1000], [18, 1, 7]),
    (1, [5], [24]), (2, [12, 700], [25, 30]), (1, [0, 9], [32, 31]), (8, [200], [32])])
@pytest.mark.parametrize("fused", [False, True])
def test_prefill(dtype, heads, before, chunk, fused):
    p = Pair(dtype, heads, len(before))
    every = list(range(len(before)))
    if any(before):
        p.append([s for s in every if before[s]], [n for n in before if n])
    kv = p.append(every, chunk, per_layer=fused, hold=not fused)
    p.check_attention(every, chunk, "prefill", kv if fused else None)
    p.check_rows(every)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,length", [(1, 8000), (3, 4100), (40, 700), (150, 90)])
def test_many_pages_and_pairs(dtype, n, length):
    """Pairs cut over many CTAs, CTAs of many pairs."""
    p = Pair(dtype, 2, n, layers=1, n_pages=n * (length // 16 + 4), most=length + 100,
             tokens=n * length)
    every = list(range(n))
    lens = [length - 13 * (i % 5) for i in every]
    p.append(every, lens)
    p.append(every, [1] * n)
    p.check_attention(every, [1] * n, "decode")
    chunk = [17 if n < 100 else 5] * n
    p.append(every, chunk)
    p.check_attention(every, chunk, "prefill")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-3, 6.0])
def test_sharp_and_flat_softmax(dtype, scale):
    """Queries scaled: nearly uniform weights, and logits of standard deviation 6.  There an error of
    2^-12 (bfloat16) or 2^-22 (binary32) of a logit of up to 6 * 5 shows in the weight as 30 times
    that: 2^-7 and 2^-17 of the root mean square."""
    p = Pair(dtype, 2, 2)
    p.append([0, 1], [500, 77])
    p.append([0, 1], [1, 1])
    q = p.queries([1, 1]) * np.float32(scale)
    q = R.in_type(q, dtype)
    out = p.attend([0, 1], [1, 1], q, 1, "decode").float().cpu().numpy()
    ref = p.reference([0, 1], [1, 1], q, 1)
    rms = np.sqrt(np.mean(ref ** 2, axis=-1, keepdims=True))
    unit = 2.0 ** (-7 if dtype == "bf16" else -17)
    assert (np.abs(out - ref) <= 2.0 ** -8 * (dtype == "bf16") * np.abs(ref) + unit * rms).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_magnitudes(dtype):
    """Large and small keys, values and queries: weights stay what they are when k grows as q
    shrinks, outputs scale with v."""
    p = Pair(dtype, 1, 1, layers=3)
    n = 100
    k, v = p.normal(n, 3, 1, p.d), p.normal(n, 3, 1, p.d)
    power = np.array([0.0, 9.0, -9.0])[None, :, None, None]
    k = R.in_type(k * (2.0 ** power).astype(np.float32), dtype)
    v = R.in_type(v * (2.0 ** -power).astype(np.float32), dtype)
    p.append([0], [n - 1], kv=(k[:-1], v[:-1]))
    p.append([0], [1], kv=(k[-1:], v[-1:]))
    q = p.queries([1]) * (2.0 ** -power).astype(np.float32)
    for layer in range(3):
        out = p.attend([0], [1], q, layer, "decode")
        assert_attention(out.float().cpu().numpy(), p.reference([0], [1], q, layer), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_special_queries(dtype):
    """A zero query weighs every key alike; one of 2^-100 too; a large one picks its largest logit."""
    p = Pair(dtype, 2, 1, layers=1)
    p.append([0], [70])
    p.append([0], [5])
    q = p.queries([5])
    q[0], q[1] = 0, q[1] * np.float32(2.0 ** -100)
    q[2] *= np.float32(2.0 ** 40)
    out = p.attend([0], [5], q, 0, "prefill").float().cpu().numpy()
    ref = p.reference([0], [5], q, 0)
    assert_attention(out, ref, dtype)
    for i in (0, 1):
        flat = p.v[0][:71 + i, 0].mean(axis=0).repeat(4, axis=0)
        assert_attention(out[i:i + 1], flat[None], dtype)


# -- eviction, exports ---------------------------------------------------------------------------
def units(rng, n):
    out = []
    for _ in range(n):
        out += [ACOUSTIC | BEGIN] + [ACOUSTIC] * 16 + [DELIM] + [TRANSCRIPT] * int(rng.poisson(3))
        out += [DELIM]
    return np.array(out, np.uint8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_eviction_moves_rows_unchanged(dtype):
    p = Pair(dtype, 2, 3, layers=2, budget=90, window=2, n_pages=200, most=600)
    types = [units(p.rng, n) for n in (4, 9, 15)]
    every = [0, 1, 2]
    p.append(every, [len(t) for t in types], types=np.concatenate(types))
    for step in range(3):
        p.cache.evict(every)
        for s in every:
            p.keep(s, np.array(p.cache.export_state(s)["pos"]))
        p.check_rows(every)
        more = [units(p.rng, 2) for _ in every]
        p.append(every, [len(t) for t in more], types=np.concatenate(more))
        p.append(every, [1] * 3, types=[TRANSCRIPT] * 3)
        p.check_attention(every, [1] * 3, "decode")
        chunk = np.array([ACOUSTIC | BEGIN] + [ACOUSTIC] * 16, np.uint8)
        p.append(every, [17] * 3, types=np.tile(chunk, 3))
        p.check_attention(every, [17] * 3, "prefill")
    p.check_rows(every)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_transcript_export(dtype):
    p = Pair(dtype, 3, 2, layers=2, budget=60, window=1, n_pages=100, most=400)
    types = units(p.rng, 9)
    p.append([1], [len(types)], types=types)
    p.cache.evict([1])
    p.keep(1, np.array(p.cache.export_state(1)["pos"]))
    is_tr = (types & 0x7F)[p.pos[1]] == TRANSCRIPT
    pos, k, v, count = p.cache.export_transcript(1, 64)
    n = int(count)
    assert n == is_tr.sum() > 10
    assert pos[:n].tolist() == p.pos[1][is_tr].tolist()
    for got, mine in ((k, p.k[1]), (v, p.v[1])):
        np.testing.assert_array_equal(got[:, :n].float().cpu().numpy(),
                                      R.in_type(mine[is_tr].transpose(1, 0, 2, 3), dtype))


# -- masked places -------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_what_a_page_held_before_does_not_reach_a_row(dtype, bad):
    """Pages that a released session filled with NaN and infinities, reused for a few positions."""
    p = Pair(dtype, 2, 2, n_pages=40, most=400)
    x = np.full((400, 2, 2, p.d), bad, np.float32)
    p.append([0], [400], kv=(x, x))
    p.cache.release([0])
    p.append([1], [3])
    p.append([1], [1])
    p.check_attention([1], [1], "decode")
    p.append([1], [17])
    p.check_attention([1], [17], "prefill")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, -np.inf])
@pytest.mark.parametrize("before", [5, 12, 100])
def test_a_later_token_of_the_chunk_does_not_reach_an_earlier_one(dtype, bad, before):
    """A NaN in the V of token 9 reaches that group of the rows of tokens 9 and on, one in its K all
    of them; the tokens before it are as without it."""
    d = DIM[dtype]
    for where in ("v", "k"):
        p = Pair(dtype, 2, 1, layers=1)
        p.append([0], [before])
        k, v = p.normal(17, 1, 2, d), p.normal(17, 1, 2, d)
        (v if where == "v" else k)[9, 0, 1, 3] = bad     # KV head 1, first group of 32
        p.append([0], [17], kv=(k, v))
        q = p.queries([17])
        out = p.attend([0], [17], q, 0, "prefill").float().cpu().numpy()
        p.k[0], p.v[0] = np.nan_to_num(p.k[0]), np.nan_to_num(p.v[0])
        ref = p.reference([0], [17], q, 0)
        assert_attention(out[:9], ref[:9], dtype)
        assert_attention(out[9:, :4], ref[9:, :4], dtype)   # the other KV head
        seen = out[9:, 4:]
        if where == "v":
            assert np.isnan(seen[..., :32]).all()
            assert_attention(seen[..., 32:], ref[9:, 4:, 32:], dtype)
        else:
            assert np.isnan(seen).all()


# -- calls ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_results_repeat_and_streams_and_graphs_agree(dtype):
    p = Pair(dtype, 4, 3, layers=2)
    every = [0, 1, 2]
    p.append(every, [900, 40, 333])
    p.append(every, [1] * 3)
    q = p.queries([1] * 3)
    first = p.attend(every, [1] * 3, q, 1, "decode")
    again = p.attend(every, [1] * 3, q, 1, "decode")
    assert torch.equal(first, again)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = p.attend(every, [1] * 3, q, 1, "decode")
    side.synchronize()
    assert torch.equal(first, other)
    # Captured with few positions, replayed when there are more.
    dq = p.device(q[:, 1])
    out = torch.zeros_like(dq)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.attn_decode(1, dq, out)
    graph.replay()
    torch.cuda.synchronize()
    # (A captured launch is cut for the pages that sessions come to hold: its last bits may differ
    # from the eager one's, not from its own.)
    assert_attention(out.float().cpu().numpy(), p.reference(every, [1] * 3, q, 1), dtype)
    once = out.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(once, out)
    p.append(every, [2000, 5, 70])
    p.append(every, [1] * 3)
    graph.replay()
    torch.cuda.synchronize()
    assert_attention(out.float().cpu().numpy(), p.reference(every, [1] * 3, q, 1), dtype)


def test_rows_past_32_bit_offsets():
    """A pool of 5 GB whose last pages are used: the first session takes the pages before them."""
    heads, layers = 8, 32
    page = layers * heads * 2 * 1152
    n_pages = 5 * 2 ** 30 // page
    p = Pair("bf16", heads, 2, layers=layers, n_pages=n_pages, most=16 * n_pages, tokens=16 * n_pages)
    filler = 16 * (n_pages - 8)
    p.cache.append_chunk([0], [0, filler], torch.full((filler,), TEXT, dtype=torch.uint8,
                                                      device="cuda"), None, None)
    p.append([1], [50])
    p.append([1], [1])
    p.check_attention([1], [1], "decode", layers=[0, 31])
    p.append([1], [17])
    p.check_attention([1], [17], "prefill", layers=[0, 31])
    p.check_rows([1])


def test_refusals():
    p = Pair("bf16", 2, 3)
    c = p.cache
    p.append([0, 1], [4, 1])
    k = torch.zeros((2, 8, 2, 128), dtype=torch.bfloat16, device="cuda")

    def refused(fn, word):
        with pytest.raises((KvcError, ValueError), match=word):
            fn()

    refused(lambda: c.read_kv([0], [0], [0, 9], k=k, v=k), "shape")
    refused(lambda: c.read_kv([0], [0, 1], [0, 8]), "entry")
    refused(lambda: c.read_kv([3], [0], [0, 8]), "out of range")
    refused(lambda: c.read_kv([0, 0], [0, 0], [0, 4, 8]), "repeated")
    refused(lambda: c.read_kv([0], [-1], [0, 8]), "negative")
    refused(lambda: c.read_kv([0], [0], [1, 8]), "must be 0")
    refused(lambda: c.read_kv([0, 1], [0, 0], [0, 8, 4]), "decreases")
    refused(lambda: c.read_kv([0], [0], [0, 8], layer0=2), "layers")
    refused(lambda: c.read_kv([0], [0], [0, 8], layer0=-1, n_layers=1), "layers")
    refused(lambda: c.read_kv([0], [0], [0, 8], layer0=1, n_layers=2 ** 31 - 1), "outside|shape|memory")
    s = np.zeros(1, np.int32)
    cu = np.array([0, 8], np.int32)
    from paper_2609_31224_gb300._lib import host_i32
    (_, sp), (_, cp) = host_i32(s), host_i32(cu)
    refused(lambda: c.read_kv_raw(1, sp, sp, cp, 0, 1, k.data_ptr() + 2, k.data_ptr(), None, 0), "aligned")
    refused(lambda: c.read_kv_raw(1, sp, sp, cp, 0, 1, None, k.data_ptr(), None, 0), "NULL")
    refused(lambda: c.read_kv_raw(1, sp, None, cp, 0, 1, k.data_ptr(), k.data_ptr(), None, 0), "NULL")
    q = torch.zeros((5, 8, 128), dtype=torch.bfloat16, device="cuda")
    refused(lambda: c.attn_decode(0, q, q), "one appended token")
    p.append([0, 1], [1, 1])
    assert c.lib.kvc_attn_decode_noalloc(c.ctx, 0, q.data_ptr(), q.data_ptr(), None) == -1
    assert b"KVC_KV4" in c.lib.kvc_last_error()
    p.append([0], [33])
    q = torch.zeros((33, 8, 128), dtype=torch.bfloat16, device="cuda")
    refused(lambda: c.attn_prefill_chunk(0, q, q), "32 tokens")
    p.check_rows([0, 1])                      # nothing of it changed the cache


@pytest.mark.parametrize("exp", [-14, -3, 0, 6])
def test_numbers_next_to_half_a_step(exp):
    """Every scale of an octave, its half steps and their neighbours on both sides: codes are those of
    the rounded quotient, ties to even."""
    half, f = [], np.float32
    for m in range(64, 128):
        s = f(m) * f(2.0 ** (exp - 6))
        at = [(2 * j + 1) * s / f(2) for j in range(7)]
        near = [np.nextafter(x, f(y)) for x in at for y in (0, np.inf)]
        half.append([7 * s] + at + near + [-x for x in at + near][:10])
    half = np.array(half, f)                                 # [64 scales, 32]
    p = Pair("f32", 2, 1, layers=1)
    rows = half.reshape(16, 1, 2, 64)
    assert (np.abs(rows).reshape(-1, 32).max(-1) == half[:, 0]).all()
    p.append([0], [16], kv=(p.normal(16, 1, 2, 64), rows))
    p.check_rows([0])


class Held(Lockstep):
    """A workload run on a cache held in 4 bits beside the oracle: states as always, outputs against
    attention over the numbers that the retained rows are held as."""

    def held(self, s, layer, pos):
        k, v = (x.astype(np.float32) for x in self.kv_source(s, layer, pos))
        return R.held(R.rotate32(k, pos)), R.held(v)

    def compare_call(self, c, layer, sessions=None, what=""):
        out = c.out.float().cpu().numpy()
        for i, s in enumerate(c.sessions.tolist()):
            pos, mine = np.array(self.orc.state(s)["pos"]), np.array(c.positions[i])
            k, v = self.held(s, layer, pos)
            ref = R.attention(self.q_raw(s, layer, mine).astype(np.float32), mine, k, v,
                              np.arange(len(pos) - len(mine) + 1, len(pos) + 1))
            assert_attention(out[c.cu[i]:c.cu[i + 1]], ref, self.w.dtype, f"{what} {c.kind}")
            self.n_compared += 1


@pytest.mark.parametrize("policy", ["unit", "position", "sink_recent"])
@pytest.mark.parametrize("per_layer", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_workload_over_rows_in_4_bits(dtype, per_layer, policy):
    """Appends, prefill, decode, evictions and the read-back of what is left, as a user runs them."""
    base = S.SINGLE_BF16 if dtype == "bf16" else S.TINY_F32
    w = base.with_(layers=2, q_heads=8, kv_heads=2, n_sessions=3, units=24, budget=200, window=2,
                   offset_max=4, policy=policy, sink=5 if policy == "sink_recent" else 0,
                   recent=120 if policy == "sink_recent" else 0, seed=11)
    synth_gpu.build()
    drv = Driver(w, S.workload_scripts(w), kv_bits=4)
    ls = Held(drv, w)
    for _ in range(len(drv.sched)):
        ls.run_step(attn_pred=lambda step, kind, call, layer: (step + layer) % 3 == 0,
                    per_layer=per_layer)
    assert ls.n_compared > 40
    for s in range(3):
        st = ls.orc.state(s)
        assert st["n_evicted"] > 0
        pos = np.array(st["pos"])
        k, v = drv.cache.read_kv([s], [0], [0, len(pos)])
        for layer in range(2):
            for got, want in zip((k, v), ls.held(s, layer, pos)):
                np.testing.assert_array_equal(got[layer].float().cpu().numpy(),
                                              R.in_type(want, dtype))
    assert drv.cache.device_status()[1] == 0


def test_pages_past_four_gib():
    """A session whose pages lie past 2^32 bytes of the pool: write, read-back, decode, prefill."""
    before = 7400                                   # pages, of 589,824 bytes each
    p = Pair("bf16", 8, 2, layers=32, n_pages=before + 60, most=120000, tokens=before * 16)
    n = before * 16
    p.cache.append_chunk([0], [0, n], torch.full((n,), TEXT, dtype=torch.uint8, device="cuda"),
                         None, None)
    p.append([1], [45])
    p.append([1], [1])
    p.check_attention([1], [1], "decode", layers=[0, 31])
    p.append([1], [17])
    p.check_attention([1], [17], "prefill", layers=[0, 31])
    p.check_rows([1])
    kv = p.append([1], [19], per_layer=True, hold=False)
    q = p.queries([19])
    for layer in range(32):
        out = p.attend([1], [19], q, layer, "prefill", kv)
        if layer % 31 == 0:
            assert_attention(out.float().cpu().numpy(), p.reference([1], [19], q, layer), "bf16")
    p.check_rows([1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("turn", ["layers first", "one by one", "mixed"])
def test_orders_of_writes_and_attention(dtype, turn):
    """Chunks whose rows are written layer by layer, in several orders with the attention over them, call
    after call: old pages may be read before the write is complete, new ones may not."""
    p = Pair(dtype, 3, 5, layers=4, n_pages=2000)
    s = [0, 1, 2, 3, 4]
    p.append(s, [300, 1, 33, 700, 16])
    for lens in ([17, 1, 2, 32, 16], [5, 31, 17, 3, 1], [32, 32, 32, 32, 32]):
        kv = p.append(s, lens, per_layer=True, hold=False)
        q = p.queries(lens)
        outs = {}
        write = lambda l: p.cache.append_kv_layer(l, kv[0][l], kv[1][l])
        read = lambda l: outs.__setitem__(l, p.attend(s, lens, q, l, "prefill"))
        if turn == "layers first":
            for l in range(4):
                write(l)
            for l in range(4):
                read(l)
        elif turn == "one by one":
            for l in range(4):
                outs[l] = p.attend(s, lens, q, l, "prefill", kv)
        else:
            write(2)
            read(2)
            outs[0] = p.attend(s, lens, q, 0, "prefill", kv)
            read(2)
            write(3)
            read(0)
            read(3)
            outs[1] = p.attend(s, lens, q, 1, "prefill", kv)
        for l, out in outs.items():
            assert_attention(out.float().cpu().numpy(), p.reference(s, lens, q, l), dtype, f"{turn} {l}")
    p.check_rows(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_replayed_append_that_fails_changes_nothing(dtype):
    """A graph of a decode step, replayed past the pool's last page: the error is recorded, and the step
    that found no page leaves rows, outputs and counts as they were."""
    p = Pair(dtype, 2, 2, layers=2, n_pages=10)
    p.append([0, 1], [30, 15])
    d = p.d
    k, v = (torch.empty(2, 2, 2, d, dtype=TD[dtype], device="cuda") for _ in range(2))  # [layer][session]
    q, out = p.device(p.normal(2, 8, d)), torch.zeros(2, 2, 8, d, dtype=TD[dtype], device="cuda")
    types = torch.full((2,), TEXT, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def rows(n):
        got = p.cache.read_kv([0, 1], [0, 0], [0, n, 2 * n])
        return [x.clone() for x in got]

    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            p.cache.append_chunk([0, 1], [0, 1, 2], types, None, None, stream=stream)
            for layer in range(2):
                p.cache.attn_decode_kv_raw(layer, k[layer].data_ptr(), v[layer].data_ptr(),
                                           q.data_ptr(), out[layer].data_ptr(), stream.cuda_stream)
        for step in range(200):
            before = rows(200)
            k.fill_(step + 1)
            v.fill_(-step - 1)
            out.fill_(7.0)
            graph.replay()
            stream.synchronize()
            if p.cache.device_status()[1] != 0:
                break
            assert (out != 7.0).any()
    # After 50 steps 80 and 65 positions take five pages each; the next needs an eleventh.
    assert step == 50, step
    for a, b in zip(before, rows(200)):
        assert torch.equal(a, b)
    assert (out == 7.0).all()
