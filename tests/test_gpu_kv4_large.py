"""The cache held in 4 bits in large calls and under rising logits: decode cut evenly over the SMs
(stream-K: several pairs a CTA, parts of one pair in many), chunks in whole waves and a rest in slices,
and softmax references that move in later stages, for some rows of a chunk only.

Tolerances.  assert_attention is that of logits of N(0, 1).  Where they are larger, of standard
deviation 6 or rising to 20, bfloat16 calls err in a logit by about 6 * 2^-11 * 0.42 (q rounded to
11 bits at random, 0.42 of the bound each): 1.2e-3, 5.5e-3 at 4.5 standard deviations.  Two keys that
share a row give the largest change, 1.2e-3 * 4.5 * (|v1 - v2| = 5) / sqrt(8) = 9.5e-3 against an
output of 0.7: 2^-6 of the row's root mean square beside the output's own rounding of 2^-8.  binary32
calls hold q in 22 bits and sum products to 2^-22 of logits up to 40: 2^-16, allowed twice that.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import kv4_reference as R  # noqa: E402
from kv4_cuts import decode_cut  # noqa: E402
from test_gpu_kv4 import Pair, assert_attention  # noqa: E402

pytestmark = pytest.mark.gpu


def assert_sharp(got, ref, dtype, what=""):
    got = got.astype(np.float64)
    assert np.isfinite(got).all(), what
    rms = np.sqrt(np.mean(ref ** 2, axis=-1, keepdims=True))
    unit, each = (2.0 ** -6, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -15, 2.0 ** -23)
    err = np.abs(got - ref)
    assert (err <= each * np.abs(ref) + unit * rms).all(), (what, (err / rms).max())


def sampled(p, sessions, lens, q, layer, out, some, check, what):
    """check() on the rows of some of the sessions."""
    cuts = np.concatenate([[0], np.cumsum(lens)])
    got = out.float().cpu().numpy()
    for i in some:
        a, b = cuts[i], cuts[i + 1]
        ref = p.reference(sessions[i:i + 1], lens[i:i + 1], q[a:b], layer)
        check(got[a:b], ref, p.dtype, f"{what}, session {i}")


def rows_of(p, sessions):
    p.check_rows(sessions)
    assert p.cache.device_status()[1] == 0


def launches(p, fn):
    before = p.cache.launches()
    got = fn()
    return got, p.cache.launches() - before


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_calls(dtype, tmp_path):
    """40 sessions of 8 heads, 700 to 2,260 positions: decode takes stream-K, the bfloat16 prefill two
    launches, the second of which starts at a later pair."""
    n = 40
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    p = Pair(dtype, 8, n, layers=2, n_pages=n * 150, most=2400, tokens=n * 2300)
    every, some = list(range(n)), [0, 1, 7, 19, 20, 38, 39]
    p.append(every, [700 + 40 * (7 * i % n) for i in every])
    ones = [1] * n
    # One token each: rows with the append, then written by the launches.
    for fused in (False, True):
        kv = p.append(every, ones, per_layer=fused, hold=not fused)
        q = p.queries(ones)
        pages = 8 * sum(len(p.pos[i]) // 16 + 1 for i in every)
        assert decode_cut(tmp_path, sms, 8 * n, pages, 2 if dtype == "bf16" else 4) == (False, 0)
        for layer in range(2):
            out = p.attend(every, ones, q, layer, "decode", kv if fused else None)
            sampled(p, every, ones, q, layer, out, some, assert_attention, f"decode, fused {fused}")
    rows_of(p, every)
    # Chunks: right behind an append with rows, then in a model's order.
    for fused in (False, True):
        lens = [17 - 5 * (i % 3) * fused for i in every]
        kv = p.append(every, lens, per_layer=fused, hold=not fused)
        q = p.queries(lens)
        for layer in range(2):
            out, made = launches(p, lambda: p.attend(every, lens, q, layer, "prefill",
                                                     kv if fused else None))
            assert made == (2 if dtype == "bf16" else 1) + fused
            sampled(p, every, lens, q, layer, out, some, assert_attention, f"chunk, fused {fused}")
    rows_of(p, every)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,length", [(1, 3000), (50, 1500)])   # pairs in slices, pairs whole
def test_sharp_softmax_of_chunks(dtype, n, length):
    """Logits of standard deviation 6 over many stages: the reference moves where a key stands out."""
    p = Pair(dtype, 2, n, layers=1, n_pages=n * (length // 16 + 8), most=length + 100,
             tokens=n * length)
    every = list(range(n))
    p.append(every, [length - 7 * (i % 9) for i in every])
    for kind, t in (("prefill", 17), ("prefill", 32), ("decode", 1)):
        lens = [t] * n
        p.append(every, lens)
        q = R.in_type(p.queries(lens) * np.float32(6), dtype)
        out = p.attend(every, lens, q, 0, kind)
        sampled(p, every, lens, q, 0, out, sorted({0, n // 2, n - 1}), assert_sharp, kind)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,length", [(1, 4000), (50, 1500)])
@pytest.mark.parametrize("tokens,first,last", [(17, 0, 17), (17, 0, 8), (17, 8, 16), (17, 16, 17),
                                               (32, 20, 25), (5, 3, 4), (1, 0, 1)])
def test_logits_that_rise_along_the_cache(dtype, n, length, tokens, first, last):
    """Keys that every 128 positions weigh 3.3 times more for the tokens [first, last): their sums pass
    any bound stage after stage, those of the other tokens' rows never do."""
    d = 128 if dtype == "bf16" else 64
    p = Pair(dtype, 1, n, layers=1, n_pages=n * (length // 16 + 8), most=length + 100,
             tokens=n * length, seed=5)
    every = list(range(n))
    along = np.where(p.rng.random(d) < 0.5, 1, -1).astype(np.float32)
    rise = 1.2 / (0.3 * np.sqrt(d))          # of a key along it, a stage: 1.2 of the logit

    def turned_back(x, pos):
        """Rows [n, heads, d] that the rotation at the positions turns into x."""
        return R.rotate64(x.astype(np.float32), -np.asarray(pos)).astype(np.float32)

    pos = np.concatenate([np.arange(length)] * n)
    k = p.normal(n * length, 1, d) + rise * (pos // 128)[:, None, None] * along
    p.append(every, [length] * n, kv=(R.in_type(turned_back(k, pos), dtype)[:, None],
                                      p.normal(n * length, 1, 1, d)))
    lens = [tokens] * n
    p.append(every, lens)
    # Queries across `along`, and 0.3 of it for those tokens.
    step = np.tile(np.arange(tokens), n)
    mine = (step >= first) & (step < last)
    q = p.normal(n * tokens, 4, d)
    q += (0.3 * mine[:, None] - q @ along / d)[..., None] * along
    q = R.in_type(turned_back(q, length + step), dtype)[:, None]
    if n > 1 and tokens > 1:
        # Weights 2^(s - m + 8) of 64 keys under the first 128 keys' maximum, session 0 (one slice).
        x = R.rotate64(q[:tokens, 0], p.pos[0][length:])
        s = np.einsum("thd,nd->thn", x, p.k[0][:length, 0, 0].astype(np.float64)) / np.sqrt(d) / np.log(2)
        w = np.exp2(s - s[..., :128].max(axis=-1, keepdims=True) + 8)[..., :length // 64 * 64]
        passes = w.reshape(tokens, 4, -1, 64).sum(axis=-1).max(axis=-1) > 2.0 ** 15
        assert (passes == mine[:tokens, None]).all()
    out = p.attend(every, lens, q, 0, "decode" if tokens == 1 else "prefill")
    some = sorted({0, n // 3, n - 1})
    sampled(p, every, lens, q, 0, out, some, assert_sharp, "rising")
