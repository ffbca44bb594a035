"""What is measured of the cache that holds its keys and values in 4 bits: the write, the
read-back and the attention over it, for the sizes that streaming sessions pass through.

A row (the key or value of one position and KV head) is held in groups of 32 dimensions.  A group
of values x has a scale s = max|x| / 7, rounded to 7 significant bits and to a multiple of 2^-20
at the finest, 9344 at most, and the codes c = round(x / s) in -7..7 (ties to even).  It stands for
the values s * c.  A group that holds an infinity or a NaN stands for NaN.  Keys are rotated (rotate-half, binary32, every product and sum rounded)
before they are held; values are held as they are.

The kinds:

  write    one chunk's keys and values of every layer, written layer by layer as a model has them,
           and read back in the element type
  decode   the attention of every layer for one token of each session
  prefill  the attention of every layer for one chunk of each session, causal inside the chunk

With per_layer, the attention call of a layer also writes the chunk's rows of that layer, and what
was written is read back.  Histories are streams of duplex units (17 acoustic positions, a
delimiter, Poisson(3) transcript tokens, a delimiter), of another length for each session, and
evicted once where the case has a budget, so that compacted pages, partly consumed first pages and
partly filled last ones all occur.  Inputs are N(0, 1), rounded to the element type.

Every kind writes the same slots again, so a pass can be repeated.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # true: the calls a user makes of the library; false: the same in elementary operations

ACOUSTIC, DELIM, TRANSCRIPT, BEGIN = 0, 1, 2, 0x80
GROUP, GQA = 32, 4
BASE = 10000.0
DEV = "cuda"


def _case(name, kind, n, *, dtype="bf16", layers=32, heads=8, history=5000, budget=4096, window=10,
          tokens=1, ragged=False, per_layer=False):
    """n sessions; layers; heads: KV heads (4 query heads each); history: positions fed before the
    chunk, at most; budget and window of the eviction (-1: none); tokens of the chunk (ragged: 1 to
    that many, another number for each session)."""
    c = dict(name=name, kind=kind, n=n, dtype=dtype, layers=layers, heads=heads, history=history,
             budget=budget, window=window, tokens=tokens, ragged=ragged, per_layer=per_layer)
    if name is None:
        del c["name"]
    return c


def listed():
    return [
        # One token of one conversation, all layers: the smallest write, where launches count.
        _case("write_s1_token", "write", 1, history=37, budget=-1),
        # One unit of nine conversations.
        _case("write_s9_unit", "write", 9, history=100, budget=-1, tokens=17),
        # Three sessions restored from their tokens: odd lengths, thousands of rows.
        _case("write_s3_history", "write", 3, layers=16, history=5, budget=-1, tokens=4099,
              ragged=True),
        # The small binary32 shape.
        _case("write_f32_s2", "write", 2, dtype="f32", layers=8, heads=4, history=21, budget=-1,
              tokens=1501),
        # One conversation answers: most rounds of a speaking turn.
        _case("decode_s1", "decode", 1),
        # A few conversations in a model's order: the call writes its layer's row and attends.
        _case("decode_s6_per_layer", "decode", 6, layers=16, per_layer=True),
        # The full batch of the benchmark.
        _case("decode_s64", "decode", 64, layers=8),
        # binary32 sessions.
        _case("decode_f32_s4", "decode", 4, dtype="f32", layers=8, history=2100, budget=-1),
        # One unit of one conversation: what a single user waits for.
        _case("prefill_s1", "prefill", 1, tokens=17),
        # Nine conversations in a model's order.
        _case("prefill_s9_per_layer", "prefill", 9, layers=16, tokens=17, per_layer=True),
        # The full batch.
        _case("prefill_s64", "prefill", 64, layers=4, tokens=17),
        # binary32 chunks of different lengths.
        _case("prefill_f32_s3", "prefill", 3, dtype="f32", layers=8, history=1100, budget=-1,
              tokens=23, ragged=True),
    ]


MOST_ROWS = 64 * 4096 * 8 * 8      # (session, position, layer, KV head) rows of a drawn decode
MOST_PRODUCTS = 64 * 17 * 4096 * 8 * 4  # and (query, key) pairs over layers and KV heads of a chunk


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "decode", "decode", "prefill", "prefill"])
    f32 = rng.random() < 0.25
    heads = rng.choice([1, 2, 4, 5, 8])
    layers = rng.randint(1, 8) if f32 else rng.choice([3, 8, 16, 32])
    window = rng.choice([1, 5, 10, 20])
    dtype = "f32" if f32 else "bf16"
    if kind == "write":
        tokens = _log(rng, 1, 4000)
        most = max(1, 3 * 4099 * 16 * 8 // (tokens * layers * heads))
        return _case(None, kind, min(_log(rng, 1, 64), most), dtype=dtype, layers=layers,
                     heads=heads, history=_log(rng, 1, 300), budget=-1, window=window,
                     tokens=tokens, ragged=rng.random() < 0.5)
    tokens = 1 if kind == "decode" else rng.choice([17, 17, rng.randint(2, 32)])
    history = _log(rng, 1, 9000)
    rows = MOST_ROWS if kind == "decode" else MOST_PRODUCTS // tokens
    n = min(_log(rng, 1, 64), max(1, rows // (layers * heads * (history + tokens))))
    budget = _log(rng, 256, 8192) if rng.random() < 0.5 else -1
    return _case(None, kind, n, dtype=dtype, layers=layers, heads=heads, history=history,
                 budget=budget, window=window, tokens=tokens,
                 ragged=kind == "prefill" and rng.random() < 0.4, per_layer=rng.random() < 0.4)


# -- the sessions ----------------------------------------------------------------------------
def _history(rng, fed):
    """Type bytes of `fed` positions of duplex units."""
    out = []
    while len(out) < fed:
        out += [ACOUSTIC | BEGIN] + [ACOUSTIC] * 16
        out += [DELIM] + [TRANSCRIPT] * min(64, int(rng.poisson(3))) + [DELIM]
    return np.array(out[:fed], np.uint8)


def _kept(types, budget, window):
    """Positions that one eviction leaves: while over budget, the acoustic and delimiter positions
    of the oldest unit outside the window go."""
    pos = np.arange(len(types))
    over = len(types) - budget
    if budget < 0 or over <= 0:
        return pos
    unit = np.cumsum((types & BEGIN) != 0) - 1
    goes = ((types & 0x7F) <= DELIM) & (unit <= unit[-1] - window)
    gone = np.cumsum(np.bincount(unit[goes], minlength=int(unit[-1]) + 1))
    return pos[~(goes & (unit <= int(np.searchsorted(gone, over))))]


def _chunk_lengths(case):
    """Tokens of each session's chunk, the same for every seed."""
    if not case["ragged"]:
        return np.full(case["n"], case["tokens"])
    return np.random.default_rng([case["n"], case["tokens"]]).integers(1, case["tokens"] + 1,
                                                                       size=case["n"])


def _sessions(case, seed):
    """Types of each session's history, and the positions of it that stay."""
    types = []
    for i in range(case["n"]):
        rng = np.random.default_rng([seed, i])
        types.append(_history(rng, int(rng.integers(-(-3 * case["history"] // 4),
                                                    case["history"] + 1))))
    return types, [_kept(t, case["budget"], case["window"]) for t in types]


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _dim(case):
    return 128 if case["dtype"] == "bf16" else 64


def _normal(case, shape, *key):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(np.random.SeedSequence(key).generate_state(1, np.uint64)[0] >> np.uint64(1)))
    return torch.randn(shape, generator=g, device=DEV, dtype=_dt(case))


def _history_kv(case, seed, layer, total):
    return _normal(case, (2, total, case["heads"], _dim(case)), seed, 1, layer)


def _chunk_kv(case, seed, total):
    return _normal(case, (2, case["layers"], total, case["heads"], _dim(case)), seed, 2)


def _queries(case, seed, total):
    return _normal(case, (case["layers"], total, GQA * case["heads"], _dim(case)), seed, 3)


# -- the plain form ---------------------------------------------------------------------------
def _table(case, positions):
    """cos and sin [positions][D/2], evaluated in 64 bits and held in 32."""
    d = _dim(case)
    theta = torch.pow(torch.tensor(BASE, dtype=torch.float64, device=DEV),
                      -2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    a = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * theta
    return torch.cos(a).float(), torch.sin(a).float()


def _rotated(x, cos, sin):
    """x [..., tokens, heads, D] in 32 bits; cos, sin [tokens, D/2]."""
    a, b = x.float().chunk(2, dim=-1)
    c, s = cos[:, None], sin[:, None]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _held(x):
    """Codes (int8, the shape of x) and scales (one for each 32 dimensions) that stand for x."""
    g = x.unflatten(-1, (-1, GROUP))
    most = g.abs().amax(dim=-1, keepdim=True)
    fine = torch.isfinite(most)
    # (Divided by a tensor: a division by a number is a product with its rounded reciprocal.)
    s = torch.where(fine, most, 0.0) / torch.full_like(most, 7.0)
    # 2 to the exponent of the seventh significant bit, made of its bits: pow may be off by one.
    q = ((torch.clamp(torch.frexp(s)[1] - 7, min=-20) + 127) << 23).view(torch.float32)
    s = torch.clamp(torch.round(s / q) * q, max=9344.0)
    c = torch.where(fine, torch.clamp(torch.round(g / torch.where(s > 0, s, 1.0)), -7, 7), 0.0)
    return c.to(torch.int8).flatten(-2), torch.where(fine, s, math.nan).squeeze(-1)


def _values(codes, scales):
    return (codes.unflatten(-1, (-1, GROUP)).float() * scales[..., None]).flatten(-2)


def _prepare_plain(case, seed, state):
    types, kept = state["types"], state["kept"]
    layers, n, heads, d = case["layers"], case["n"], case["heads"], _dim(case)
    state["cos"], state["sin"] = _table(case, max(len(t) for t in types) + int(case["tokens"]))
    if case["kind"] == "write":
        return
    # Rows [layer][session][head][position]: the kept history, then the chunk.
    room = max(len(k) for k in kept) + int(state["lens"].max())
    state["codes"] = torch.zeros((2, layers, n, heads, room, d), dtype=torch.int8, device=DEV)
    state["scales"] = torch.zeros((2, layers, n, heads, room, d // GROUP), device=DEV)
    base = np.concatenate([[0], np.cumsum([len(t) for t in types])])
    rows = torch.as_tensor(np.concatenate([k + b for k, b in zip(kept, base)]), device=DEV)
    pos = torch.as_tensor(np.concatenate(kept), device=DEV)
    who = torch.as_tensor(np.repeat(np.arange(n), [len(k) for k in kept]), device=DEV)
    at = torch.as_tensor(np.concatenate([np.arange(len(k)) for k in kept]), device=DEV)
    for layer in range(layers):
        k, v = _history_kv(case, seed, layer, int(base[-1]))[:, rows]
        for i, x in enumerate((_rotated(k, state["cos"][pos], state["sin"][pos]), v.float())):
            c, s = _held(x)
            state["codes"][i, layer, who, :, at] = c
            state["scales"][i, layer, who, :, at] = s
    state["room"] = room
    if not case["per_layer"]:
        _write_plain(state)


def _write_plain(state):
    """The chunk's rows into their slots; their codes and scales [layer][token][head]."""
    pos = state["pos"]
    got = [_held(_rotated(state["k"], state["cos"][pos], state["sin"][pos])),
           _held(state["v"].float())]
    if "codes" in state:
        for i, (c, s) in enumerate(got):
            state["codes"][i][:, state["who"], :, state["at"]] = c.transpose(0, 1)
            state["scales"][i][:, state["who"], :, state["at"]] = s.transpose(0, 1)
    return got


def _run_plain(state):
    case = state["case"]
    out = {}
    if case["kind"] == "write" or case["per_layer"]:
        out["k"], out["v"] = (_values(c, s).to(_dt(case)) for c, s in _write_plain(state))
    if case["kind"] == "write":
        return out
    n, heads, d, layers = case["n"], case["heads"], _dim(case), case["layers"]
    who, step, pos = state["who"], state["step"], state["pos"]
    most = int(state["lens"].max())
    q = torch.zeros((layers, n, most, heads * GQA, d), device=DEV)
    q[:, who, step] = _rotated(state["q"], state["cos"][pos], state["sin"][pos])
    # [layer, session, head, token * query head of the group, D]
    q = q.unflatten(3, (heads, GQA)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4)
    k, v = (_values(state["codes"][i], state["scales"][i]) for i in (0, 1))
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(d)
    last = state["first"][:, None] + torch.arange(most, device=DEV)  # index of each token's own row
    hidden = torch.arange(state["room"], device=DEV) > last[..., None]
    s = s.unflatten(3, (most, GQA)).masked_fill(hidden[None, :, None, :, None], -math.inf)
    p = torch.exp(s - s.amax(dim=-1, keepdim=True))
    p = (p / p.sum(dim=-1, keepdim=True)).flatten(3, 4)
    o = torch.matmul(p, v).unflatten(3, (most, GQA)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4)
    out["out"] = o[:, who, step].to(_dt(case))
    return out


# -- the library's calls ------------------------------------------------------------------------
def _layers(x):
    return [x.data_ptr() + i * x.stride(0) * x.element_size() for i in range(x.shape[0])]


def _prepare_own(case, seed, state):
    from paper_2609_31224_gb300 import KVCache
    from paper_2609_31224_gb300._lib import host_i32

    types, lens, n = state["types"], state["lens"], case["n"]
    fed = np.array([len(t) for t in types])
    pages = (fed + lens) // 16 + 4
    pages += np.array([len(k) for k in state["kept"]]) // 16 if case["budget"] >= 0 else 0
    cache = KVCache(n_sessions=n, layers=case["layers"], q_heads=GQA * case["heads"],
                    kv_heads=case["heads"], head_dim=_dim(case), budget=case["budget"],
                    window=case["window"], dtype=case["dtype"], rope_base=BASE,
                    n_pages=int(pages.sum()), max_pages_per_session=int(pages.max()),
                    max_positions=int((fed + lens).max()) + 1, max_seq_per_call=n,
                    max_tokens_per_call=int(max(fed.sum(), lens.sum())), device=DEV, kv_bits=4)
    sessions = np.arange(n, dtype=np.int32)
    cache.append_chunk(sessions, np.concatenate([[0], np.cumsum(fed)]),
                       torch.as_tensor(np.concatenate(types), device=DEV), None, None)
    for layer in range(case["layers"]):
        k, v = _history_kv(case, seed, layer, int(fed.sum()))
        cache.append_kv_layer(layer, k, v)
    if case["budget"] >= 0:
        cache.evict(sessions)
    chunk = np.zeros(int(lens.sum()), np.uint8)
    whole = case["kind"] != "write" and not case["per_layer"]
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cache.append_chunk(sessions, cu, torch.as_tensor(chunk, device=DEV),
                       state["k"] if whole else None, state["v"] if whole else None)
    state["cache"] = cache
    state["k_ptr"], state["v_ptr"] = _layers(state["k"]), _layers(state["v"])
    if case["kind"] != "write":
        state["out"] = torch.zeros_like(state["q"])
        state["q_ptr"], state["out_ptr"] = _layers(state["q"]), _layers(state["out"])
    # The rows to read back: each session's chunk, behind what stays of its history.
    state["k_read"], state["v_read"] = torch.zeros_like(state["k"]), torch.zeros_like(state["v"])
    state["sess"], state["sess_p"] = host_i32(sessions)
    state["cu"], state["cu_p"] = host_i32(cu)
    state["skip"], state["skip_p"] = host_i32([len(k) for k in state["kept"]])


def _run_own(state):
    case, cache = state["case"], state["cache"]
    stream = torch.cuda.current_stream().cuda_stream
    out = {}
    if case["kind"] == "write":
        for layer, (k, v) in enumerate(zip(state["k_ptr"], state["v_ptr"])):
            cache.append_kv_layer_raw(layer, k, v, stream)
    elif case["per_layer"]:
        fn = cache.attn_decode_kv_raw if case["kind"] == "decode" else cache.attn_prefill_kv_raw
        for layer, (k, v, q, o) in enumerate(zip(state["k_ptr"], state["v_ptr"], state["q_ptr"],
                                                 state["out_ptr"])):
            fn(layer, k, v, q, o, stream)
    else:
        fn = cache.attn_decode_raw if case["kind"] == "decode" else cache.attn_prefill_raw
        for layer, (q, o) in enumerate(zip(state["q_ptr"], state["out_ptr"])):
            fn(layer, q, o, stream)
    if case["kind"] == "write" or case["per_layer"]:
        cache.read_kv_raw(case["n"], state["sess_p"], state["skip_p"], state["cu_p"], 0,
                          case["layers"], state["k_read"].data_ptr(), state["v_read"].data_ptr(),
                          None, stream)
        out["k"], out["v"] = state["k_read"], state["v_read"]
    if case["kind"] != "write":
        out["out"] = state["out"]
    return out


# -- what is measured ---------------------------------------------------------------------------
def prepare(case, seed):
    types, kept = _sessions(case, seed)
    lens = _chunk_lengths(case)
    total = int(lens.sum())
    state = dict(case=case, types=types, kept=kept, lens=lens)
    state["k"], state["v"] = _chunk_kv(case, seed, total)
    if case["kind"] != "write":
        state["q"] = _queries(case, seed, total)
    if own:
        _prepare_own(case, seed, state)
        return state
    who = np.repeat(np.arange(case["n"]), lens)
    step = np.concatenate([np.arange(t) for t in lens])
    first = np.array([len(k) for k in kept])
    fed = np.array([len(t) for t in types])
    for name, x in (("who", who), ("step", step), ("pos", fed[who] + step),
                    ("at", first[who] + step), ("first", first)):
        state[name] = torch.as_tensor(x, device=DEV)
    _prepare_plain(case, seed, state)
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Rows in the element type are read or written once each; rows of the cache are D/2 bytes of
    codes and D/16 bytes of scales."""
    d, esz = _dim(case), 2 if case["dtype"] == "bf16" else 4
    lens = _chunk_lengths(case)
    every = case["layers"] * case["heads"] * d
    row, held = every * esz, every * 9 // 16      # K or V of one position, all layers and heads
    written = 2.0 * lens.sum() * (2 * row + held)  # given, held, and given back
    if case["kind"] == "write":
        return {"bytes": written, "flops": 12.0 * 2 * lens.sum() * every}
    # Histories are 7/8 of the most on average; an eviction leaves the budget, or what it cannot
    # remove: transcripts (3 of 22 positions) and the units of the window.
    fed = 7 * case["history"] / 8
    keys = fed if case["budget"] < 0 else min(
        fed, max(case["budget"], 3 * fed / 22 + 19 * case["window"]))
    b = sum(2 * (keys + t) * held + 2 * t * GQA * row for t in lens)
    f = sum(4.0 * t * (keys + (t + 1) / 2) * GQA * every for t in lens)
    if case["per_layer"]:
        b += written
    return {"bytes": float(b), "flops": float(f)}


# -- the same in 64 bits --------------------------------------------------------------------------
def _exact_turn(x, pos):
    """Rotate-half of x [..., positions, heads, D] by pos * BASE^(-2 i / D)."""
    d = x.shape[-1]
    z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double())
    i = torch.arange(d // 2, dtype=torch.float64, device=DEV)
    angle = torch.as_tensor(pos, device=DEV).double()[:, None, None] * BASE ** (-2 * i / d)
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], dim=-1)


def _exact_round(x):
    """The values that the cache holds for x."""
    g = x.double().unflatten(-1, (-1, GROUP))
    s = g.abs().max(dim=-1, keepdim=True).values / 7
    powers = torch.tensor([2.0 ** i for i in range(-20, 128)], dtype=torch.float64, device=x.device)
    step = powers[torch.clamp(torch.frexp(s)[1].long() - 7, min=-20) + 20]
    s = torch.clamp(torch.round(s / step) * step, max=9344.0)
    c = torch.round(g / torch.where(s > 0, s, 1.0)).clamp(-7, 7)
    return (c * s).flatten(-2)


def exact(case, seed):
    types, kept = _sessions(case, seed)
    lens = _chunk_lengths(case)
    cuts = np.concatenate([[0], np.cumsum(lens)])
    fed = [len(t) for t in types]
    base = np.concatenate([[0], np.cumsum(fed)])
    k, v = _chunk_kv(case, seed, int(cuts[-1]))
    pos = np.concatenate([np.arange(f, f + t) for f, t in zip(fed, lens)])
    new_k = torch.stack([_exact_round(_exact_turn(x, pos)) for x in k])
    new_v = torch.stack([_exact_round(x) for x in v])
    out = {}
    if case["kind"] == "write" or case["per_layer"]:
        out["k"], out["v"] = new_k, new_v
    if case["kind"] == "write":
        return out
    d = _dim(case)
    q = _queries(case, seed, int(cuts[-1]))
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    for layer in range(case["layers"]):
        hist = _history_kv(case, seed, layer, int(base[-1]))
        for i in range(case["n"]):
            a, b, t = int(cuts[i]), int(cuts[i + 1]), int(lens[i])
            rows = torch.as_tensor(kept[i] + base[i], device=DEV)
            keys = torch.cat([_exact_round(_exact_turn(hist[0, rows], kept[i])), new_k[layer, a:b]])
            vals = torch.cat([_exact_round(hist[1, rows]), new_v[layer, a:b]])
            x = _exact_turn(q[layer, a:b], pos[a:b]).unflatten(1, (case["heads"], GQA))
            s = torch.einsum("thgd,shd->htgs", x, keys) / math.sqrt(d)
            s += torch.triu(torch.full((t, len(keys)), -math.inf, dtype=torch.float64, device=DEV),
                            diagonal=len(keys) - t + 1)[:, None]
            o[layer, a:b] = torch.einsum("htgs,shd->thgd", torch.softmax(s, dim=-1),
                                         vals).flatten(1, 2)
    out["out"] = o
    return out
