"""What is measured of whole prompts: the attention over a prompt of any length, the weight that
each resident position draws, and the eviction of the positions that draw least.

A program that takes a prompt (a system prompt, a document, a conversation restored from its tokens)
feeds it in one chunk, attends over it, adds up what attention weight every position drew, and drops
the positions with the smallest sums so that the cache fits its budget.  The same sums go on growing
while tokens are decoded.

The kinds:

  prompt   the attention of every layer for one chunk of each session, of any length and another for
           each session, causal inside the chunk, over what the session holds: softmax(q . k / sqrt(D)) v
  weights  for the same chunks (single tokens too) the softmax weights themselves, summed over layers,
           query heads and the chunk's queries for each position that is resident
  evict    sessions fed in turns: a turn's keys and values of every layer into the cache, then, of the
           positions of some types that are neither among the first `sink` nor the last `recent` ones,
           those of the smallest weight (of equal ones the oldest) dropped until `keep` are left; then
           the rows that stay read back, and which positions they are

Keys and queries are rotated (rotate-half) at their positions; the cache holds keys rounded to the
element type after the rotation: products with a binary32 table, x1 c - (x2 s) rounded once behind the
rounded product x2 s.  Histories are streams of duplex units (17 acoustic positions, a delimiter,
Poisson(3) transcript tokens, a delimiter), of another length for each session, evicted once where the
case has a budget, so that compacted pages, partly consumed first pages and partly filled last ones all
occur.  Inputs are N(0, 1), rounded to the element type; weights to evict by are products of uniform
numbers in steps of 2^-12, so that small ones are many and often equal.

Every kind leaves its state so that a pass can be repeated.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # true: the calls a user makes of the library; false: the same in elementary operations

ACOUSTIC, DELIM, TRANSCRIPT, BEGIN = 0, 1, 2, 0x80
GQA = 4
BASE = 10000.0
STEP = 2.0 ** -12
DEV = "cuda"


def _case(name, kind, n, *, dtype="bf16", layers=4, heads=8, history=0, budget=-1, window=10,
          tokens=1, ragged=False, turns=1, keep=0, sink=0, recent=0, text=False):
    """n sessions; layers; heads: KV heads (4 query heads each); history: positions fed before the
    chunk, at most (0: none); budget and window of its eviction (-1: none); tokens of the chunk
    (ragged: 1 to that many, another number for each session).  evict: turns of chunks, keep, sink and
    recent as above; text: transcripts stay whatever they weigh."""
    c = dict(name=name, kind=kind, n=n, dtype=dtype, layers=layers, heads=heads, history=history,
             budget=budget, window=window, tokens=tokens, ragged=ragged, turns=turns, keep=keep,
             sink=sink, recent=recent, text=text)
    if name is None:
        del c["name"]
    return c


def listed():
    return [
        # A short system prompt of one conversation: what a user waits for before the first unit.
        _case("prompt_s1_short", "prompt", 1, layers=8, tokens=250),
        # A document of one conversation.
        _case("prompt_s1_4k", "prompt", 1, tokens=4099),
        # Conversations of different lengths restored from their tokens, packed into one call.
        _case("prompt_s8_ragged", "prompt", 8, layers=2, tokens=2500, ragged=True),
        # Long questions asked of sessions that hold an evicted stream.
        _case("prompt_s4_history", "prompt", 4, history=5000, budget=4096, tokens=700, ragged=True),
        # The longest prompt.
        _case("prompt_s1_16k", "prompt", 1, layers=1, tokens=16384),
        # The small binary32 shape.
        _case("prompt_f32_s3", "prompt", 3, dtype="f32", heads=4, tokens=1501, ragged=True),
        # One decoded token of one conversation, all layers: the smallest call, where latency counts.
        _case("weights_s1_token", "weights", 1, layers=32, history=5000, budget=4096),
        # A token of each session of the benchmark's full batch.
        _case("weights_s64_token", "weights", 64, layers=8, history=5000, budget=4096),
        # Two prompts: every query counts.
        _case("weights_s2_prompt", "weights", 2, layers=2, tokens=3001, ragged=True),
        # One unit of binary32 sessions.
        _case("weights_f32_s3_unit", "weights", 3, dtype="f32", layers=8, heads=4, history=1100,
              tokens=17),
        # One prompt thinned out to half, its transcript kept.
        _case("evict_s1_prompt", "evict", 1, layers=32, tokens=4099, keep=2048, sink=4, recent=64,
              text=True),
        # Sixteen sessions in turns, thinned out each time: what stayed is thinned out again.
        _case("evict_s16_turns", "evict", 16, layers=16, tokens=1300, ragged=True, turns=3, keep=700,
              sink=4, recent=33),
    ]


MOST_PAIRS = 16384 ** 2 // 2 * 8      # (query, key) pairs over layers and KV heads of a drawn chunk
MOST_ROWS = 64 * 4096 * 8 * 8         # (session, position, layer, KV head) rows of single tokens
MOST_FED = 16 * 1200 * 16 * 8           # and of what an evict case feeds


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "weights", "weights", "evict"])
    f32 = rng.random() < 0.25
    heads = rng.choice([1, 2, 4, 5, 8])
    layers = rng.choice([1, 2, 3, 4]) if f32 or rng.random() < 0.7 else rng.choice([8, 16, 32])
    dtype = "f32" if f32 else "bf16"
    ragged = rng.random() < 0.5
    if kind == "evict":
        turns = rng.choice([1, 1, 2, 3])
        tokens = _log(rng, 2, 9000)
        most = max(1, MOST_FED // (tokens * turns * layers * heads))
        keep = max(1, int(tokens * rng.uniform(0.1, 0.95)))
        sink = min(rng.choice([0, 0, 4, 17]), keep // 4)
        return _case(None, kind, min(_log(rng, 1, 64), most), dtype=dtype, layers=layers, heads=heads,
                     tokens=tokens, ragged=ragged, turns=turns, keep=keep, sink=sink,
                     recent=min(rng.choice([0, 1, 33, 256]), keep // 2), text=rng.random() < 0.3)
    single = kind == "weights" and rng.random() < 0.5
    tokens = 1 if single else _log(rng, 2, 16000)
    history = _log(rng, 1, 9000) if single or rng.random() < 0.6 else 0

    def most_sessions():
        rows = MOST_ROWS // (1 if kind == "weights" else 3) // (layers * heads * (history + tokens))
        pairs = layers * heads * tokens * (history + tokens // 2 + 1)
        return min(rows, MOST_PAIRS // (4 if f32 else 1) // pairs)

    while most_sessions() < 1:  # too much for one session: fewer layers, then fewer tokens
        if layers > 1:
            layers //= 2
        else:
            tokens = tokens * 3 // 4
    most = most_sessions()
    budget = _log(rng, 256, 8192) if history and rng.random() < 0.5 else -1
    return _case(None, kind, min(_log(rng, 1, 64), most), dtype=dtype, layers=layers, heads=heads,
                 history=history, budget=budget, window=rng.choice([1, 5, 10, 20]), tokens=tokens,
                 ragged=ragged and not single)


# -- the sessions ----------------------------------------------------------------------------
def _stream(rng, fed):
    """Type bytes of `fed` positions of duplex units."""
    units = max(1, -(-fed // 19))
    words = np.minimum(64, rng.poisson(3, size=units))
    out = np.full(int((19 + words).sum()), TRANSCRIPT, np.uint8)
    at = np.concatenate([[0], np.cumsum(19 + words)[:-1]])
    out[(at[:, None] + np.arange(17)).ravel()] = ACOUSTIC
    out[at] = ACOUSTIC | BEGIN
    out[at + 17] = out[at + 18 + words] = DELIM
    return out[:fed]


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
    """Tokens of each session's chunk [turns][n], the same for every seed."""
    if not case["ragged"]:
        return np.full((case["turns"], case["n"]), case["tokens"])
    rng = np.random.default_rng([case["n"], case["tokens"], case["turns"]])
    lens = rng.integers(1, case["tokens"] + 1, size=(case["turns"], case["n"]))
    lens[0, 0] = case["tokens"]
    return lens


def _sessions(case, seed):
    """Types of each session's history, and the positions of it that stay."""
    types = []
    for i in range(case["n"]):
        rng = np.random.default_rng([seed, i])
        types.append(_stream(rng, int(rng.integers(-(-3 * case["history"] // 4),
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


def _chunk_kv(case, seed, turn, total):
    return _normal(case, (2, case["layers"], total, case["heads"], _dim(case)), seed, 2, turn)


def _queries(case, seed, total):
    return _normal(case, (case["layers"], total, GQA * case["heads"], _dim(case)), seed, 3)


def _draw_weights(case, seed, shape):
    """What the positions weigh: products of three uniform numbers in steps of 2^-12."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(np.random.SeedSequence([seed, 4]).generate_state(1, np.uint64)[0] >> np.uint64(1)))
    u = torch.rand((3, *shape), generator=g, device=DEV)
    return torch.floor(u.prod(dim=0) / STEP) * STEP


def _dev(x):
    return torch.as_tensor(np.ascontiguousarray(x), device=DEV)


def _cat(parts):
    return np.concatenate(parts) if len(parts) else np.zeros(0, np.int64)


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


def _held(case, x, cos, sin):
    """Keys as the cache holds them: the first product and the sum in 64 bits, where they are exact,
    rounded to 32 and then to the element type."""
    a, b = x.float().chunk(2, dim=-1)
    c, s = cos[:, None], sin[:, None]
    y = torch.cat([(a.double() * c - (b * s)).float(), (b.double() * c + (a * s)).float()], dim=-1)
    return y.to(_dt(case))


def _prepare_plain(case, seed, state):
    n, layers, heads, d = case["n"], case["layers"], case["heads"], _dim(case)
    types, kept, lens = state["types"], state["kept"], state["lens"]
    fed = np.array([len(t) for t in types])
    state["cos"], state["sin"] = _table(case, state["positions"])
    if case["kind"] == "evict":
        return
    # Rows [layer][session][head][row]: the kept history, then the chunk.
    first = np.array([len(k) for k in kept])
    who = np.repeat(np.arange(n), lens[0])
    step = _cat([np.arange(t) for t in lens[0]])
    room = int((first + lens[0]).max())
    pos = fed[who] + step
    state["room"] = room
    for name, x in (("who", who), ("step", step), ("pos", pos), ("first", first)):
        state[name] = _dev(x)
    rows_at = np.concatenate([_cat([np.arange(len(k)) for k in kept]), first[who] + step])
    rows_who = np.concatenate([np.repeat(np.arange(n), first), who])
    state["rows_pos"] = _dev(np.concatenate([_cat(kept), pos]).astype(np.int64))
    state["rows_at"], state["rows_who"] = _dev(rows_at.astype(np.int64)), _dev(rows_who)
    base = np.concatenate([[0], np.cumsum(fed)])
    rows = _dev(_cat([k + b for k, b in zip(kept, base)]).astype(np.int64))
    held = torch.zeros((2, layers, n, heads, room, d), dtype=_dt(case), device=DEV)
    for layer in range(layers):
        k, v = torch.cat([_history_kv(case, seed, layer, int(base[-1]))[:, rows],
                          torch.stack([state["k"][0][layer], state["v"][0][layer]])], dim=1)
        k = _held(case, k, state["cos"][state["rows_pos"]], state["sin"][state["rows_pos"]])
        held[0, layer, state["rows_who"], :, state["rows_at"]] = k
        held[1, layer, state["rows_who"], :, state["rows_at"]] = v
    state["held"] = held


def _softmax_plain(state):
    """Softmax weights [layer, session, KV head, token * query head of the group, row] in 32 bits."""
    case = state["case"]
    n, heads, d, layers = case["n"], case["heads"], _dim(case), case["layers"]
    who, step, pos = state["who"], state["step"], state["pos"]
    most = int(state["lens"].max())
    q = torch.zeros((layers, n, most, heads * GQA, d), device=DEV)
    q[:, who, step] = _rotated(state["q"], state["cos"][pos], state["sin"][pos]) / math.sqrt(d)
    q = q.unflatten(3, (heads, GQA)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4)
    s = torch.matmul(q, state["held"][0].float().transpose(-1, -2))
    last = state["first"][:, None] + torch.arange(most, device=DEV)  # index of each token's own row
    hidden = torch.arange(state["room"], device=DEV) > last[..., None]
    s.unflatten(3, (most, GQA)).masked_fill_(hidden[None, :, None, :, None], -math.inf)
    s.sub_(s.amax(dim=-1, keepdim=True)).exp_()
    return s.div_(s.sum(dim=-1, keepdim=True))


def _prompt_plain(state):
    case = state["case"]
    p = _softmax_plain(state)
    o = torch.matmul(p, state["held"][1].float())
    o = o.unflatten(3, (-1, GQA)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4)
    return {"out": o[:, state["who"], state["step"]].to(_dt(case))}


def _weights_plain(state):
    case = state["case"]
    p = _softmax_plain(state).unflatten(3, (-1, GQA))
    # (A padding token's row is a softmax too: it does not count.)
    real = torch.arange(p.shape[3], device=DEV) < _dev(state["lens"][0])[:, None]
    p.mul_(real[None, :, None, :, None, None])
    drawn = p.sum(dim=(2, 3, 4)).double().sum(dim=0)
    out = torch.zeros((case["n"], state["positions"]), dtype=torch.float64, device=DEV)
    out[state["rows_who"], state["rows_pos"]] = drawn[state["rows_who"], state["rows_at"]]
    return {"weights": out.float()}


def _evict_plain(state):
    case = state["case"]
    n, positions = case["n"], state["positions"]
    here = torch.zeros((n, positions), dtype=torch.bool, device=DEV)
    at = torch.arange(positions, device=DEV)
    for turn, fed in enumerate(state["ends"]):  # positions fed by the end of each turn [n, 1]
        here |= state["turn_of"] == turn
        goes = here & state["may_go"] & (at >= case["sink"]) & (at < fed - case["recent"])
        over = here.sum(dim=1, keepdim=True) - case["keep"]
        order = torch.where(goes, state["weights"], math.inf).sort(dim=1, stable=True).indices
        rank = torch.zeros_like(order).scatter_(1, order, at.expand(n, -1).contiguous())
        here &= ~(goes & (rank < over))
    k, v = (torch.cat(x, dim=1) for x in (state["k"], state["v"]))
    k = _held(case, k, state["cos"][state["fed_pos"]], state["sin"][state["fed_pos"]])
    rows = state["fed_row"][here]     # row of each position that stays, session by session
    return {"kept": here, "resident": here.sum(dim=1), "k": k[:, rows], "v": v[:, rows]}


# -- the library's calls ------------------------------------------------------------------------
def _layers(x):
    return [x.data_ptr() + i * x.stride(0) * x.element_size() for i in range(x.shape[0])]


def _prepare_own(case, seed, state):
    from paper_2609_31224_gb300 import KVCache
    from paper_2609_31224_gb300._lib import host_i32

    types, lens, n = state["types"], state["lens"], case["n"]
    fed = np.array([len(t) for t in types])
    pages = (fed + lens.sum(axis=0)) // 16 + 6
    pages += np.array([len(k) for k in state["kept"]]) // 16 if case["budget"] >= 0 else 0
    cache = KVCache(n_sessions=n, layers=case["layers"], q_heads=GQA * case["heads"],
                    kv_heads=case["heads"], head_dim=_dim(case), budget=case["budget"],
                    window=case["window"], dtype=case["dtype"], rope_base=BASE,
                    n_pages=int(pages.sum()), max_pages_per_session=int(pages.max()),
                    max_positions=state["positions"], max_seq_per_call=n,
                    max_tokens_per_call=int(max(fed.sum(), lens.sum(axis=1).max())), device=DEV)
    state["cache"] = cache
    sessions = state["sessions"] = np.arange(n, dtype=np.int32)
    if fed.any():
        some = sessions[fed > 0]
        cache.append_chunk(some, np.concatenate([[0], np.cumsum(fed[fed > 0])]),
                           _dev(np.concatenate(types)), None, None)
        for layer in range(case["layers"]):
            k, v = _history_kv(case, seed, layer, int(fed.sum()))
            cache.append_kv_layer(layer, k, v)
        if case["budget"] >= 0:
            cache.evict(some)
    state["cu"] = [np.concatenate([[0], np.cumsum(t)]).astype(np.int32) for t in lens]
    if case["kind"] == "evict":
        state["turn_types"] = [_dev(t) for t in state["turn_types"]]
        rows = state["rows"]  # that stay, of each session
        state["first"] = np.zeros(n, np.int32)
        state["cu_rows"] = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        shape = (case["layers"], int(rows.sum()), case["heads"], _dim(case))
        state["k_read"], state["v_read"] = (torch.zeros(shape, dtype=_dt(case), device=DEV)
                                            for _ in range(2))
        state["kept_out"] = torch.zeros((n, state["positions"]), dtype=torch.bool, device=DEV)
        state["resident"] = torch.zeros(n, dtype=torch.int64, device=DEV)
        state["keep"] = np.full(n, case["keep"], np.int32)
        return
    chunk = np.zeros(int(lens[0].sum()), np.uint8)
    cache.append_chunk(sessions, state["cu"][0], _dev(chunk), state["k"][0], state["v"][0])
    state["q_ptr"] = _layers(state["q"])
    if case["kind"] == "prompt":
        state["out"] = torch.zeros_like(state["q"])
        state["out_ptr"] = _layers(state["out"])
    else:
        state["weights"] = cache.make_weights()
        state["work"] = cache.make_weights_workspace()


def _run_own(state):
    case, cache = state["case"], state["cache"]
    stream = torch.cuda.current_stream().cuda_stream
    if case["kind"] == "prompt":
        for layer, (q, o) in enumerate(zip(state["q_ptr"], state["out_ptr"])):
            cache.attn_prompt_raw(layer, q, o, stream)
        return {"out": state["out"]}
    if case["kind"] == "weights":
        state["weights"].zero_()
        weights, work = state["weights"].data_ptr(), state["work"].data_ptr()
        for layer, q in enumerate(state["q_ptr"]):
            cache.attn_weights_raw(layer, q, weights, work, state["work"].numel(), stream)
        return {"weights": state["weights"]}
    sessions = state["sessions"]
    cache.release(sessions, stream)
    state["kept_out"].zero_()
    for cu, types, k, v in zip(state["cu"], state["turn_types"], state["k"], state["v"]):
        cache.append_chunk(sessions, cu, types, k, v, stream)
        cache.evict_weighted(sessions, state["keep"], state["weights"], kinds=state["kinds"],
                             sink=case["sink"], recent=case["recent"], resident_out=state["resident"],
                             kept=state["kept_out"], stream=stream)
    cache.read_kv(sessions, state["first"], state["cu_rows"], k=state["k_read"], v=state["v_read"],
                  stream=stream)
    return {"kept": state["kept_out"], "resident": state["resident"], "k": state["k_read"],
            "v": state["v_read"]}


# -- what is measured ---------------------------------------------------------------------------
def _prepare_evict(case, seed, state):
    """Types and weights of the positions that the turns feed, and where their rows are."""
    n, lens = case["n"], state["lens"]
    total = lens.sum(axis=0)
    types = [_stream(np.random.default_rng([seed, i, 5]), int(t)) for i, t in enumerate(total)]
    cuts = np.concatenate([np.zeros((1, n), np.int64), np.cumsum(lens, axis=0)])
    state["turn_types"] = [np.concatenate([t[a:b] for t, a, b in zip(types, cuts[j], cuts[j + 1])])
                           for j in range(case["turns"])]
    state["kinds"] = (1 << ACOUSTIC | 1 << DELIM) if case["text"] else 0xF
    state["weights"] = _draw_weights(case, seed, (n, state["positions"]))
    may_go = np.zeros((n, state["positions"]), bool)
    fed_row = np.zeros((n, state["positions"]), np.int64)
    at = 0
    for j in range(case["turns"]):
        for i in range(n):
            fed_row[i, cuts[j][i]:cuts[j + 1][i]] = at + np.arange(lens[j][i])
            at += int(lens[j][i])
    for i, t in enumerate(types):
        may_go[i, :len(t)] = (state["kinds"] >> (t & 0x7F).astype(np.int64)) & 1 != 0
    # Rows that stay: as many as `keep`, more where too few positions may go.
    w, rows = state["weights"].cpu().numpy(), np.zeros(n, np.int64)
    for i in range(n):
        here = np.zeros(state["positions"], bool)
        for j in range(case["turns"]):
            a, b = cuts[j][i], cuts[j + 1][i]
            here[a:b] = True
            goes = np.flatnonzero(here & may_go[i])
            goes = goes[(goes >= case["sink"]) & (goes < b - case["recent"])]
            over = max(0, int(here.sum()) - case["keep"])
            here[goes[np.argsort(w[i, goes], kind="stable")[:over]]] = False
        rows[i] = here.sum()
    state["rows"] = rows
    if own:
        return
    state["may_go"], state["fed_row"] = _dev(may_go), _dev(fed_row)
    state["fed_pos"] = _dev(_cat([np.arange(a, b) for j in range(case["turns"])
                                  for a, b in zip(cuts[j], cuts[j + 1])]))
    state["ends"] = [_dev(c[:, None]) for c in cuts[1:]]
    turn_of = np.full((n, state["positions"]), -1)  # the turn that feeds a position
    for j in range(case["turns"]):
        for i in range(n):
            turn_of[i, cuts[j][i]:cuts[j + 1][i]] = j
    state["turn_of"] = _dev(turn_of)


def prepare(case, seed):
    lens = _chunk_lengths(case)
    if case["kind"] == "evict":
        types, kept = [np.zeros(0, np.uint8)] * case["n"], [np.zeros(0, np.int64)] * case["n"]
    else:
        types, kept = _sessions(case, seed)
    state = dict(case=case, types=types, kept=kept, lens=lens)
    state["positions"] = case["history"] + int(lens.sum(axis=0).max()) + 1
    turns = [_chunk_kv(case, seed, j, int(t)) for j, t in enumerate(lens.sum(axis=1))]
    state["k"], state["v"] = [t[0] for t in turns], [t[1] for t in turns]
    if case["kind"] == "evict":
        _prepare_evict(case, seed, state)
    else:
        state["q"] = _queries(case, seed, int(lens.sum()))
    if own:
        _prepare_own(case, seed, state)
    else:
        _prepare_plain(case, seed, state)
    return state


def run(state):
    if own:
        return _run_own(state)
    return {"prompt": _prompt_plain, "weights": _weights_plain,
            "evict": _evict_plain}[state["case"]["kind"]](state)


def work(case):
    """Rows of keys, values, queries and outputs once each; two operations for each product."""
    d, esz = _dim(case), 2 if case["dtype"] == "bf16" else 4
    lens = _chunk_lengths(case)
    every = case["layers"] * case["heads"] * d
    row = every * esz                      # K or V of one position, all layers and heads
    if case["kind"] == "evict":
        # Fed: read and written.  What stays: moved together (read and written) in the last turn,
        # and read back.
        fed = float(lens.sum())
        stay = sum(min(int(t), case["keep"]) for t in lens.sum(axis=0))
        return {"bytes": 2 * row * (2 * fed + 4 * stay), "flops": 6.0 * fed * every}
    # Histories are 7/8 of the most on average; an eviction leaves the budget, or what it cannot
    # remove: transcripts (3 of 22 positions) and the units of the window.
    fed = 7 * case["history"] / 8
    keys = fed if case["budget"] < 0 else min(
        fed, max(case["budget"], 3 * fed / 22 + 19 * case["window"]))
    pairs = sum(t * (keys + (t + 1) / 2) for t in lens[0])
    if case["kind"] == "prompt":
        b = sum(2 * (keys + t) * row + 2 * t * GQA * row for t in lens[0])
        return {"bytes": float(b), "flops": 4.0 * pairs * GQA * every}
    b = sum((keys + t) * row + t * GQA * row + 8 * (keys + t) for t in lens[0])
    return {"bytes": float(b), "flops": 2.0 * pairs * GQA * every}


# -- the same in 64 bits --------------------------------------------------------------------------
def _exact_angles(x, pos):
    d = x.shape[-1]
    i = torch.arange(d // 2, dtype=torch.float64, device=DEV)
    return torch.as_tensor(pos, device=DEV).double()[:, None, None] * BASE ** (-2 * i / d)


def _exact_turn(x, pos):
    """Rotate-half of x [..., positions, heads, D] by pos * BASE^(-2 i / D)."""
    d = x.shape[-1]
    z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double())
    angle = _exact_angles(x, pos)
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], dim=-1)


def _exact_key(x, pos):
    """What the cache holds of keys x [positions, heads, D]: each rounding to 32 bits by itself."""
    d = x.shape[-1]
    angle = _exact_angles(x, pos)
    cos, sin = angle.cos().float().double(), angle.sin().float().double()
    a, b = x[..., :d // 2].double(), x[..., d // 2:].double()

    def r32(y):
        return y.float().double()

    y = torch.cat([r32(a * cos - r32(b * sin)), r32(b * cos + r32(a * sin))], dim=-1)
    return y.float().to(x.dtype).double()


def _exact_attention(case, seed):
    types, kept = _sessions(case, seed)
    lens = _chunk_lengths(case)[0]
    cuts = np.concatenate([[0], np.cumsum(lens)])
    base = np.concatenate([[0], np.cumsum([len(t) for t in types])])
    new = _chunk_kv(case, seed, 0, int(cuts[-1]))
    q = _queries(case, seed, int(cuts[-1]))
    d, heads = _dim(case), case["heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    positions = case["history"] + int(lens.max()) + 1
    weights = torch.zeros((case["n"], positions), dtype=torch.float64, device=DEV)
    for layer in range(case["layers"]):
        hist = _history_kv(case, seed, layer, int(base[-1]))
        for i in range(case["n"]):
            a, b, t = int(cuts[i]), int(cuts[i + 1]), int(lens[i])
            at = np.concatenate([kept[i], len(types[i]) + np.arange(t)])
            rows = torch.as_tensor(kept[i] + base[i], device=DEV)
            keys = torch.cat([hist[0, rows], new[0, layer, a:b]])
            vals = torch.cat([hist[1, rows], new[1, layer, a:b]]).double()
            keys = _exact_key(keys, at)
            x = _exact_turn(q[layer, a:b], at[-t:])
            n_hist = len(kept[i])
            for t0 in range(0, t, 1024):
                t1 = min(t, t0 + 1024)
                seen = n_hist + t1
                mask = torch.triu(torch.full((t1 - t0, seen), -math.inf, dtype=torch.float64,
                                             device=DEV), diagonal=n_hist + t0 + 1)
                for h in range(heads):
                    y = x[t0:t1, GQA * h:GQA * (h + 1)].transpose(0, 1)      # [G, tokens, D]
                    p = torch.softmax(y @ keys[:seen, h].T / math.sqrt(d) + mask, dim=-1)
                    if case["kind"] == "prompt":
                        out[layer, a + t0:a + t1, GQA * h:GQA * (h + 1)] = (
                            p @ vals[:seen, h]).transpose(0, 1)
                    else:
                        weights[i, torch.as_tensor(at[:seen], device=DEV)] += p.sum(dim=(0, 1))
    return {"out": out} if case["kind"] == "prompt" else {"weights": weights}


def _exact_evict(case, seed):
    lens = _chunk_lengths(case)
    n, turns = lens.shape[1], lens.shape[0]
    positions = int(lens.sum(axis=0).max()) + 1
    weights = _draw_weights(case, seed, (n, positions)).double().cpu().numpy()
    news = [_chunk_kv(case, seed, j, int(lens[j].sum())) for j in range(turns)]
    kept = np.zeros((n, positions), bool)
    ks, vs = [], []
    for i in range(n):
        types = _stream(np.random.default_rng([seed, i, 5]), int(lens[:, i].sum())) & 0x7F
        left, fed, k_in, v_in = [], 0, [], []
        for j in range(turns):
            a = int(lens[j, :i].sum())
            k_in.append(news[j][0][:, a:a + lens[j, i]])
            v_in.append(news[j][1][:, a:a + lens[j, i]])
            left += range(fed, fed + int(lens[j, i]))
            fed += int(lens[j, i])
            may = [p for p in left if case["sink"] <= p < fed - case["recent"]
                   and (not case["text"] or types[p] <= DELIM)]
            may.sort(key=lambda p: (weights[i, p], p))
            gone = set(may[:max(0, len(left) - case["keep"])])
            left = [p for p in left if p not in gone]
        kept[i, left] = True
        rows = torch.as_tensor(left, device=DEV)
        ks.append(_exact_turn(torch.cat(k_in, dim=1)[:, rows], left))
        vs.append(torch.cat(v_in, dim=1)[:, rows].double())
    return {"kept": kept, "resident": kept.sum(axis=1), "k": torch.cat(ks, dim=1),
            "v": torch.cat(vs, dim=1)}


def exact(case, seed):
    return _exact_evict(case, seed) if case["kind"] == "evict" else _exact_attention(case, seed)
