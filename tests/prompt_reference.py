"""Plain references of the calls on whole prompts, in 64 bits, and sessions to run them on.

A reference takes the rows that the cache holds (kvc_read_kv gives them exactly), so that it knows
nothing of pages; what is resident, and where, comes from kvc_export_state."""
import numpy as np
import torch

from paper_2609_31224_gb300 import KVCache

GQA, BASE = 4, 10000.0


def make_cache(n, *, dtype="bf16", layers=2, heads=2, budget=-1, window=2, pages=64, positions=2048,
               tokens=4096, n_pages=None, max_seq=None, kv_bits=None):
    return KVCache(n_sessions=n, layers=layers, q_heads=GQA * heads, kv_heads=heads,
                   head_dim=128 if dtype == "bf16" else 64, budget=budget, window=window, dtype=dtype,
                   n_pages=n_pages or n * pages, max_pages_per_session=pages, max_positions=positions,
                   max_seq_per_call=max_seq or n, max_tokens_per_call=tokens, rope_base=BASE,
                   kv_bits=kv_bits)


def stream_types(n, rng):
    """Type bytes of n positions: units of 5 to 9 acoustic positions, a delimiter, a few words."""
    out = []
    while len(out) < n:
        out += [0x80] + [0] * int(rng.integers(4, 9)) + [1] + [2] * int(rng.integers(0, 4))
    return np.array(out[:n], np.uint8)


def rows(cache, total, rng, layers=None):
    """K or V rows [L][total][Hkv][D] and their seed."""
    c = cache.cfg
    g = torch.Generator(device="cuda")
    g.manual_seed(int(rng.integers(1 << 31)))
    return torch.randn((layers or c.layers, total, c.kv_heads, c.head_dim), generator=g, device="cuda",
                       dtype=cache.torch_dtype)


def queries(cache, total, rng):
    c = cache.cfg
    g = torch.Generator(device="cuda")
    g.manual_seed(int(rng.integers(1 << 31)))
    return torch.randn((c.layers, total, c.q_heads, c.head_dim), generator=g, device="cuda",
                       dtype=cache.torch_dtype)


def feed(cache, sessions, lens, rng, types=None):
    """One append of K and V of every layer; the types fed."""
    lens = np.asarray(lens)
    if types is None:
        types = [stream_types(int(t), rng) for t in lens]
    total = int(lens.sum())
    cache.append_chunk(sessions, np.concatenate([[0], np.cumsum(lens)]),
                       torch.as_tensor(np.concatenate(types), device="cuda"), rows(cache, total, rng),
                       rows(cache, total, rng))
    return types


def held(cache, session):
    """Rows that a session holds, K and V [L][n][Hkv][D] in 64 bits."""
    n = cache.resident_size(session)
    k, v = cache.read_kv([session], [0], [0, n])
    return k.double(), v.double()


def rotated(x, positions):
    """Rotate-half of x [tokens, heads, D] in 64 bits."""
    d = x.shape[-1]
    i = torch.arange(d // 2, dtype=torch.float64, device=x.device)
    a = torch.as_tensor(np.asarray(positions), device=x.device).double()[:, None, None] * BASE ** (-2 * i / d)
    lo, hi = x[..., :d // 2].double(), x[..., d // 2:].double()
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], dim=-1)


def attention(cache, session, q, k, v):
    """Outputs [tokens][Hq][D] and weights [n] (summed over tokens and heads) of the chunk's queries q
    [tokens][Hq][D] over one layer's rows k, v [n][Hkv][D]; keys that a token does not see count as
    absent, whatever they hold."""
    st = cache.export_state(session)
    t, n, d = len(q), len(k), q.shape[-1]
    x = rotated(q, np.arange(st["pos_next"] - t, st["pos_next"])).unflatten(1, (-1, GQA))
    seen = torch.arange(n, device=q.device)[None] <= torch.arange(n - t, n, device=q.device)[:, None]
    s = torch.einsum("thgd,nhd->thgn", x, k) / d ** 0.5
    s = torch.where(seen[:, None, None], s, -torch.inf)
    p = torch.softmax(s, dim=-1)
    p = torch.where(seen[:, None, None], p, 0.0)
    o = torch.zeros(t, *x.shape[1:], dtype=torch.float64, device=q.device)
    if torch.isfinite(v).all():
        o = torch.einsum("thgn,nhd->thgd", p, v)
    else:
        for i in range(t):
            m = n - t + i + 1
            o[i] = torch.einsum("hgn,nhd->hgd", p[i, ..., :m], v[:m])
    return o.flatten(1, 2), p.sum(dim=(0, 1, 2))
