"""Rows held in 4 bits, without a GPU: the layout of a tile, the arithmetic that the kernels rely on
(every step exact in binary16), and the host's checks."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2609_31224_gb300 import _lib as L
from paper_2609_31224_gb300 import build as B
from kv4_reference import held

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "kvc_kv4.h"
#include <cstdio>
#include <vector>
using namespace kvc::kv4;

int main() {
  for (int D : {64, 128})
    for (int kv = 0; kv < 2; ++kv) {
      // Each byte of a tile belongs to one row: to two neighbouring dims' codes or half a scale.
      std::vector<int> owner(tile_bytes(D), -1);
      auto take = [&](int at, int row) {
        if (at < 0 || at >= (int)owner.size() || owner[at] != -1) return false;
        owner[at] = row;
        return true;
      };
      for (int slot = 0; slot < ROWS; ++slot) {
        for (int d = 0; d < D; d += 8) {
          const int at = kv ? v_codes(D, slot, d) : k_codes(D, slot, d);
          if (at % 4) return 1;
          for (int i = 0; i < 4; ++i)
            if (!take(at + i, slot)) return 2;
        }
        for (int g = 0; g < D / GROUP; ++g) {
          const int at = kv ? v_scale(D, slot, g) : k_scale(D, slot, g);
          if (at % 2 || !take(at, slot) || !take(at + 1, slot)) return 3;
        }
        // The pieces that an eviction moves are the row's codes.
        for (int p = 0; p < 8; ++p)
          for (int i = 0; i < D / 16; ++i)
            if (owner[(kv ? v_piece(D, slot, p) : k_piece(D, slot, p)) + i] != slot) return 4;
      }
      for (int o : owner)
        if (o < 0) return 5;
      // What lane (g, t) loads at once.
      for (int g = 0; g < 8; ++g)
        for (int t = 0; t < 4; ++t) {
          if (v_piece(D, 2 * t, g) != (g * 4 + t) * (D / 8)) return 6;
          if (v_piece(D, 2 * t + 1, g) != v_piece(D, 2 * t, g) + D / 16) return 7;
          if (v_piece(D, 2 * t + 8, g) != v_piece(D, 2 * t, g) + 4 * D) return 8;
          if (v_scale(D, 2 * t + 1, 0) != v_scale(D, 2 * t, 0) + 2 || v_scale(D, 2 * t, 0) % 4) return 9;
          for (int w = 0; w < D / 32; ++w)
            if (k_codes(D, g, 32 * w + 8 * t) != g * (D / 2) + t * (D / 8) + 4 * w) return 10;
        }
    }
  // Tiles do not overlap, K and V of a head side by side, 16-byte aligned, past 32 bits too.
  if (tile_at(128, 32, 8, 1 << 20, 31, 7, 1) != (((((size_t)1 << 20) * 32 + 31) * 8 + 7) * 2 + 1) * 1152)
    return 11;
  if (page_bytes(128, 2, 3) != tile_at(128, 2, 3, 1, 0, 0, 0) || tile_bytes(64) % 16 || tile_bytes(128) % 16)
    return 12;
  return 0;
}
"""


def test_every_byte_of_a_tile_has_one_owner(tmp_path):
    src, exe = tmp_path / "tile.cpp", tmp_path / "tile"
    src.write_text(PROGRAM)
    inc = os.path.join(ROOT, "paper_2609_31224_gb300", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", inc, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def scales():
    """Every scale: 7 significant bits, multiples of 2^-20, up to 9344."""
    every = {m * 2.0 ** e for e in range(-20, 8) for m in range(128)}
    return np.array(sorted(s for s in every if s <= 9344.0))


def test_a_nibble_becomes_an_exact_binary16_operand():
    """m = s / 16, 72 m, 64 + n and the result (n - 8) m are binary16 numbers, none of them infinite."""
    m = scales() / 16
    n = np.arange(1, 16)
    for x in (m, 72 * m, np.outer(m, n - 8), 64.0 + n):
        with np.errstate(over="raise"):
            assert np.array_equal(x.astype(np.float16).astype(np.float64), x)
    patterns = (0x5400 | n << 4).astype(np.uint16).view(np.float16)
    assert np.array_equal(patterns.astype(np.float64), 64.0 + n)


def test_reference_rounding():
    """The reference itself: a scale within half a unit of its seventh bit, codes within half a
    scale, and the special groups."""
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((4000, 32)) * 10.0 ** rng.uniform(-5, 3, (4000, 1))).astype(np.float32)
    y = held(x)
    most = np.abs(x).max(axis=1, keepdims=True)
    step = np.maximum(most / 7 * 2.0 ** -7, 2.0 ** -21)   # error of a scale, at most
    assert (np.abs(y - x) <= most / 14 + 8 * step).all()
    assert (held(np.zeros((1, 32), np.float32)) == 0).all()
    assert (held(np.full((1, 32), 3.0 * 2.0 ** -20, np.float32)) == 0).all()
    big = np.full((1, 32), 1e30, np.float32)
    assert (held(big) == 65408).all() and (held(-big) == -65408).all()
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones((1, 64), np.float32)
        x[0, 40] = bad
        y = held(x)
        assert np.isnan(y[0, 32:]).all() and np.isfinite(y[0, :32]).all()


def _cfg(**kw):
    base = dict(n_sessions=4, layers=2, q_heads=32, kv_heads=8, head_dim=128, page_size=16,
                budget=4096, window=10, dtype=L.KVC_BF16 | L.KVC_KV4, rope_base=10000.0,
                n_pages=1024, max_pages_per_session=512, max_positions=20000, max_seq_per_call=4,
                max_tokens_per_call=68)
    base.update(kw)
    return L.Config(**base)


def test_pool_size_and_refused_types():
    B.build()
    lib = L.load_library()
    assert L.query_sizes(_cfg())[0] == 1024 * 2 * 8 * 2 * 16 * (64 + 8)
    assert L.query_sizes(_cfg(dtype=L.KVC_F32 | L.KVC_KV4, head_dim=64))[0] == \
        1024 * 2 * 8 * 2 * 16 * (32 + 4)
    for bad in (dict(dtype=0x20), dict(dtype=L.KVC_KV4 | 2), dict(head_dim=64),
                dict(dtype=L.KVC_F32 | L.KVC_KV4), dict(dtype=L.KVC_BF16 | 0x30),
                dict(dtype=L.KVC_BF16 | -0x80), dict(q_heads=16)):
        rc = lib.kvc_query_sizes(ctypes.byref(_cfg(**bad)), None, None)
        assert rc == -1, bad
    # 4-bit rows have no 32-bit row coordinates: only slots are counted in 32 bits.
    assert L.query_sizes(_cfg(n_pages=1 << 23))[0] == (1 << 23) * 2 * 8 * 2 * 16 * 72
    with pytest.raises(L.KvcError):
        L.query_sizes(_cfg(n_pages=1 << 23, dtype=L.KVC_BF16))
    with pytest.raises(L.KvcError):
        L.query_sizes(_cfg(n_pages=1 << 27))
    with pytest.raises(L.KvcError):
        L.query_sizes(_cfg(n_pages=1 << 61))


def test_read_kv_refuses_a_null_context():
    lib = L.load_library()
    assert lib.kvc_read_kv(None, 1, None, None, None, 0, 1, None, None, None, None) == -1


def test_kv_bits_values():
    with pytest.raises(ValueError):
        L.KVCache(n_sessions=1, layers=1, q_heads=4, kv_heads=1, head_dim=64, budget=-1, window=1,
                  dtype="f32", n_pages=4, max_pages_per_session=4, max_positions=64,
                  max_seq_per_call=1, max_tokens_per_call=16, kv_bits=8)


ORDER = r"""
#include "kvc_order.h"
#include <cstdio>

// Launches in stream order.  `complete`: what is surely complete when the next launch can start;
// `flight`: what launches before it write.  Bits 0 and 1: rows of two layers, bit 2: the plan.  A launch
// that waits before it lets others start moves all of `flight` over; one that does not, nothing.
struct Model {
  kvc::LaunchOrder order;
  unsigned complete = 0, flight = 0;
  void wait() {
    complete |= flight;
    flight = 0;
  }
  bool op(int o) {
    if (o < 2) {  // an append with and without rows: lets others start before it has waited
      order.append(o == 0, 2);
      complete = 0;
      flight = o == 0 ? 7 : 4;
      return true;
    }
    const int l = o & 1;
    if (o < 4) {  // a layer's rows: reads the plan's slots early, waits, lets others start
      const bool ok = !order.planned() || (complete & 4);
      wait();
      flight = 1u << l;
      complete &= ~flight;
      order.layer_write(l);
      return ok;
    }
    if (!order.layer_written(l)) return true;  // (refused by the library)
    const kvc::Early e = order.early_pages(l);
    if (e == kvc::EARLY_NONE) wait();
    order.launched_pages(l, e);
    if (e == kvc::EARLY_NONE) return true;
    if (!(complete & 4)) return false;
    return e == kvc::EARLY_OLD || (complete & (1u << l));
  }
};

int main() {
  for (int len = 1; len <= 7; ++len) {
    long n = 1;
    for (int i = 0; i < len; ++i) n *= 6;
    for (long s = 0; s < 2 * n; ++s) {
      Model m;
      m.op(s & 1);
      long x = s / 2;
      for (int i = 0; i < len; ++i, x /= 6)
        if (!m.op((int)(x % 6))) {
          std::printf("sequence %ld of length %d fails at call %d\n", s, len, i);
          return 1;
        }
    }
  }
  // A model's order, layer by layer: every write behind the first finds the plan complete, every attention
  // reads the old pages early.
  kvc::LaunchOrder o;
  o.append(false, 8);
  for (int l = 0; l < 8; ++l) {
    if (o.planned() != (l > 0)) return 2;
    o.layer_write(l);
    const kvc::Early e = o.early_pages(l);
    if (e != kvc::EARLY_OLD) return 3;
    o.launched_pages(l, e);
  }
  return 0;
}
"""


def test_no_early_read_of_a_chunk_in_flight(tmp_path):
    """csrc/kvc_order.h over every short sequence of appends, layer writes and chunked attention."""
    src, exe = tmp_path / "order.cpp", tmp_path / "order"
    src.write_text(ORDER)
    inc = os.path.join(ROOT, "paper_2609_31224_gb300", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", inc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout)


def test_a_bfloat16_cache_in_4_bits_has_no_slots_for_prefill_parts():
    """Its prefill merges within clusters: of the workspace of 16-bit rows, neither the prefill's partial
    rows (512 slots of 128 rows with their maximum and sum) nor the tagged ones of its decode."""
    B.build()
    of = lambda **kw: L.query_sizes(_cfg(**kw))[1]
    prefill, tagged = 512 * 128 * (128 * 4 + 8), 2048 * (4 * 128 + 8) * 8
    assert of(dtype=L.KVC_BF16) - of() == prefill + tagged
    # binary32 in 4 bits keeps them (its slices meet in memory), binary32 has only the tagged ones.
    f32 = dict(head_dim=64)
    assert of(dtype=L.KVC_F32 | L.KVC_KV4, **f32) - of(dtype=L.KVC_F32, **f32) == \
        prefill - 2048 * (4 * 64 + 8) * 8


def test_launches_refuses_null():
    lib = L.load_library()
    out = ctypes.c_int64()
    assert lib.kvc_launches(None, ctypes.byref(out)) == -1 and b"NULL" in lib.kvc_last_error()
