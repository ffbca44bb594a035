// Attention over whole prompts on the 5th-generation tensor cores (tcgen05 + TMEM): bfloat16 K, V and
// q, binary32 softmax and accumulation.
//
// An item is 64 tokens of one session and KV head: two tiles A and B of 32 tokens x G = 4 query heads =
// 128 rows each, against the session's pages up to the last one that its last token sees, 128 keys (8
// pages) a step.  Items go to the CTAs (one per SM) from a counter, a session's last tokens, which see
// most, first; few items have their keys cut into parts (kvc_prompt.cu).  A step has four products of
// 128^3: S_A, S_B (Q K^T) and O_A, O_B += P V; while the softmax of one tile runs, the tensor cores have
// the other tile's.
//
// Work and bound: 4 D flops a query row and key, 2.2 TFLOP for one prompt of 16,384 tokens and 8 KV
// heads; 1,660 to 1,690 us, 1,310 TFLOP/s, 69 % of what the tensor cores were measured to do in a library
// product (figures that steps are compared by here are of one machine, where it took 1,596).  A product instruction takes 77 cycles, 128 columns wide or 64: the 48 of a step, whose scores
// come in halves (below), 3,700 of its 3,800 cycles.  With scores of 128 keys a product they would be 2,470,
// but then the softmax is what a step waits for, 450 cycles and more for 32 keys of a row: measured with P
// of the second half in shared memory, so that the next scores can start early (16,384 tokens 1,608 us,
// 4,099 135 a layer, 250 14.9), and earlier, at 1,811 us, with both halves' scores in one product (1,970 us;
// 16 warps of softmax, two a row, the same).  Code counts as much: the loop of a wait out of line took
// 1,657 us to 1,617; a softmax with one copy of its arithmetic instead of two spills (2,076 us).
// K and V are read once per item, 745 us of copies that run beside.
//
// Shorter prompts are bound by what stands between steps: with the busiest SM's steps and items counted off
// the lists (61, 61 and 872 steps; 3.4, 7.8 and 13.5 items an SM), 4,099 tokens (140 us a layer, 980
// TFLOP/s), eight prompts of up to 2,500 (175 us) and 16,384 tokens come out at 1.7 us a step, some 8 us
// an item and 6 us a launch.  An item has an edge step whose V rows one warp looks through, a last softmax
// and product with nothing beside them, and an output that the softmax warps write before the next
// item's first scores.  Four prompts of up to 700 tokens behind 4,096 positions, 157 us: 72 steps on the
// busiest SM for a mean of 62, since whole items go to the SMs.  One of 250 tokens, 15 to 16 us: 32 items for
// 152 SMs, a launch, an item's set-up, two steps one after the other.
//
// q and P are rounded to bfloat16 once each, as over short chunks (kvc_attn_prefill_tc.cu), since a product of
// bfloat16 K or V takes no wider operand: 2.4e-3 to 2.9e-3 of the outputs' norm, of which their own
// rounding is 1.6e-3.  Two pieces of either would be half as many products again (of 128 x 128 x 128 four a
// step, two of them scores).
//
// Warp roles (512 threads):
//   warp 0      items from the counter; K and V by TMA, a page's 4 KiB of a head a copy (twice as many of
//               2 KiB took 2,600 cycles a step for 1,900), into a ring of four 32 KiB stages in turn
//   warps 1, 2  one thread each issues the products of a tile
//   warp 3      V rows that have to be zero (below)
//   warps 4-7   query rows, rotated, scaled and rounded, into three tiles of shared memory: an item's
//               first one while the item before still runs
//   warps 8-15  softmax, four warps a tile: a thread has one row of S, 32 keys at a time, and writes P over
//               it.  P is taken against a reference 20 above the maximum of the row's first keys, for as long
//               as a sum of 32 stays below 1 (sums and roundings do not depend on the scale, and P <= 1 keeps
//               its products with the largest V finite): later ones look for no maximum, and O is rescaled in
//               tensor memory only when a sum passes that
// A step's keys come in halves, each with scores of its own: while the softmax of one half runs, the
// tensor cores have the other half's O += P V and next scores, so that a row's warp need not wait.
// Tensor memory: S_A, S_B (two halves each, P over the first part of a half), O_A, O_B, 128 columns each:
// all 512.
//
// A key that no row of a product may see has P = 0, but 0 times a value that is not finite is not 0.  So
// the V rows of slots that hold no resident position are zeroed in shared memory, and those of the
// chunk's own tokens that some rows of the item see and others do not, where they are not finite: the
// rows that do see such a one add it by themselves at the end (odd_value).
//
// All waits are bounded; a timeout records KVC_DERR_WAIT and the CTA stops.
#include <cuda.h>

#include <algorithm>
#include <cmath>

#include "kvc_prompt.h"
#include "kvc_prompt_merge.cuh"
#include "kvc_prompt_tc.cuh"

namespace kvc {

namespace {

constexpr int RING = 4, Q_SLOTS = 3;
constexpr int EDGES = 4;
constexpr int TC_THREADS = 512;
constexpr int S_COL = 0, O_COL = 256, ALL_COLS = 512;
constexpr int HALF = KEYS / 2;                     // of a step's keys
constexpr int CHUNK = 32;                          // keys that a row takes at a time
constexpr float ROOM = 20.f;                        // by which a reference lies above the maximum it is taken from
constexpr float SUM_LIMIT = 1.f;                    // of a chunk's P in a row, 2^ROOM times what it starts with
constexpr float NO_KEY = -3.402823466e38f;          // reference of a row whose keys so far all score -infinity
constexpr float ALL_UP = 200.f;                     // a rise of the reference behind which nothing is left of P

enum {
  B_FULL = 0,                    // [RING] a stage has landed
  B_EMPTY = B_FULL + RING,       // [RING] and was read
  B_Q_FULL = B_EMPTY + RING,     // [Q_SLOTS] a tile's query rows are there
  B_Q_EMPTY = B_Q_FULL + Q_SLOTS,  // [Q_SLOTS] and its last scores complete
  // Halves of a step's keys: [2 tiles][2].
  B_S = B_Q_EMPTY + Q_SLOTS,     // scores complete (and every product before them)
  B_P = B_S + 4,                 // P written, O rescaled
  // (A phase of its own, not one more of B_S: the next item's first scores do not wait for the softmax, and
  // a warp that finds two phases complete takes the first for one to come.)
  B_LAST = B_P + 4,              // [2] the last step's first half of O += P V complete
  B_O = B_LAST + 2,              // [2] the item's output complete
  B_O_EMPTY = B_O + 2,           // [2] and read
  // V stages of edge steps land here instead (their B_FULL phase completes at once), and have their
  // rows zeroed: the e-th such stage of the CTA, at e % EDGES.  A ring holds fewer.
  B_EDGE = B_O_EMPTY + 2,        // [EDGES]
  B_FIX = B_EDGE + EDGES,        // [EDGES]
  B_ITEM = B_FIX + EDGES,        // [2] an item is known
  B_ITEM_EMPTY = B_ITEM + 2,     // [2] and every warp is through with it
  B_FINAL = B_ITEM_EMPTY + 2,    // every product of the CTA complete
  N_BARS = B_FINAL + 1
};
constexpr int ITEM_READERS = 2 + 1 + 4 + 8;        // warps that arrive at B_ITEM_EMPTY

// What every role knows of an item.
struct Item {
  SeqInfo si;
  int32_t head, t0, steps;       // steps = 0: no more items
  int32_t odd;                   // some V row was zeroed because it is not finite
  int32_t first;                 // step that it starts with
  int32_t slot;                  // of its first tile's part, -1: the item has all keys
  int32_t pad[10];
};
static_assert(sizeof(Item) == 128, "Item size");

constexpr int OFF_BARS = 0;
constexpr int OFF_ITEM = 512;                      // [2]
constexpr int OFF_TMEM = OFF_ITEM + 2 * 128;
constexpr int OFF_STOP = OFF_TMEM + 4;
constexpr int OFF_GROUP = OFF_STOP + 4;            // the work list
constexpr int OFF_TILES = 3 * 1024;                // query tiles, then the ring
constexpr int SMEM_BYTES = OFF_TILES + (Q_SLOTS + RING) * SLOT;
static_assert(N_BARS * 8 <= OFF_ITEM && OFF_GROUP + (GROUPS + 1) * 4 <= OFF_TILES, "header fits");
static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of a CTA");

// Page of block b of a session with nhp compacted pages.
__device__ inline int page_of(const Dev& d, int sid, int nhp, int b) {
  const size_t row = (size_t)sid * d.max_pages_per_session;
  return b < nhp ? d.hist_pt[row + b] : d.live_pt[row + b - nhp];
}

// Steps [*j0, *j1) of a part of an item's keys, of `all`.  Each part but an empty one starts with keys that
// all rows of the item see (its first token, on which the rest of the rows follow, is in step `diag`).
__device__ inline void part_steps(int all, int diag, int part, int parts, int* j0, int* j1) {
  *j0 = min(all * part / parts, diag);
  *j1 = part == parts - 1 ? all : min(all * (part + 1) / parts, diag);
}

__device__ inline bool not_finite(uint32_t two) {
  return (two & 0x7F80u) == 0x7F80u || (two & 0x7F800000u) == 0x7F800000u;
}

// What a row draws of the V rows that were zeroed because they are not finite (rare: slow and
// simple), dims [c0, c0 + 32), unnormalised.  Keys behind the item's first token up to the row's own.
__device__ __noinline__ void odd_value(const Dev& d, const SeqInfo& si, int layer, int head, int t0, int tok,
                                       int g, const __nv_bfloat16* q, float qk_scale, float m, int c0,
                                       float* o) {
  const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
  const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
  const __nv_bfloat16* pool = reinterpret_cast<const __nv_bfloat16*>(d.pool);
  const __nv_bfloat16* row = q + ((size_t)(si.q_row0 + tok) * d.q_heads + head * G + g) * D;
  const float2* cs = d.rope + (size_t)(si.pos_first + tok) * (D / 2);
  for (int i = 0; i < 32; ++i) o[i] = 0.f;
  for (int key = t0 + 1; key <= tok; ++key) {
    const int slot = si.live_head + si.n_live - si.t + key;
    const int page = block_page(si, hrow, lrow, si.n_hist_pages + slot / PS);
    const __nv_bfloat16* v = pool + pool_offset_elems(d, page, layer, 1, head, slot % PS);
    bool odd = false;
    for (int i = 0; i < D / 2; ++i) odd |= not_finite(reinterpret_cast<const uint32_t*>(v)[i]);
    if (!odd) continue;
    const __nv_bfloat16* k = pool + pool_offset_elems(d, page, layer, 0, head, slot % PS);
    float s = 0.f;
    for (int i = 0; i < D / 2; ++i) {
      float a, b;
      rope_pair(__bfloat162float(row[i]), __bfloat162float(row[i + D / 2]), cs[i], a, b);
      s = fmaf(__bfloat162float(__float2bfloat16_rn(a * qk_scale)), __bfloat162float(k[i]), s);
      s = fmaf(__bfloat162float(__float2bfloat16_rn(b * qk_scale)), __bfloat162float(k[i + D / 2]), s);
    }
    const float p = __bfloat162float(__float2bfloat16_rn(exp2f(s - m)));
    for (int i = 0; i < 32; ++i) o[i] = fmaf(p, __bfloat162float(v[c0 + i]), o[i]);
  }
}

__global__ void __launch_bounds__(TC_THREADS, 1) prompt_tc_kernel(
    Dev d, int layer, const __grid_constant__ CUtensorMap map,
    const __nv_bfloat16* __restrict__ q,
    __nv_bfloat16* __restrict__ out, float qk_scale, int most_parts) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + OFF_BARS);
  Item* items = reinterpret_cast<Item*>(smem + OFF_ITEM);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_TMEM);
  int* s_group = reinterpret_cast<int*>(smem + OFF_GROUP);
  volatile int* stop = reinterpret_cast<int*>(smem + OFF_STOP);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int H = d.kv_heads;
  uint8_t* s_q = smem + OFF_TILES;
  uint8_t* s_ring = s_q + Q_SLOTS * SLOT;
  pdl_wait();
  pdl_launch_dependents();
  const int n_seq = d.g->total_tokens > 0 ? d.g->n_seq : 0;  // (no tokens: the append failed)
  if (tid < N_BARS) {  // (by one thread they took 2.5 us of a short prompt's 17.5)
    const int count = (tid >= B_EMPTY && tid < B_Q_FULL) || tid == B_FINAL ? 2
                      : tid >= B_Q_FULL && tid < B_Q_EMPTY                 ? 4
                      : tid >= B_P && tid < B_LAST                         ? 4
                      : tid >= B_O_EMPTY && tid < B_EDGE                   ? 4
                      : tid >= B_ITEM_EMPTY && tid < B_FINAL               ? ITEM_READERS
                                                                           : 1;
    mbar_init(&bars[tid], count);
    fence_mbar_init();
  }
  if (tid == 0) *stop = 0;
  // Items of a session: 64-token tiles of its chunk, for each KV head (and parts of their keys).
  auto items_of = [&](int i) { return (d.seq[i].t + 2 * TOKENS - 1) / (2 * TOKENS) * H; };
  if (warp == 3) list_items(n_seq, lane, s_group, items_of);
  __syncwarp();
  if (warp == 1) tmem_alloc(tmem_slot, ALL_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp < 4) {
    if (warp == 0) {
      // ---------------- items, K and V ----------------
      const int parts = parts_now(d, most_parts, s_group[GROUPS]), total = s_group[GROUPS] * parts;
      uint32_t seq_no = 0, edges = 0;  // stages so far, and V stages of edge steps
      bool ok = true;
      auto wait = [&](int bar, uint32_t parity) {
        ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
        return ok;
      };
      // The next item, taken from the counter and looked up while the stages of the one before are on
      // their way.  (word: lane i has word i of its session's info.)
      int word, sid, nhp, head, t0, nb, first, slot, steps, pid, pid_next;
      EdgeSteps edge;
      auto fetch = [&] {
        for (steps = 0; steps == 0;) {
          int at = 0, in;
          if (lane == 0) at = take_item(d);
          at = __shfl_sync(FULL, at, 0);
          if (at >= total) return;
          const int seq = find_item(n_seq, lane, s_group, at / parts, items_of, &in), part = at % parts;
          word = lane < 16 ? reinterpret_cast<const int*>(d.seq + seq)[lane] : 0;
          const SeqInfo& si = d.seq[seq];
          sid = si.sid;
          nhp = si.n_hist_pages;
          head = in % H;
          t0 = ((si.t + 2 * TOKENS - 1) / (2 * TOKENS) - 1 - in / H) * 2 * TOKENS;
          nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1);
          edge = edge_steps(si, t0);
          part_steps((nb + PAGES - 1) / PAGES, edge.diag, part, parts, &first, &steps);
          steps -= first;
          edge.from(first);
          slot = parts > 1 ? 2 * at : -1;
        }
        auto page_at = [&](int b) { return b < nb ? page_of(d, sid, nhp, b) : 0; };
        pid = page_at(PAGES * first + lane);
        pid_next = page_at(PAGES * first + 32 + lane);
      };
      auto publish = [&](int n) {
        Item* it = items + (n & 1);
        if (lane < 16) reinterpret_cast<int*>(&it->si)[lane] = word;
        if (lane == 0) {
          it->head = head;
          it->t0 = t0;
          it->steps = steps;
          it->odd = 0;
          it->first = first;
          it->slot = slot;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_ITEM + (n & 1)]);
      };
      fetch();
      publish(0);
      for (int n = 0; ok && steps > 0; ++n) {
        const int c_sid = sid, c_nhp = nhp, c_head = head, c_nb = nb, c_steps = steps, c_first = first;
        const EdgeSteps c_edge = edge;
        int c_pid = pid, c_pid_next = pid_next;
        const int next_bar = B_ITEM_EMPTY + ((n + 1) & 1);
        const uint32_t next_parity = (((n + 1) >> 1) & 1) ^ 1;
        bool published = false;
        for (int j = 0; j < c_steps && ok; ++j) {
          if (j > 0 && (j & 3) == 0) {
            c_pid = c_pid_next;
            const int b = PAGES * (c_first + j) + 32 + lane;
            c_pid_next = b < c_nb ? page_of(d, c_sid, c_nhp, b) : 0;
          }
          const int page = __shfl_sync(FULL, c_pid, PAGES * (j & 3) + (lane & 7));
          const int n_pg = min(PAGES, c_nb - PAGES * (c_first + j));
#pragma unroll
          for (int kv = 0; kv < 2; ++kv, ++seq_no) {
            const int st = seq_no % RING;
            if (seq_no >= RING && !wait(B_EMPTY + st, ((seq_no / RING) & 1) ^ 1)) break;
            uint64_t* bar = &bars[B_FULL + st];
            if (kv == 1 && c_edge.at(j)) {
              if (lane == 0) mbar_arrive(bar);
              bar = &bars[B_EDGE + edges % EDGES];
              ++edges;
            }
            if (lane == 0) mbar_arrive_expect_tx(bar, n_pg * PS * D * 2);
            __syncwarp();
            load_tile(d, layer, kv, c_head, page, n_pg, s_ring + st * SLOT, &map, bar, lane);
          }
          if (j == min(1, c_steps - 1)) fetch();
          if (j >= 1 && !published && (n == 0 || __all_sync(FULL, mbar_test(&bars[next_bar], next_parity)))) {
            publish(n + 1);
            published = true;
          }
        }
        if (!published) {
          if (n > 0 && !wait(next_bar, next_parity)) break;
          publish(n + 1);
        }
      }
      // Copies still in flight land before the CTA ends.
      for (uint32_t s = seq_no > RING ? seq_no - RING : 0; s < seq_no; ++s)
        mbar_wait(d, &bars[B_FULL + s % RING], (s / RING) & 1);
      for (uint32_t e = edges > EDGES ? edges - EDGES : 0; e < edges; ++e)
        mbar_wait(d, &bars[B_EDGE + e % EDGES], (e / EDGES) & 1);
    } else if (warp < 3 && lane == 0) {
      // ---------------- products: one thread a tile ----------------
      constexpr uint32_t ID_S = instr_desc(HALF, M, false), ID_O = instr_desc(D, M, true);
      const int x = warp - 1;
      const uint32_t t_s = tmem + S_COL + x * KEYS, t_o = tmem + O_COL + x * D;
      const uint64_t qd0 = desc_columns(smem_u32(s_q));
      const uint64_t kd0 = desc_columns(smem_u32(s_ring)), vd0 = desc_rows(smem_u32(s_ring));
      bool ok = true;
      auto wait = [&](int bar, uint32_t parity) {
        ok = ok && wait_or_stop(d, &bars[bar], parity, stop);
        return ok;
      };
      // Stages are counted on: `st` is the ring's slot of the next one, `pass` its pass over the ring.
      int st = 0, q_slot = 0;
      uint32_t pass = 0, edges = 0, p_no = 0, o_no = 0;
      uint32_t q_no = 0;  // query tiles of the items before
      auto full = [&] { return wait(B_FULL + st, pass & 1); };
      auto next = [&] {
        if (++st == RING) {
          st = 0;
          ++pass;
        }
      };
      // S = Q K^T of half h of the stage at `st`, which has landed.
      auto scores = [&](int h) {
        tc_fence_after();
        const uint64_t kd = desc_at(kd0, st * SLOT + h * (HALF / 8) * ROW_GROUP), qd = desc_at(qd0, q_slot * SLOT);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          tc_mma_ss(t_s + h * HALF, desc_at(qd, step_columns(kk)), desc_at(kd, step_columns(kk)), ID_S, kk > 0);
      };
      // An item's first scores.
      auto begin = [&](const Item& it, bool mine) {
        if (!full()) return;
        if (mine) {
          q_slot = (q_no + x) % Q_SLOTS;
          if (!wait(B_Q_FULL + q_slot, ((q_no + x) / Q_SLOTS) & 1)) return;
          scores(0);
          tc_commit(&bars[B_S + 2 * x]);
          scores(1);
          tc_commit(&bars[B_S + 2 * x + 1]);
          if (it.steps == 1) tc_commit(&bars[B_Q_EMPTY + q_slot]);
          tc_commit(&bars[B_EMPTY + st]);
        } else {
          mbar_arrive(&bars[B_EMPTY + st]);
        }
        next();
      };
      auto tiles_of = [](const Item& it) { return it.t0 + TOKENS < it.si.t ? 2 : 1; };
      if (wait(B_ITEM, 0)) {
        int steps = items[0].steps, tiles = steps > 0 ? tiles_of(items[0]) : 0;
        if (steps > 0) begin(items[0], x < tiles);
        for (int n = 0; ok && steps > 0; ++n) {
          const Item& it = items[n & 1];
          EdgeSteps edge = edge_steps(it.si, it.t0);
          edge.from(it.first);
          const bool mine = x < tiles;
          q_no += tiles;
          for (int j = 0; j < steps && ok; ++j) {
            // What is there early is waited for first: V, then the next step's K.
            const bool last = j == steps - 1;
            const int sv = st;
            if (!full()) break;
            next();
            if (!last && !full()) break;
            if (edge.at(j)) {
              if (mine && !wait(B_FIX + edges % EDGES, (edges / EDGES) & 1)) break;
              ++edges;
            }
            if (mine) {
              if (j == 0 && o_no++ > 0 && !wait(B_O_EMPTY + x, (o_no - 2) & 1)) break;
              const uint64_t vd = desc_at(vd0, sv * SLOT);
#pragma unroll 1
              for (int h = 0; h < 2; ++h) {
                if (!wait(B_P + 2 * x + h, p_no & 1)) break;
                tc_fence_after();
#pragma unroll
                for (int kk = 0; kk < HALF / 16; ++kk)
                  tc_mma_ts(t_o, t_s + h * HALF + kk * 8, desc_at(vd, (h * (HALF / 16) + kk) * 2 * ROW_GROUP), ID_O,
                            j > 0 || h > 0 || kk > 0);
                if (!last) scores(h);
                tc_commit(&bars[!last ? B_S + 2 * x + h : h == 0 ? B_LAST + x : B_O + x]);
              }
              ++p_no;
              if (j + 2 == steps) tc_commit(&bars[B_Q_EMPTY + q_slot]);
              tc_commit(&bars[B_EMPTY + sv]);
              if (!last) tc_commit(&bars[B_EMPTY + st]);
            } else {
              mbar_arrive(&bars[B_EMPTY + sv]);
              if (!last) mbar_arrive(&bars[B_EMPTY + st]);
            }
            if (!last) next();
          }
          // The next item's first scores go ahead of this one's output.
          if (!wait(B_ITEM + ((n + 1) & 1), ((n + 1) >> 1) & 1)) break;
          const Item& nx = items[(n + 1) & 1];
          steps = nx.steps;
          tiles = steps > 0 ? tiles_of(nx) : 0;
          if (steps > 0) begin(nx, x < tiles);
          mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
        }
      }
      // No product may still be running when the tensor memory is released.
      tc_commit(&bars[B_FINAL]);
      mbar_wait(d, &bars[B_FINAL], 0);
    } else if (warp == 3) {
      // ---------------- V rows to zero ----------------
      bool ok = true;
      auto wait = [&](int bar, uint32_t parity) {
        ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
        return ok;
      };
      uint32_t stages = 0, edges = 0;
      for (int n = 0; ok; ++n) {
        if (!wait(B_ITEM + (n & 1), (n >> 1) & 1)) break;
        Item& it = items[n & 1];
        if (it.steps == 0) break;
        const SeqInfo& si = it.si;
        const int t0 = it.t0, steps = it.steps, q_log0 = si.n_hist + si.n_live - si.t;
        const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1);
        EdgeSteps edge = edge_steps(si, t0);
        edge.from(it.first);
        for (int j = 0; j < steps && ok; ++j) {
          if (!edge.at(j)) continue;
          uint8_t* tile = s_ring + (stages + 2 * j + 1) % RING * SLOT;
          if (!wait(B_EDGE + edges % EDGES, (edges / EDGES) & 1)) break;
#pragma unroll 1
          for (int r = lane; r < KEYS; r += 32) {
            const int b = PAGES * (it.first + j) + r / PS;
            const uint32_t bit = 1u << (r % PS);
            bool zero = !(slots_seen(si, b, nb, q_log0 + si.t) & bit);
            if (!zero && !(slots_seen(si, b, nb, q_log0 + t0) & bit)) {  // some rows see it
              bool odd = false;
#pragma unroll 4
              for (int i = 0; i < 16; ++i) {
                const uint4 v = *reinterpret_cast<const uint4*>(tile + tile_at(r, i));
                odd |= not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w);
              }
              if (odd) {
                it.odd = 1;
                zero = true;
              }
            }
            if (zero)
              for (int i = 0; i < 16; ++i)
                *reinterpret_cast<uint4*>(tile + tile_at(r, i)) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[B_FIX + edges % EDGES]);
          ++edges;
        }
        stages += 2 * steps;
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
      }
    }
  } else if (warp < 8) {
    // ---------------- query rows ----------------
    const int ts = tid - 4 * 32;
    bool ok = true;
    auto wait = [&](int bar, uint32_t parity) {
      ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
      return ok;
    };
    uint32_t q_no = 0;
    for (int n = 0; ok; ++n) {
      if (!wait(B_ITEM + (n & 1), (n >> 1) & 1)) break;
      const Item& it = items[n & 1];
      if (it.steps == 0) break;
      const int tiles = it.t0 + TOKENS < it.si.t ? 2 : 1;
      for (int x = 0; x < tiles; ++x, ++q_no) {
        const int slot = q_no % Q_SLOTS;
        stage_q<1, 128>(d, it.si, it.head, it.t0 + x * TOKENS, q, qk_scale, s_q + slot * SLOT, ts,
                      [&] { return q_no < Q_SLOTS || wait(B_Q_EMPTY + slot, ((q_no / Q_SLOTS) & 1) ^ 1); });
        if (!ok) break;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_Q_FULL + slot]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
    }
  } else {
    // ---------------- softmax ----------------
    // (Loops stay rolled: with a step's 128 keys in one piece the code of all roles did not fit the
    // instruction caches, and a warp was without an instruction for as long as it issued one.)
    const int x = (warp - 8) >> 2;             // tile
    const int r = (warp & 3) * 32 + lane;      // row
    const uint32_t trow = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t t_s = trow + S_COL + x * KEYS, t_o = trow + O_COL + x * D;
    bool ok = true;
    auto wait = [&](int bar, uint32_t parity) {
      ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
      return ok;
    };
    uint32_t s0_no = 0, s1_no = 0, o_no = 0;  // phases of the halves' scores so far, and of outputs
    for (int n = 0; ok; ++n) {
      if (!wait(B_ITEM + (n & 1), (n >> 1) & 1)) break;
      const Item& it = items[n & 1];
      const int steps = it.steps;
      if (steps == 0) break;
      const SeqInfo& si = it.si;
      const int t0 = it.t0, tok = t0 + x * TOKENS + r / G;
      if (t0 + x * TOKENS < si.t) {
        const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1);
        const int q_log = si.n_hist + si.n_live - si.t + tok;
        EdgeSteps edge = edge_steps(si, t0);
        edge.from(it.first);
        float m = 0.f, l = 0.f;
        for (int j = 0; ok && j < steps; ++j) {
          const bool masks = edge.at(j);
          float add = 0.f;  // the step's part of l
          // Chunk c of the row's scores: P = 2^(s - m) over what was read of S already.
          auto weigh = [&](int c, uint32_t (&w)[CHUNK]) {
            if (masks) {
#pragma unroll
              for (int p = 0; p < CHUNK / PS; ++p) {
                const uint32_t seen = slots_seen(si, PAGES * (it.first + j) + CHUNK / PS * c + p, nb, q_log);
#pragma unroll
                for (int i = 0; i < PS; ++i) w[p * PS + i] = (seen >> i & 1) ? w[p * PS + i] : 0xFF800000u;
              }
            }
            auto most = [&] {  // a reference for these keys
              float a[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) a[i] = __uint_as_float(w[i]);
#pragma unroll
              for (int i = 4; i < CHUNK; i += 4)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] = fmaxf(a[k], __uint_as_float(w[i + k]));
              return fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])) + ROOM;
            };
            uint32_t pw[CHUNK / 2];
            auto sum_of = [&] {
              const float2 nref = make_float2(-m, -m);
              float2 rs[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
              for (int i = 0; i < CHUNK; i += 2) {
                const float2 y = __fadd2_rn(make_float2(__uint_as_float(w[i]), __uint_as_float(w[i + 1])), nref);
                const float2 p = make_float2(ex2(y.x), ex2(y.y));
                rs[(i / 2) & 1] = __fadd2_rn(rs[(i / 2) & 1], p);
                pw[i / 2] = pack_bf16(p.x, p.y);
              }
              const float2 r2 = __fadd2_rn(rs[0], rs[1]);
              return r2.x + r2.y;
            };
            // The reference goes by the maximum of the row's first chunk (which holds position 0 of what is
            // resident, so that each row sees a key of it), until a sum passes the limit (or is NaN):
            // then it rises by a whole number, so that what was written of P scales exactly.  O may be
            // rescaled behind the last O += P V: the other half's scores come after it, of the same step
            // behind the second half's of the step before, of the next one behind the first half's.
            // A first chunk all at -infinity leaves a finite reference, under which every other score's P is
            // infinite, and -infinity's 0.
            if (j == 0 && c == 0) m = fmaxf(most(), NO_KEY);
            float sum = sum_of();
            if (!__all_sync(FULL, sum < SUM_LIMIT)) {
              const float top = most(), up = fmaxf(ceilf(top - m), 0.f), f = exp2f(-up);
              l *= f;
              add *= f;
              const int h = c / 2;
              const bool end = h == 1 && j == steps - 1;
              wait(end ? B_LAST + x : B_S + 2 * x + (h ^ 1), (end ? o_no : h == 0 ? s1_no : s0_no) & 1);
              tc_fence_after();
              tmem_st_wait();
#pragma unroll 1
              for (int k = 0; (j > 0 || h > 0) && k < D; k += 16) {
                float o[16];
                tmem_ld16(t_o + k, o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] *= f;
                tmem_st16(t_o + k, o);
              }
#pragma unroll 1
              for (int k = 0; k < (c & 1); ++k) {
                float o[16];
                uint32_t to[16];
                tmem_ld16(t_s + h * HALF, o);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  to[i] = pack_bf16(bf16lo(__float_as_uint(o[i])) * f, bf16hi(__float_as_uint(o[i])) * f);
                tmem_st16(t_s + h * HALF, to);
              }
              m = up > ALL_UP ? top : m + up;  // (far scores have no whole numbers between them)
              sum = sum_of();
            }
            add += sum;
            __syncwarp();
            tmem_st16_begin(t_s + (c >> 1) * HALF + 16 * (c & 1), pw);
          };
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            if (!wait(B_S + 2 * x + h, (h == 0 ? s0_no++ : s1_no++) & 1)) break;
            tc_fence_after();
            uint32_t wa[CHUNK], wb[CHUNK];
            tmem_ld32_begin(t_s + h * HALF, wa);
            tmem_ld32_begin(t_s + h * HALF + CHUNK, wb);
            tmem_ld32_wait(wa);
            tmem_ld32_wait(wb);
            weigh(2 * h, wa);
            weigh(2 * h + 1, wb);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars[B_P + 2 * x + h]);
          }
          l += add;
        }
        if (!ok || !wait(B_O + x, o_no & 1)) break;  // (B_LAST's phase is complete then, too)
        ++o_no;
        tc_fence_after();
        const float inv = 1.f / l;
        const int slot = it.slot + x;
        const bool partly = it.slot >= 0;
        if (partly) part_sums<D>(d, slot)[r] = make_float2(m, l);
        const bool odd = *reinterpret_cast<volatile const int*>(&it.odd) != 0;
        __nv_bfloat16* row = out + ((size_t)(si.q_row0 + tok) * d.q_heads + it.head * G + r % G) * D;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          tmem_ld32(t_o + c, o);
          if (odd && tok < si.t) {
            float more[32];
            odd_value(d, si, layer, it.head, t0, tok, r % G, q, qk_scale, m, c, more);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] += more[i];
          }
          if (partly) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              part_rows<D>(d, slot)[(c + i) / 4 * PART_ROWS + r] =
                  make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          } else if (tok < si.t) {
#pragma unroll
            for (int i = 0; i < 32; i += 8)
              *reinterpret_cast<uint4*>(row + c + i) =
                  make_uint4(pack_bf16(o[i] * inv, o[i + 1] * inv), pack_bf16(o[i + 2] * inv, o[i + 3] * inv),
                             pack_bf16(o[i + 4] * inv, o[i + 5] * inv), pack_bf16(o[i + 6] * inv, o[i + 7] * inv));
          }
          __syncwarp();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_O_EMPTY + x]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, ALL_COLS);
  if (tid == 0) leave_counters(d);
}

__global__ void __launch_bounds__(MERGE_THREADS) prompt_merge_kernel(Dev d, __nv_bfloat16* out, int most_parts) {
  merge_parts<__nv_bfloat16, D, 2>(d, out, most_parts, [](const SeqInfo& si, int t0, int part, int parts) {
    const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1);
    int j0, j1;
    part_steps((nb + PAGES - 1) / PAGES, edge_steps(si, t0).diag, part, parts, &j0, &j1);
    return j0 == j1;
  });
}

}  // namespace

cudaError_t prompt_tc_attributes() {
  return cudaFuncSetAttribute(prompt_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              SMEM_BYTES);
}

cudaError_t launch_prompt_tc(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int parts,
                             int64_t items, cudaStream_t s, int64_t* launches) {
  CUtensorMap map;
  if (!pool_tile_map(d, &map)) return cudaErrorInvalidValue;
  __nv_bfloat16* to = static_cast<__nv_bfloat16*>(out);
  cudaError_t e = launch_ex(&prompt_tc_kernel, dim3(lim.sms), dim3(TC_THREADS), SMEM_BYTES, s, true, d, layer,
                            map, static_cast<const __nv_bfloat16*>(q), to, LOG2E / sqrtf((float)D), parts);
  *launches += e == cudaSuccess;
  if (e != cudaSuccess || parts == 1) return e;
  e = launch_ex(&prompt_merge_kernel, dim3(merge_grid(2 * items, D)), dim3(MERGE_THREADS), 0, s, true, d, to,
                parts);
  *launches += e == cudaSuccess;
  return e;
}

}  // namespace kvc
