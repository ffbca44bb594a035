// Attention over whole prompts on the 5th-generation tensor cores (tcgen05 + TMEM): bfloat16 K, V and
// q, binary32 softmax and accumulation.
//
// An item is 64 tokens of one session and KV head: two tiles A and B of 32 tokens x G = 4 query heads =
// 128 rows each, against the session's pages up to the last one that its last token sees, 128 keys (8
// pages) a step.  Items go to the CTAs (one per SM) from a counter, a session's last tokens, which see
// most, first.  A step has four products of 128^3: S_A, S_B (Q K^T) and O_A, O_B += P V; while the
// softmax of one tile runs, the tensor cores have the other tile's.
// Warp roles (512 threads):
//   warp 0      items from the counter; K and V by TMA, a page's 4 KiB of a head a copy (twice as many of
//               2 KiB took 2,600 cycles a step for 1,900), into a ring of five 32 KiB stages in turn
//   warps 1, 2  one thread each issues the products of a tile
//   warps 4-7   query rows, rotated, scaled and rounded, into shared memory, the next item's as soon as
//               this one's last score product of the tile is complete; V rows that have to be zero (below)
//   warps 8-15  softmax, four warps a tile: a thread has one row of S, from tensor memory to registers in
//               one go, and writes P over it.  P is taken against the maximum of the row's first step,
//               for as long as a step's sum stays below 2^20 (sums and roundings do not depend on the
//               scale): later steps look for no maximum, and O is rescaled in tensor memory only
//               when a sum passes that
// Tensor memory: S_A, S_B (P over the first half of each), O_A, O_B, 128 columns each: all 512.
//
// A key that no row of a product may see has P = 0, but 0 times a value that is not finite is not 0.  So
// the V rows of slots that hold no resident position are zeroed in shared memory, and those of the
// chunk's own tokens that some rows of the item see and others do not, where they are not finite: the
// rows that do see such a one add it by themselves at the end (add_odd_values).
//
// All waits are bounded; a timeout records KVC_DERR_WAIT and the CTA stops.
#include <cuda.h>

#include <cmath>

#include "kvc_prompt.h"
#include "kvc_prompt_tc.cuh"

namespace kvc {

namespace {

constexpr int RING = 5;
constexpr int EDGES = 4;
constexpr int HALF = KEYS / 2;                     // of a step's keys, and of a row's dims
// 24 warps, 80 registers a thread at launch: issuing and query warps give some to the softmax.
constexpr int TC_THREADS = 768, BASE_REGS = 80, FEW_REGS = 64, MANY_REGS = 88;
static_assert(256 * FEW_REGS + 512 * MANY_REGS <= TC_THREADS * BASE_REGS, "registers of the launch");
constexpr int S_COL = 0, O_COL = 256, ALL_COLS = 512;
constexpr float SUM_LIMIT = 1048576.f;              // of a step's P in a row: 2^20

enum {
  B_FULL = 0,                    // [RING] a stage has landed
  B_EMPTY = B_FULL + RING,       // [RING] and was read
  B_Q_FULL = B_EMPTY + RING,     // [2] a tile's query rows are there
  B_Q_EMPTY = B_Q_FULL + 2,      // [2] and its last scores of the item complete
  B_S = B_Q_EMPTY + 2,           // [2] scores complete (and every product before them)
  B_P = B_S + 2,                 // [2] P written, O rescaled
  B_O = B_P + 2,                 // [2] the item's output complete
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
constexpr int ITEM_READERS = 2 + 4 + 16;           // warps that arrive at B_ITEM_EMPTY

// What every role knows of an item.
struct Item {
  SeqInfo si;
  int32_t seq, head, t0, steps;  // steps = 0: no more items
  int32_t odd;                   // some V row was zeroed because it is not finite
  int32_t pad[11];
};
static_assert(sizeof(Item) == 128, "Item size");

constexpr int OFF_BARS = 0;
constexpr int OFF_ITEM = 512;                      // [2]
constexpr int OFF_TMEM = OFF_ITEM + 2 * 128;
constexpr int OFF_STOP = OFF_TMEM + 4;
constexpr int OFF_GROUP = OFF_STOP + 4;            // the work list
constexpr int OFF_HALF = OFF_GROUP + 136;          // [2 tiles][2 halves][M] what halves of a row exchange
constexpr int OFF_TILES = 3072;                    // query tiles A, B, then the ring
constexpr int SMEM_BYTES = OFF_TILES + (2 + RING) * SLOT;
static_assert(N_BARS * 8 <= OFF_ITEM && (GROUPS + 1) * 4 <= 136 && OFF_HALF + 4 * M * 4 <= OFF_TILES,
              "header fits");
static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of a CTA");

// Barrier of the two warps that share rows: whether `say` holds in any of their threads.
__device__ inline bool meet_any(int id, bool say) {
  int any;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.s32 p, %2, 0;\n\t"
      "barrier.cta.red.or.pred.aligned q, %1, 64, p;\n\t"
      "selp.s32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"(id), "r"((int)say)
      : "memory");
  return any != 0;
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
    __nv_bfloat16* __restrict__ out, float qk_scale) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + OFF_BARS);
  Item* items = reinterpret_cast<Item*>(smem + OFF_ITEM);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_TMEM);
  int* s_group = reinterpret_cast<int*>(smem + OFF_GROUP);
  volatile int* stop = reinterpret_cast<int*>(smem + OFF_STOP);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int H = d.kv_heads;
  uint8_t* s_q = smem + OFF_TILES;
  uint8_t* s_ring = s_q + 2 * SLOT;
  pdl_wait();
  pdl_launch_dependents();
  const int n_seq = d.g->n_units > 0 ? d.g->n_seq : 0;  // (no units: the append failed)
  if (tid == 0) {
    for (int i = 0; i < N_BARS; ++i) {
      const int count = i >= B_EMPTY && i < B_Q_FULL || i == B_FINAL ? 2
                        : i >= B_Q_FULL && i < B_Q_EMPTY             ? 4
                        : i >= B_P && i < B_O          ? 8
                        : i >= B_O_EMPTY && i < B_EDGE ? 8
                        : i >= B_FIX && i < B_ITEM     ? 4
                        : i >= B_ITEM_EMPTY && i < B_FINAL ? ITEM_READERS
                                                           : 1;
      mbar_init(&bars[i], count);
    }
    fence_mbar_init();
    *stop = 0;
  }
  // Items of a session: 64-token tiles of its chunk, for each KV head.
  auto items_of = [&](int i) { return (d.seq[i].t + 2 * TOKENS - 1) / (2 * TOKENS) * H; };
  if (warp == 3) list_items(n_seq, lane, s_group, items_of);
  __syncwarp();
  if (warp == 1) tmem_alloc(tmem_slot, ALL_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp < 4) {
    set_registers<BASE_REGS, FEW_REGS>();
  if (warp == 0) {
    // ---------------- items, K and V ----------------
    const int total = s_group[GROUPS];
    uint32_t seq_no = 0, edges = 0;  // stages so far, and V stages of edge steps
    bool ok = true;
    for (int n = 0; ok; ++n) {
      Item* it = items + (n & 1);
      if (n >= 2) ok = __all_sync(FULL, wait_or_stop(d, &bars[B_ITEM_EMPTY + (n & 1)], ((n >> 1) & 1) ^ 1, stop));
      if (!ok) break;
      int at = 0;
      if (lane == 0) at = atomicAdd(&d.pf_count[0], 1);
      at = __shfl_sync(FULL, at, 0);
      if (at >= total) {
        if (lane == 0) {
          it->steps = 0;
          mbar_arrive(&bars[B_ITEM + (n & 1)]);
        }
        break;
      }
      int in;
      const int seq = find_item(n_seq, lane, s_group, at, items_of, &in);
      if (lane < 16)
        reinterpret_cast<int*>(&it->si)[lane] = reinterpret_cast<const int*>(d.seq + seq)[lane];
      __syncwarp();
      const SeqInfo& si = it->si;
      const int n_t = (si.t + 2 * TOKENS - 1) / (2 * TOKENS), head = in % H;
      const int t0 = (n_t - 1 - in / H) * 2 * TOKENS;
      const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1), steps = (nb + PAGES - 1) / PAGES;
      if (lane == 0) {
        it->seq = seq;
        it->head = head;
        it->t0 = t0;
        it->steps = steps;
        it->odd = 0;
        mbar_arrive(&bars[B_ITEM + (n & 1)]);
      }
      const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
      const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
      auto page_at = [&](int b) { return b < nb ? block_page(si, hrow, lrow, b) : 0; };
      const EdgeSteps edge = edge_steps(si, t0);
      int pid = page_at(lane), pid_next = page_at(32 + lane);
      for (int j = 0; j < steps && ok; ++j) {
        if (j > 0 && (j & 3) == 0) {
          pid = pid_next;
          pid_next = page_at(PAGES * j + 32 + lane);
        }
        const int page = __shfl_sync(FULL, pid, PAGES * (j & 3) + (lane & 7));
        const int n_pg = min(PAGES, nb - PAGES * j);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++seq_no) {
          const int st = seq_no % RING;
          if (seq_no >= RING) {
            ok = __all_sync(FULL, wait_or_stop(d, &bars[B_EMPTY + st], ((seq_no / RING) & 1) ^ 1, stop));
            if (!ok) break;
          }
          uint64_t* bar = &bars[B_FULL + st];
          if (kv == 1 && edge.at(j)) {
            if (lane == 0) mbar_arrive(bar);
            bar = &bars[B_EDGE + edges % EDGES];
            ++edges;
          }
          if (lane == 0) mbar_arrive_expect_tx(bar, n_pg * PS * D * 2);
          __syncwarp();
          load_tile(d, layer, kv, head, page, n_pg, s_ring + st * SLOT, &map, bar, lane);
        }
      }
    }
    // Copies still in flight land before the CTA ends.
    for (uint32_t s = seq_no > RING ? seq_no - RING : 0; s < seq_no; ++s)
      mbar_wait(d, &bars[B_FULL + s % RING], (s / RING) & 1);
    for (uint32_t e = edges > EDGES ? edges - EDGES : 0; e < edges; ++e)
      mbar_wait(d, &bars[B_EDGE + e % EDGES], (e / EDGES) & 1);
  } else if (warp < 3) {
    // ---------------- products: one thread a tile ----------------
    if (lane == 0) {
      constexpr uint32_t ID_S = instr_desc(KEYS, M, false), ID_O = instr_desc(D, M, true);
      const int x = warp - 1;
      const uint32_t t_s = tmem + S_COL + x * KEYS, t_o = tmem + O_COL + x * D;
      const uint64_t qd = desc_columns(smem_u32(s_q) + x * SLOT);
      const uint64_t kd0 = desc_columns(smem_u32(s_ring)), vd0 = desc_rows(smem_u32(s_ring));
      bool ok = true;
      auto wait = [&](int bar, uint32_t parity) {
        ok = ok && wait_or_stop(d, &bars[bar], parity, stop);
        return ok;
      };
      // Stages are counted on: `st` is the ring's slot of the next one, `pass` its pass over the ring.
      int st = 0;
      uint32_t pass = 0, edges = 0, p_no = 0, q_no = 0, o_no = 0;
      auto full = [&] { return wait(B_FULL + st, pass & 1); };
      auto next = [&] {
        if (++st == RING) {
          st = 0;
          ++pass;
        }
      };
      // S = Q K^T of the next stage; the last one of an item frees its query rows.
      auto scores = [&](bool last) {
        if (!full()) return;
        tc_fence_after();
        const uint64_t kd = desc_at(kd0, st * SLOT);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t at = step_columns(kk);
          tc_mma_ss(t_s, desc_at(qd, at), desc_at(kd, at), ID_S, kk > 0);
        }
        tc_commit(&bars[B_S + x]);
        if (last) tc_commit(&bars[B_Q_EMPTY + x]);
        tc_commit(&bars[B_EMPTY + st]);
        next();
      };
      // A stage that this tile has no use for.
      auto skip = [&] {
        if (!full()) return;
        mbar_arrive(&bars[B_EMPTY + st]);
        next();
      };
      auto begin = [&](int steps, bool mine) {
        if (!mine) return skip();
        if (!wait(B_Q_FULL + x, q_no & 1)) return;
        ++q_no;
        scores(steps == 1);
      };
      if (wait(B_ITEM, 0)) {
        int steps = items[0].steps;
        bool mine = x == 0 || (steps > 0 && items[0].t0 + TOKENS < items[0].si.t);
        if (steps > 0) begin(steps, mine);
        for (int n = 0; ok && steps > 0; ++n) {
          const Item& it = items[n & 1];
          const EdgeSteps edge = edge_steps(it.si, it.t0);
          int steps_next = 0;
          bool mine_next = false;
          for (int j = 0; j < steps && ok; ++j) {
            const bool last = j == steps - 1;
            if (!full()) break;
            if (edge.at(j)) {
              if (!wait(B_FIX + edges % EDGES, (edges / EDGES) & 1)) break;
              ++edges;
            }
            if (mine) {
              if (!wait(B_P + x, p_no & 1)) break;
              ++p_no;
              if (j == 0) {
                if (o_no > 0 && !wait(B_O_EMPTY + x, (o_no - 1) & 1)) break;
                ++o_no;
              }
              tc_fence_after();
              const uint64_t vd = desc_at(vd0, st * SLOT);
#pragma unroll
              for (int kk = 0; kk < KEYS / 16; ++kk)
                tc_mma_ts(t_o, t_s + (kk >> 2) * HALF + (kk & 3) * 8, desc_at(vd, kk * 2 * ROW_GROUP), ID_O, j > 0 || kk > 0);
              if (last) tc_commit(&bars[B_O + x]);
              tc_commit(&bars[B_EMPTY + st]);
            } else {
              mbar_arrive(&bars[B_EMPTY + st]);
            }
            next();
            if (!last) {
              if (mine) scores(j + 2 == steps);
              else skip();
            } else {
              // The next item's first scores go ahead of this one's output.
              if (!wait(B_ITEM + ((n + 1) & 1), ((n + 1) >> 1) & 1)) break;
              const Item& nx = items[(n + 1) & 1];
              steps_next = nx.steps;
              mine_next = x == 0 || (steps_next > 0 && nx.t0 + TOKENS < nx.si.t);
              if (steps_next > 0) begin(steps_next, mine_next);
            }
          }
          if (!ok) break;
          mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
          steps = steps_next;
          mine = mine_next;
        }
      }
      // No product may still be running when the tensor memory is released.
      tc_commit(&bars[B_FINAL]);
      mbar_wait(d, &bars[B_FINAL], 0);
    }
  }
  } else if (warp < 8) {
    set_registers<BASE_REGS, FEW_REGS>();
    // ---------------- query rows, V rows to zero ----------------
    const int ts = tid - 4 * 32;
    bool ok = true;
    auto wait = [&](int bar, uint32_t parity) {
      ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
      return ok;
    };
    uint32_t s0 = 0, edges = 0, q_no[2] = {0, 0};
    for (int n = 0; ok; ++n) {
      if (!wait(B_ITEM + (n & 1), (n >> 1) & 1)) break;
      Item& it = items[n & 1];
      if (it.steps == 0) break;
      const SeqInfo& si = it.si;
      const int head = it.head, t0 = it.t0, steps = it.steps;
      const int tiles = t0 + TOKENS < si.t ? 2 : 1;
      for (int x = 0; x < tiles && ok; ++x) {
        stage_q<1, 2>(d, si, head, t0 + x * TOKENS, q, qk_scale, s_q + x * SLOT, ts,
                   [&] { return q_no[x] == 0 || wait(B_Q_EMPTY + x, (q_no[x] - 1) & 1); });
        if (!ok) break;
        ++q_no[x];
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_Q_FULL + x]);
      }
      // Thread ts has row ts of each such step's V.
      const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1);
      const int q_log0 = si.n_hist + si.n_live - si.t;
      const EdgeSteps edge = edge_steps(si, t0);
      for (int j = 0; j < steps && ok; ++j) {
        const int b = PAGES * j + ts / PS;
        if (!edge.at(j)) continue;
        const uint32_t s = s0 + 2 * j + 1;
        if (!wait(B_EDGE + edges % EDGES, (edges / EDGES) & 1)) break;
        uint8_t* tile = s_ring + (s % RING) * SLOT;
        const uint32_t bit = 1u << (ts % PS);
        bool zero = !(slots_seen(si, b, nb, q_log0 + si.t) & bit);
        if (!zero && !(slots_seen(si, b, nb, q_log0 + t0) & bit)) {  // some rows see it
          bool odd = false;
          for (int i = 0; i < 16; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(tile + tile_at(ts, i));
            odd |= not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w);
          }
          if (odd) {
            it.odd = 1;
            zero = true;
          }
        }
        if (zero)
          for (int i = 0; i < 16; ++i)
            *reinterpret_cast<uint4*>(tile + tile_at(ts, i)) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_FIX + edges % EDGES]);
        ++edges;
      }
      s0 += 2 * steps;
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
    }
  } else {
    set_registers<BASE_REGS, MANY_REGS>();
    // ---------------- softmax ----------------
    const int x = (warp - 8) >> 3, half = (warp - 8) >> 2 & 1;  // tile; keys [64 half, + 64) of a step
    const int quarter = warp & 3, r = quarter * 32 + lane;      // row
    const uint32_t trow = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t t_s = trow + S_COL + x * KEYS + half * HALF, t_o = trow + O_COL + x * D + half * HALF;
    float* mine = reinterpret_cast<float*>(smem + OFF_HALF) + (2 * x + half) * M + r;
    const float* other = reinterpret_cast<float*>(smem + OFF_HALF) + (2 * x + (half ^ 1)) * M + r;
    const int meet = 1 + x * 4 + quarter;                       // barrier of the two warps of a row
    bool ok = true;
    auto wait = [&](int bar, uint32_t parity) {
      ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
      return ok;
    };
    uint32_t s_no = 0, o_no = 0;
    // A warp whose wait gave up goes on to the item's end without waiting or writing results, so that
    // its partner never waits for it alone; then both stop.
    for (int n = 0;; ++n) {
      wait(B_ITEM + (n & 1), (n >> 1) & 1);
      if (meet_any(meet, !ok)) break;
      const Item& it = items[n & 1];
      const int steps = it.steps;
      if (steps == 0) break;
      const SeqInfo& si = it.si;
      const int t0 = it.t0, tok = t0 + x * TOKENS + r / G;
      if (t0 + x * TOKENS < si.t) {
        const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1);
        const int q_log = si.n_hist + si.n_live - si.t + tok;
        const EdgeSteps edge = edge_steps(si, t0);
        float m = 0.f, l = 0.f;
        for (int j = 0; j < steps; ++j, ++s_no) {
          wait(B_S + x, s_no & 1);
          tc_fence_after();
          float s[HALF];
          auto load = [&] {
            tmem_ld32(t_s, s);
            tmem_ld32(t_s + 32, s + 32);
            if (edge.at(j)) {
#pragma unroll
              for (int p = 0; p < PAGES / 2; ++p) {
                const uint32_t seen = slots_seen(si, PAGES * j + PAGES / 2 * half + p, nb, q_log);
#pragma unroll
                for (int i = 0; i < PS; ++i) s[p * PS + i] = (seen >> i & 1) ? s[p * PS + i] : -INFINITY;
              }
            }
          };
          // P = 2^(s - m), which goes over this half's S, and its sum.
          float add = 0.f;
          auto weigh = [&](bool check) {
            uint32_t pw[HALF / 2];
            const float2 nref = make_float2(-m, -m);
            float2 rs[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int i = 0; i < HALF; i += 2) {
              const float2 y = __fadd2_rn(make_float2(s[i], s[i + 1]), nref);
              const float2 p = make_float2(ex2(y.x), ex2(y.y));
              rs[(i / 2) & 1] = __fadd2_rn(rs[(i / 2) & 1], p);
              pw[i / 2] = pack_bf16(p.x, p.y);
            }
            const float2 r2 = __fadd2_rn(rs[0], rs[1]);
            add = r2.x + r2.y;
            if (check && meet_any(meet, !(add < SUM_LIMIT))) return false;
            __syncwarp();
            tmem_st32(t_s, pw);
            return true;
          };
          // The first step, and one where a sum is out of bounds against the reference so far (or NaN):
          // the row's maximum becomes the reference.  (The scores' barrier says that the products
          // before them are complete too, the last O += P V among them, so O may be rescaled.)
          bool done = false;
          if (j > 0) {
            load();
            done = weigh(true);
          }
          if (!done) {
            load();
            float m4[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) m4[i] = s[i];
#pragma unroll
            for (int i = 4; i < HALF; i += 4)
#pragma unroll
              for (int c = 0; c < 4; ++c) m4[c] = fmaxf(m4[c], s[i + c]);
            *mine = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            meet_any(meet, false);
            const float mx = fmaxf(*mine, *other);
            const float to = j == 0 ? (mx == -INFINITY ? 0.f : mx) : fmaxf(m, mx);
            if (j > 0) {
              const float f = exp2f(m - to);
              l *= f;
              __syncwarp();
#pragma unroll 1
              for (int c = 0; c < HALF / 16; ++c) {
                float o[16];
                tmem_ld16(t_o + c * 16, o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] *= f;
                tmem_st16(t_o + c * 16, o);
              }
            }
            m = to;
            weigh(false);
          }
          l += add;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[B_P + x]);
        }
        // The row's sum, then dims [64 half, + 64) of its output.
        wait(B_O + x, o_no & 1);
        ++o_no;
        tc_fence_after();
        *mine = l;
        meet_any(meet, false);
        const float inv = 1.f / (l + *other);
        meet_any(meet, false);  // (read before the next item's exchange)
        const bool odd = *reinterpret_cast<volatile const int*>(&it.odd) != 0;
        __nv_bfloat16* row = out + ((size_t)(si.q_row0 + tok) * d.q_heads + it.head * G + r % G) * D + half * HALF;
#pragma unroll 1
        for (int c = 0; c < HALF; c += 32) {
          float o[32];
          tmem_ld32(t_o + c, o);
          if (odd && tok < si.t) {
            float more[32];
            odd_value(d, si, layer, it.head, t0, tok, r % G, q, qk_scale, m, half * HALF + c, more);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] += more[i];
          }
          if (ok && tok < si.t) {
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
  // The last CTA leaves the counters as it found them.
  if (tid == 0 && atomicAdd(&d.dec_count[0], 1) == (int)gridDim.x - 1) {
    d.pf_count[0] = 0;
    d.dec_count[0] = 0;
  }
}

}  // namespace

cudaError_t prompt_tc_attributes() {
  return cudaFuncSetAttribute(prompt_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              SMEM_BYTES);
}

cudaError_t launch_prompt_tc(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                             cudaStream_t s) {
  CUtensorMap map;
  if (!pool_tile_map(d, &map)) return cudaErrorInvalidValue;
  return launch_ex(&prompt_tc_kernel, dim3(lim.sms), dim3(TC_THREADS), SMEM_BYTES, s, true, d,
                   layer, map, static_cast<const __nv_bfloat16*>(q), static_cast<__nv_bfloat16*>(out),
                   LOG2E / sqrtf((float)D));
}

}  // namespace kvc
