// Attention weights of chunks (kvc_attn_weights) over bfloat16 rows, on the 5th-generation tensor cores.
//
// Weights are sums of probabilities in binary32, so the scores keep more of q than bfloat16 has: q is
// held in two bfloat16 pieces, q_up = bf16(q) and bf16(q - q_up), and S = K q_up + K q_low adds up both
// products in one accumulator; what is left out is below 2^-17 of q.  K is what the cache holds, exact.
// Two passes over the scores, since a weight needs its row's sum:
//   weights_stat_kernel   S = Q K^T, a thread has a query row: running (max, sum), of `parts` ranges of
//                         the keys where the chunk alone has too few rows for all SMs
//   weights_sums_kernel   S^T = K Q^T, a thread has a key and adds up 2^(s - lse) along its row, for 512
//                         keys of one (session, KV head) and a share of the chunk's tokens an item; no
//                         sum crosses threads
// The sums of heads and shares are added up by weights_add_kernel (kvc_weights.cu) in their order.
// Both are bound by the products, 16 of 74 cycles for a tile of 128 x 128; its exponentials take half of
// that.  What else decided their layout (two prompts of 3,001 and 940 tokens, 8 KV heads, a layer; all
// three kernels):
//   - Tensor cores stand still between a thread's products of one tile and the next: a commit and a wait,
//     400 cycles.  Two threads issue them, a tile each: statistics 72 -> 64 us.  In the sums both tiles'
//     scores would then come at once, with no buffer left for the next ones, so the threads take turns, and
//     the turn passes on six products early: 168 -> 163.5 us, 177 with one thread.
//   - A query tile, rotated and cut into pieces, costs its warps 2,500 cycles.  The sums stage one for four
//     tiles of keys, which wait in tensor memory as rows of A (two tiles: 182 us with the shares below).
//   - A row's lse comes from a warp of its own: in the staging warps it cost them a load's time a tile.
//   - Shares of the tokens that see a key, rather than of all tokens: 205 -> 182 us.
// Warp roles as in kvc_prompt_tc.cu: warp 0 items and K by TMA, warps 1 and 2 the products, warp 3 the
// sums' lse, then the warps that stage query tiles (statistics: eight, with four they were what the products
// waited for), the last eight what becomes of the scores.  All waits are bounded.
#include <cuda.h>

#include <cmath>

#include "kvc_prompt_tc.cuh"
#include "kvc_weights_plain.cuh"

namespace kvc {

namespace {

// Warps that stage query tiles: an item of the statistics starts with two; one of the sums' meets four tiles of
// keys, and its last warps want the registers.
constexpr int STAT_Q_WARPS = 8, SUMS_Q_WARPS = 4;
constexpr int STAT_THREADS = 128 + 32 * STAT_Q_WARPS + 256, SUMS_THREADS = 128 + 32 * SUMS_Q_WARPS + 256;
constexpr int CHUNK = 32;                          // columns that a row takes at a time
constexpr float SUM_LIMIT = 1048576.f;              // 2^20, see below
constexpr int K_RING = 3;
constexpr int LSE_RING = 4;                        // query tiles whose lse is kept
constexpr int ALL_COLS = 512;                      // two tiles' scores, twice each: 4 x 128 columns
constexpr int TURN_EARLY = 6;                      // sums: products that a thread issues behind its turn
constexpr int KEY_TILES = 4;                       // of an item of the sums
constexpr int KT_COL = 2 * KEYS;                   // its keys, as rows of A, behind two tiles' scores
static_assert(KT_COL + KEY_TILES * D / 2 == ALL_COLS, "tensor memory of the sums");
constexpr int OFF_ITEM = 512;                      // [2]
constexpr int OFF_TMEM = OFF_ITEM + 2 * 128;
constexpr int OFF_STOP = OFF_TMEM + 4;
constexpr int OFF_GROUP = OFF_STOP + 4;            // the work list
constexpr int OFF_TILES = 3 * 1024;
constexpr int SMEM_BYTES = OFF_TILES + 7 * SLOT;
static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of a CTA");

enum {
  B_FULL = 0,                        // [K_RING] a K tile has landed
  B_EMPTY = B_FULL + K_RING,         // [K_RING] and was read
  B_Q_FULL = B_EMPTY + K_RING,       // [2] a query tile is there
  B_Q_EMPTY = B_Q_FULL + 2,          // [2] and was read
  B_S = B_Q_EMPTY + 2,               // [2 tiles][2] scores complete
  B_S_EMPTY = B_S + 4,               // [2 tiles][2] and read
  B_ITEM = B_S_EMPTY + 4,            // [2] an item is known
  B_ITEM_EMPTY = B_ITEM + 2,         // [2] and every warp is through with it
  B_LSE_EMPTY = B_ITEM_EMPTY + 2,    // sums: [LSE_RING] lse of a query tile was read
  B_LSE = B_LSE_EMPTY + LSE_RING,    // sums: [LSE_RING] and is there
  B_KT = B_LSE + LSE_RING,           // sums: [KEY_TILES] keys are in tensor memory
  B_TURN = B_KT + KEY_TILES,         // sums: [2] a thread's turn to issue products
  B_FINAL = B_TURN + 2,              // [2] all products are there
  N_BARS = B_FINAL + 2
};
static_assert(N_BARS * 8 <= OFF_ITEM, "barriers fit");
constexpr int ITEM_READERS = 2 + 8;                // and the staging warps, and warp 3 where sums are formed

struct Item {
  SeqInfo si;
  int32_t valid;          // 0: no more items
  int32_t head;
  int32_t at;             // stat: first token; sums: first page
  int32_t part;           // stat: part of the keys; sums: share of the tokens
  int32_t begin, end;     // stat: steps of keys; sums: tiles of tokens
  int32_t upper;          // sums: first tile of tokens that sees a key of tiles 2 and 3
  int32_t tiles;          // sums: tiles of keys that some of the tokens see
  int32_t pad[8];
};
static_assert(sizeof(Item) == 128, "Item size");

__device__ inline void init_barriers(uint64_t* bars, bool sums) {  // a thread a barrier
  const int q_warps = sums ? SUMS_Q_WARPS : STAT_Q_WARPS, i = threadIdx.x;
  if (i >= N_BARS) return;
  const int count = i >= B_EMPTY && i < B_Q_FULL           ? (sums ? 4 : 2)
                    : i >= B_Q_FULL && i < B_Q_EMPTY       ? q_warps
                    : i >= B_Q_EMPTY && i < B_S && sums    ? 2
                    : i >= B_S_EMPTY && i < B_ITEM         ? 4
                    : i >= B_ITEM_EMPTY && i < B_LSE_EMPTY ? ITEM_READERS + q_warps + sums
                    : i >= B_LSE_EMPTY && i < B_LSE        ? 8
                    : i >= B_KT && i < B_TURN              ? 4
                                                           : 1;
  mbar_init(&bars[i], count);
  fence_mbar_init();
}

// Both pieces' products of a tile: A the rows at a (a_step bytes to its other piece), B at b likewise.
__device__ inline void piece_products(uint32_t to, uint32_t a, uint32_t a_step, uint32_t b, uint32_t b_step,
                                      uint32_t idesc) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint64_t ad = desc_columns(a + p * a_step), bd = desc_columns(b + p * b_step);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const uint32_t at = step_columns(kk);
      tc_mma_ss(to, desc_at(ad, at), desc_at(bd, at), idesc, p > 0 || kk > 0);
    }
  }
}

// ---------------------------------------------------------------------------
// Row statistics: an item is 64 tokens (tiles A and B) of one (session, KV head) and a part of the keys.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(STAT_THREADS, 1) weights_stat_kernel(
    Dev d, int layer, const __grid_constant__ CUtensorMap map,
    const __nv_bfloat16* __restrict__ q, float qk_scale,
    int most_parts, WeightsWork work) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem);
  Item* items = reinterpret_cast<Item*>(smem + OFF_ITEM);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_TMEM);
  volatile int* stop = reinterpret_cast<int*>(smem + OFF_STOP);
  int* s_group = reinterpret_cast<int*>(smem + OFF_GROUP);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = d.kv_heads;
  uint8_t* s_q = smem + OFF_TILES;      // A upper, A lower, B upper, B lower
  uint8_t* s_k = s_q + 4 * SLOT;
  pdl_wait();
  pdl_launch_dependents();
  const int n_seq = d.g->total_tokens > 0 ? d.g->n_seq : 0, parts = stat_parts(d, most_parts, d.g->total_tokens);
  init_barriers(bars, false);
  if (tid == 0) *stop = 0;
  auto items_of = [&](int i) { return (d.seq[i].t + 2 * TOKENS - 1) / (2 * TOKENS) * H * parts; };
  if (warp == 2) list_items(n_seq, lane, s_group, items_of);
  __syncwarp();
  if (warp == 1) tmem_alloc(tmem_slot, ALL_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true;
  auto wait_warp = [&](int bar, uint32_t parity) {
    ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
    return ok;
  };

  if (warp < 4) {
    if (warp == 0) {
      const int total = s_group[GROUPS];
      uint32_t k_no = 0;
      for (int n = 0; ok; ++n) {
        Item* it = items + (n & 1);
        if (n >= 2 && !wait_warp(B_ITEM_EMPTY + (n & 1), ((n >> 1) & 1) ^ 1)) break;
        int at = 0;
        if (lane == 0) at = take_item(d);
        at = __shfl_sync(FULL, at, 0);
        if (at >= total) {
          if (lane == 0) {
            it->valid = 0;
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
        const int n_t = (si.t + 2 * TOKENS - 1) / (2 * TOKENS), head = in % H, part = in / H % parts;
        const int t0 = (n_t - 1 - in / H / parts) * 2 * TOKENS;
        const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1), steps = (nb + PAGES - 1) / PAGES;
        const int j0 = (int)((int64_t)steps * part / parts), j1 = (int)((int64_t)steps * (part + 1) / parts);
        if (lane == 0) {
          it->valid = 1;
          it->head = head;
          it->at = t0;
          it->part = part;
          it->begin = j0;
          it->end = j1;
          mbar_arrive(&bars[B_ITEM + (n & 1)]);
        }
        const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
        const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
        auto page_at = [&](int b) { return b < nb ? block_page(si, hrow, lrow, b) : 0; };
        int pid = page_at(PAGES * j0 + lane), pid_next = page_at(PAGES * j0 + 32 + lane);
        for (int j = j0; j < j1; ++j, ++k_no) {
          if (j > j0 && ((j - j0) & 3) == 0) {
            pid = pid_next;
            pid_next = page_at(PAGES * j + 32 + lane);
          }
          const int page = __shfl_sync(FULL, pid, PAGES * ((j - j0) & 3) + (lane & 7));
          const int n_pg = min(PAGES, nb - PAGES * j), st = k_no % K_RING;
          if (k_no >= K_RING && !wait_warp(B_EMPTY + st, ((k_no / K_RING) & 1) ^ 1)) break;
          if (lane == 0) mbar_arrive_expect_tx(&bars[B_FULL + st], n_pg * PS * D * 2);
          __syncwarp();
          load_tile(d, layer, 0, head, page, n_pg, s_k + st * SLOT, &map, &bars[B_FULL + st], lane);
        }
      }
      for (uint32_t s = k_no > K_RING ? k_no - K_RING : 0; s < k_no; ++s)
        mbar_wait(d, &bars[B_FULL + s % K_RING], (s / K_RING) & 1);
    } else if (warp < 3) {  // the products with query tile x
      if (lane == 0) {
        const int x = warp - 1;
        constexpr uint32_t ID = instr_desc(KEYS, M, false);
        const uint32_t a_q = smem_u32(s_q), a_k = smem_u32(s_k);
        auto wait = [&](int bar, uint32_t parity) {
          ok = ok && wait_or_stop(d, &bars[bar], parity, stop);
          return ok;
        };
        uint32_t k_no = 0, q_no = 0, s_no = 0;
        for (int n = 0; ok; ++n) {
          if (!wait(B_ITEM + (n & 1), (n >> 1) & 1)) break;
          const Item& it = items[n & 1];
          if (!it.valid) break;
          const int j0 = it.begin, j1 = it.end;
          const bool mine = it.at + x * TOKENS < it.si.t;
          if (mine && j0 < j1 && !wait(B_Q_FULL + x, q_no++ & 1)) break;
          for (int j = j0; j < j1; ++j, ++k_no) {
            if (!wait(B_FULL + k_no % K_RING, (k_no / K_RING) & 1)) break;
            if (!mine) {
              mbar_arrive(&bars[B_EMPTY + k_no % K_RING]);
              continue;
            }
            const int b = 2 * x + (s_no & 1);
            if (s_no >= 2 && !wait(B_S_EMPTY + b, ((s_no >> 1) & 1) ^ 1)) break;
            ++s_no;
            tc_fence_after();
            piece_products(tmem + b * KEYS, a_q + 2 * x * SLOT, SLOT, a_k + (k_no % K_RING) * SLOT, 0, ID);
            tc_commit(&bars[B_S + b]);
            if (j == j1 - 1) tc_commit(&bars[B_Q_EMPTY + x]);
            tc_commit(&bars[B_EMPTY + k_no % K_RING]);
          }
          mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
        }
        tc_commit(&bars[B_FINAL + x]);
        mbar_wait(d, &bars[B_FINAL + x], 0);
      }
    }
  } else if (warp < 4 + STAT_Q_WARPS) {
    const int ts = tid - 4 * 32;
    uint32_t q_no[2] = {0, 0};
    for (int n = 0; ok; ++n) {
      if (!wait_warp(B_ITEM + (n & 1), (n >> 1) & 1)) break;
      const Item& it = items[n & 1];
      if (!it.valid) break;
      const int tiles = it.at + TOKENS < it.si.t ? 2 : 1;
      for (int x = 0; x < tiles && ok && it.begin < it.end; ++x) {
        stage_q<2, 32 * STAT_Q_WARPS>(d, it.si, it.head, it.at + x * TOKENS, q, qk_scale, s_q + 2 * x * SLOT, ts,
                   [&] { return q_no[x] == 0 || wait_warp(B_Q_EMPTY + x, (q_no[x] - 1) & 1); });
        if (!ok) break;
        ++q_no[x];
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_Q_FULL + x]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
    }
  } else {
    const int x = (warp - 4 - STAT_Q_WARPS) >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    uint32_t s_no = 0;
    for (int n = 0; ok; ++n) {
      if (!wait_warp(B_ITEM + (n & 1), (n >> 1) & 1)) break;
      const Item& it = items[n & 1];
      if (!it.valid) break;
      const SeqInfo& si = it.si;
      const int t0 = it.at, tok = t0 + x * TOKENS + r / G;
      if (t0 + x * TOKENS < si.t) {
        const int nb = blocks_seen(si, min(t0 + 2 * TOKENS, si.t) - 1);
        const int q_log = si.n_hist + si.n_live - si.t + tok;
        const EdgeSteps edge = edge_steps(si, t0);
        float m = -INFINITY, l = 0.f;
        for (int j = it.begin; j < it.end; ++j, ++s_no) {
          const int b = 2 * x + (s_no & 1);
          if (!wait_warp(B_S + b, (s_no >> 1) & 1)) break;
          tc_fence_after();
          // The reference is the maximum of the first keys, until a sum against it passes the limit (or is
          // NaN); sums and roundings do not depend on its scale.
          const bool masks = edge.at(j);
          float add = 0.f;
#pragma unroll 1
          for (int c = 0; c < KEYS / CHUNK; ++c) {
            uint32_t w[CHUNK];
            tmem_ld32_begin(trow + b * KEYS + CHUNK * c, w);
            tmem_ld32_wait(w);
            if (masks) {
#pragma unroll
              for (int p = 0; p < CHUNK / PS; ++p) {
                const uint32_t seen = slots_seen(si, PAGES * j + CHUNK / PS * c + p, nb, q_log);
#pragma unroll
                for (int i = 0; i < PS; ++i) w[p * PS + i] = (seen >> i & 1) ? w[p * PS + i] : 0xFF800000u;
              }
            }
            auto most = [&] {
              float a[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) a[i] = __uint_as_float(w[i]);
#pragma unroll
              for (int i = 4; i < CHUNK; i += 4)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] = fmaxf(a[k], __uint_as_float(w[i + k]));
              return fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
            };
            auto sum_of = [&] {
              const float ref = m == -INFINITY ? 0.f : m;  // (a row that has seen no key yet)
              const float2 nref = make_float2(-ref, -ref);
              float2 rs[4] = {};
#pragma unroll
              for (int i = 0; i < CHUNK; i += 2) {
                const float2 y = __fadd2_rn(make_float2(__uint_as_float(w[i]), __uint_as_float(w[i + 1])), nref);
                rs[(i / 2) & 3] = __fadd2_rn(rs[(i / 2) & 3], make_float2(ex2(y.x), ex2(y.y)));
              }
              const float2 r2 = __fadd2_rn(__fadd2_rn(rs[0], rs[1]), __fadd2_rn(rs[2], rs[3]));
              return r2.x + r2.y;
            };
            float sum = m == -INFINITY ? INFINITY : sum_of();
            if (!__all_sync(FULL, sum < SUM_LIMIT)) {
              const float to = fmaxf(m, most()), f = m == -INFINITY ? 0.f : exp2f(m - to);
              l *= f;
              add *= f;
              m = to;
              sum = sum_of();
            }
            add += sum;
          }
          l += add;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[B_S_EMPTY + b]);
        }
        if (ok && tok < si.t && isnan(l)) {
          const float2 again = plain_stat<__nv_bfloat16, D>(d, si, layer, it.head, tok, r % G, q, qk_scale,
                                                            PAGES * it.begin, PAGES * it.end, nb);
          m = again.x;
          l = again.y;
        }
        if (ok && tok < si.t)
          work.stats[((size_t)it.part * d.g->total_tokens + si.q_row0 + tok) * d.q_heads + it.head * G + r % G] =
              make_float2(m, l);
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

// ---------------------------------------------------------------------------
// Sums by key: an item is 512 keys (four tiles) of one (session, KV head) and a share of the tokens.
// ---------------------------------------------------------------------------
constexpr int OFF_LSE = OFF_GROUP + 136;
static_assert((GROUPS + 1) * 4 <= 136 && OFF_LSE % 16 == 0 && OFF_LSE + LSE_RING * M * 4 <= OFF_TILES,
              "header fits");

__global__ void __launch_bounds__(SUMS_THREADS, 1) weights_sums_kernel(
    Dev d, int layer, const __grid_constant__ CUtensorMap map,
    const __nv_bfloat16* __restrict__ q, float qk_scale,
    int most_parts, int shares, WeightsWork work) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem);
  Item* items = reinterpret_cast<Item*>(smem + OFF_ITEM);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_TMEM);
  volatile int* stop = reinterpret_cast<int*>(smem + OFF_STOP);
  int* s_group = reinterpret_cast<int*>(smem + OFF_GROUP);
  float* s_lse = reinterpret_cast<float*>(smem + OFF_LSE);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = d.kv_heads;
  uint8_t* s_k = smem + OFF_TILES;
  uint8_t* s_q = s_k + 2 * SLOT;        // two tiles of two pieces
  pdl_wait();
  pdl_launch_dependents();
  const int n_seq = d.g->total_tokens > 0 ? d.g->n_seq : 0;
  auto items_of = [&](int i) {
    return (d.seq[i].n_blocks + KEY_TILES * PAGES - 1) / (KEY_TILES * PAGES) * H * shares;
  };
  init_barriers(bars, true);
  if (tid == 0) *stop = 0;
  if (warp == 2) list_items(n_seq, lane, s_group, items_of);
  __syncwarp();
  if (warp == 1) tmem_alloc(tmem_slot, ALL_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true;
  auto wait_warp = [&](int bar, uint32_t parity) {
    ok = ok && __all_sync(FULL, wait_or_stop(d, &bars[bar], parity, stop));
    return ok;
  };

  if (warp < 4) {
    if (warp == 0) {
      const int total = s_group[GROUPS];
      uint32_t k_used[2] = {0, 0};  // tiles that each slot took, one of them for each four of the last warps
      for (int n = 0; ok; ++n) {
        Item* it = items + (n & 1);
        if (n >= 2 && !wait_warp(B_ITEM_EMPTY + (n & 1), ((n >> 1) & 1) ^ 1)) break;
        int at = 0;
        if (lane == 0) at = take_item(d);
        at = __shfl_sync(FULL, at, 0);
        if (at >= total) {
          if (lane == 0) {
            it->valid = 0;
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
        const int head = in % H, share = in / H % shares, b0 = in / H / shares * KEY_TILES * PAGES;
        const int n_t = (si.t + TOKENS - 1) / TOKENS, q_log0 = si.n_hist + si.n_live - si.t;
        const int first = max(0, block_range(si, b0).base - q_log0) / TOKENS;
        // (The tokens that see a key of the tile, shared out evenly: long items come first.)
        const int i0 = first + (int)((int64_t)(n_t - first) * share / shares);
        const int i1 = first + (int)((int64_t)(n_t - first) * (share + 1) / shares);
        const int upper =
            b0 + 2 * PAGES < si.n_blocks ? max(0, block_range(si, b0 + 2 * PAGES).base - q_log0) / TOKENS : i1;
        const int tiles = min(upper < i1 ? KEY_TILES : 2, (si.n_blocks - b0 + PAGES - 1) / PAGES);
        if (lane == 0) {
          it->valid = 1;
          it->head = head;
          it->at = b0;
          it->part = share;
          it->upper = upper;
          it->tiles = tiles;
          it->begin = i0;
          it->end = i1;
          mbar_arrive(&bars[B_ITEM + (n & 1)]);
        }
        if (i0 == i1) continue;
        const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
        const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
        const int b = b0 + lane;
        const int pid = b < si.n_blocks ? block_page(si, hrow, lrow, b) : 0;
        for (int y = 0; y < tiles; ++y) {
          const int page = __shfl_sync(FULL, pid, PAGES * y + (lane & 7));
          const int n_pg = min(PAGES, si.n_blocks - b0 - y * PAGES), st = y & 1;
          if (k_used[st] && !wait_warp(B_EMPTY + st, (k_used[st] & 1) ^ 1)) break;
          ++k_used[st];
          if (lane == 0) mbar_arrive_expect_tx(&bars[B_FULL + st], n_pg * PS * D * 2);
          __syncwarp();
          load_tile(d, layer, 0, head, page, n_pg, s_k + st * SLOT, &map, &bars[B_FULL + st], lane);
        }
      }
      for (int st = 0; st < 2; ++st)
        if (k_used[st]) mbar_wait(d, &bars[B_FULL + st], (k_used[st] & 1) ^ 1);
    } else if (warp < 3) {  // the products with key tiles x and x + 2
      if (lane == 0) {
        const int x = warp - 1;
        auto wait = [&](int bar, uint32_t parity) {
          ok = ok && wait_or_stop(d, &bars[bar], parity, stop);
          return ok;
        };
        uint32_t q_no = 0, s_no = 0, kt_no = 0, turn = 0;  // (kt_no: parities, a bit a tile)
        for (int n = 0; ok; ++n) {
          if (!wait(B_ITEM + (n & 1), (n >> 1) & 1)) break;
          const Item& it = items[n & 1];
          if (!it.valid) break;
          const int tiles = it.tiles, upper = it.upper, i0 = it.begin, i1 = it.end, t = it.si.t;
          uint32_t there = 0;  // tiles in tensor memory
          for (int i = i0; i < i1 && ok; ++i, ++q_no) {
            if (!wait(B_Q_FULL + (q_no & 1), (q_no >> 1) & 1)) break;
            const int rows = min(TOKENS, t - i * TOKENS) * G;
            const uint32_t id = instr_desc((rows + 31) / 32 * 32, M, false);
            const int seen = i < upper ? min(tiles, 2) : tiles;
            // The threads take turns: the tensor cores work off both threads' products together, and both tiles'
            // scores would be there, and read, at the same time, with nothing to do meanwhile.
#pragma unroll 1
            for (int y = x; y - x < seen && ok; y += 2) {
              if (y < seen) {
                if (!(there >> y & 1)) {
                  if (!wait(B_KT + y, kt_no >> y & 1)) break;
                  kt_no ^= 1u << y;
                  there |= 1u << y;
                }
                if (s_no > 0 && !wait(B_S_EMPTY + x, (s_no & 1) ^ 1)) break;
                ++s_no;
              }
              if ((x == 1 || turn > 0) && !wait(B_TURN + x, (turn & 1) ^ (x ^ 1))) break;
              ++turn;
              if (y >= seen) {
                mbar_arrive(&bars[B_TURN + (x ^ 1)]);
                continue;
              }
              tc_fence_after();
              const uint32_t a_q = smem_u32(s_q) + (q_no & 1) * 2 * SLOT;
#pragma unroll
              for (int p = 0; p < 2; ++p) {
                const uint64_t bd = desc_columns(a_q + p * SLOT);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                  // (The next turn's wait takes as long as the last products.)
                  if (p == 1 && kk == D / 16 - TURN_EARLY) mbar_arrive(&bars[B_TURN + (x ^ 1)]);
                  tc_mma_ts(tmem + x * KEYS, tmem + KT_COL + y * (D / 2) + kk * 8, desc_at(bd, step_columns(kk)), id,
                            p > 0 || kk > 0);
                }
              }
              tc_commit(&bars[B_S + x]);
            }
            tc_commit(&bars[B_Q_EMPTY + (q_no & 1)]);
          }
          mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
        }
        tc_commit(&bars[B_FINAL + x]);
        mbar_wait(d, &bars[B_FINAL + x], 0);
      }
    } else {  // four rows of a query tile each lane: their denominators; rows past the chunk draw nothing
      uint32_t q_no = 0;
      const int parts = stat_parts(d, most_parts, d.g->total_tokens);
      const size_t stride = (size_t)d.g->total_tokens * d.q_heads;
      for (int n = 0; ok; ++n) {
        if (!wait_warp(B_ITEM + (n & 1), (n >> 1) & 1)) break;
        const Item& it = items[n & 1];
        if (!it.valid) break;
        for (int i = it.begin; i < it.end; ++i, ++q_no) {
          const int tok = i * TOKENS + lane;
          const float2* row = work.stats + (size_t)(it.si.q_row0 + tok) * d.q_heads + it.head * G;
          float4 lse = make_float4(INFINITY, INFINITY, INFINITY, INFINITY);
          if (tok < it.si.t)
            lse = make_float4(row_lse(row, stride, parts), row_lse(row + 1, stride, parts),
                              row_lse(row + 2, stride, parts), row_lse(row + 3, stride, parts));
          const uint32_t ring = q_no % LSE_RING;
          if (q_no >= LSE_RING && !wait_warp(B_LSE_EMPTY + ring, ((q_no / LSE_RING) & 1) ^ 1)) break;
          reinterpret_cast<float4*>(s_lse + ring * M)[lane] = lse;
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[B_LSE + ring]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
      }
    }
  } else if (warp < 4 + SUMS_Q_WARPS) {
    const int ts = tid - 4 * 32;
    uint32_t q_no = 0;
    for (int n = 0; ok; ++n) {
      if (!wait_warp(B_ITEM + (n & 1), (n >> 1) & 1)) break;
      const Item& it = items[n & 1];
      if (!it.valid) break;
      const SeqInfo& si = it.si;
      for (int i = it.begin; i < it.end && ok; ++i, ++q_no) {
        stage_q<2, 32 * SUMS_Q_WARPS>(d, si, it.head, i * TOKENS, q, qk_scale, s_q + (q_no & 1) * 2 * SLOT, ts,
                   [&] { return q_no < 2 || wait_warp(B_Q_EMPTY + (q_no & 1), ((q_no >> 1) & 1) ^ 1); });
        if (!ok) break;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_Q_FULL + (q_no & 1)]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_ITEM_EMPTY + (n & 1)]);
    }
  } else {
    const int x = (warp - 4 - SUMS_Q_WARPS) >> 2, r = (warp & 3) * 32 + lane;  // key r of tiles x and x + 2
    const uint32_t trow = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    uint32_t s_no = 0, q_no = 0, k_no = 0;
    for (int n = 0; ok; ++n) {
      if (!wait_warp(B_ITEM + (n & 1), (n >> 1) & 1)) break;
      const Item& it = items[n & 1];
      if (!it.valid) break;
      const SeqInfo& si = it.si;
      const int i0 = it.begin, i1 = it.end, tiles = it.tiles, slot = r % PS;
      bool in[2];
      int seen_from[2], page[2];  // first token
      float sum[2] = {0.f, 0.f}, rest[2] = {0.f, 0.f};  // (what additions to the sums rounded off)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int y = x + 2 * h, blk = it.at + y * PAGES + r / PS;
        const BlockRange br = blk < si.n_blocks ? block_range(si, blk) : BlockRange{0, 0, 0};
        in[h] = slot >= br.lo && slot < br.hi;
        page[h] = in[h] ? block_page(si, d.hist_pt + (size_t)si.sid * d.max_pages_per_session,
                                     d.live_pt + (size_t)si.sid * d.max_pages_per_session, blk)
                        : 0;
        seen_from[h] = in[h] ? br.base + slot - (si.n_hist + si.n_live - si.t) : 0;
        if (y >= tiles || i0 == i1) continue;
        // The key's row, from the tile that has landed into tensor memory.
        if (!wait_warp(B_FULL + x, k_no++ & 1)) break;
        tc_fence_after();  // (the last item's products are behind its last scores, which were read)
#pragma unroll
        for (int c = 0; c < 16; c += 4) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(w + 4 * e) = *reinterpret_cast<const uint4*>(s_k + x * SLOT + tile_at(r, c + e));
          tmem_st16_begin(trow + KT_COL + y * (D / 2) + 4 * c, w);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars[B_KT + y]);
          mbar_arrive(&bars[B_EMPTY + x]);
        }
      }
      for (int i = i0; i < i1 && ok && x < tiles; ++i) {
        const uint32_t at = q_no + i - i0, ring = at % LSE_RING;
        const float4* lse = reinterpret_cast<const float4*>(s_lse + ring * M);
        const int rows = min(TOKENS, si.t - i * TOKENS) * G;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (h == 1 && (x + 2 >= tiles || i < it.upper)) continue;
          if (!wait_warp(B_S + x, s_no++ & 1)) break;
          // (In this order: the tile's products are behind those of the ring's last round, whose lse was read.)
          if (h == 0 && !wait_warp(B_LSE + ring, (at / LSE_RING) & 1)) break;
          tc_fence_after();
          const int first = seen_from[h] - i * TOKENS;  // first token of the tile that sees the key
          const bool edge = __any_sync(FULL, first > 0);
          float2 a[2] = {};
          auto add_up = [&](const uint32_t (&w)[32], int c) {
#pragma unroll
            for (int g = 0; g < 8; ++g) {  // a token's four heads
              const float4 o = lse[c / 4 + g];
              float2 u = __fadd2_rn(make_float2(__uint_as_float(w[4 * g]), __uint_as_float(w[4 * g + 1])),
                                    make_float2(-o.x, -o.y));
              float2 v = __fadd2_rn(make_float2(__uint_as_float(w[4 * g + 2]), __uint_as_float(w[4 * g + 3])),
                                    make_float2(-o.z, -o.w));
              u = make_float2(ex2(u.x), ex2(u.y));
              v = make_float2(ex2(v.x), ex2(v.y));
              if (edge && c / 4 + g < first) u = v = make_float2(0.f, 0.f);
              a[0] = __fadd2_rn(a[0], u);
              a[1] = __fadd2_rn(a[1], v);
            }
          };
          // The buffer is free once the last 32 columns are here, which is when the first were added up.
          uint32_t w0[32], w1[32], w2[32];
          tmem_ld32_begin(trow + x * KEYS, w0);
          tmem_ld32_begin(trow + x * KEYS + 32, w1);
          tmem_ld32_begin(trow + x * KEYS + 64, w2);
          tmem_ld32_wait(w0);
          tmem_ld32_wait(w1);
          tmem_ld32_wait(w2);
          add_up(w0, 0);
          tmem_ld32_begin(trow + x * KEYS + 96, w0);
          tmem_ld32_wait(w0);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[B_S_EMPTY + x]);
          if (rows > 32) add_up(w1, 32);
          if (rows > 64) add_up(w2, 64);
          if (rows > 96) add_up(w0, 96);
          const float2 a2 = __fadd2_rn(a[0], a[1]);
          const float add = (a2.x + a2.y) + rest[h], to = sum[h] + add;
          rest[h] = add - (to - sum[h]);
          sum[h] = to;
        }
        if (ok && lane == 0) {
          mbar_arrive(&bars[B_LSE_EMPTY + ring]);
          if (tiles == 1) mbar_arrive(&bars[B_LSE_EMPTY + ring]);  // (for the other four warps, without a tile)
        }
      }
      if (!ok) break;
      q_no += i1 - i0;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (in[h] && isnan(sum[h]))
          sum[h] = plain_sum<__nv_bfloat16, D>(d, si, layer, it.head, page[h], slot, max(i0 * TOKENS, seen_from[h]),
                                               min(i1 * TOKENS, si.t), q, qk_scale, work.stats,
                                               stat_parts(d, most_parts, d.g->total_tokens));
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (in[h]) work.scores[((size_t)(it.head * shares + it.part) * d.n_pages + page[h]) * PS + slot] = sum[h];
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

}  // namespace

cudaError_t weights_tc_attributes() {
  const cudaError_t e = cudaFuncSetAttribute(weights_stat_kernel,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
  return e != cudaSuccess ? e
                          : cudaFuncSetAttribute(weights_sums_kernel,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
}

cudaError_t launch_weights_tc(const Dev& d, const Limits& lim, int layer, const void* q,
                              const WeightsWork& work, int parts, int shares, cudaStream_t s,
                              int64_t* launches) {
  CUtensorMap map;
  if (!pool_tile_map(d, &map)) return cudaErrorInvalidValue;
  const float scale = LOG2E / sqrtf((float)D);
  const __nv_bfloat16* qt = static_cast<const __nv_bfloat16*>(q);
  cudaError_t e = launch_ex(&weights_stat_kernel, dim3(lim.sms), dim3(STAT_THREADS), SMEM_BYTES, s, true, d,
                            layer, map, qt, scale, parts, work);
  *launches += e == cudaSuccess;
  if (e != cudaSuccess) return e;
  e = launch_ex(&weights_sums_kernel, dim3(lim.sms), dim3(SUMS_THREADS), SMEM_BYTES, s, true, d, layer, map,
                qt, scale, parts, shares, work);
  *launches += e == cudaSuccess;
  return e;
}

}  // namespace kvc
