// What the tensor-core kernels of whole prompts share: tiles of 128 rows (32 tokens x 4 query heads of a
// KV head, or 128 keys) by 128 dims, their products, waits, masks and work lists.
#pragma once

#include "kvc_prefill_tc.cuh"

namespace kvc {

namespace {

constexpr int KEYS = 128, PAGES = KEYS / PS;       // of a step
constexpr int TOKENS = 32;                         // of a tile
constexpr int PANEL = KEYS * 128;                  // 128 rows x 64 columns
constexpr int SLOT = 2 * PANEL;                    // a tile: 32 KiB
constexpr int TC_THREADS = 512;
constexpr int FEW_REGS = 96, MANY_REGS = 160;      // 256 threads each: what 128 a thread make together

__device__ inline void tc_mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                 uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ inline void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_u32(bar))
      : "memory");
}
template <int N>
__device__ inline void give_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ inline void take_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// Bounded wait that also ends when another warp has given up.
__device__ inline bool wait_or_stop(const Dev& d, uint64_t* bar, uint32_t parity, volatile int* stop) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (*stop) return false;
    if (clock64() - t0 > WAIT_LIMIT_CYCLES) {
      set_error(d, KVC_DERR_WAIT);
      *stop = 1;
      return false;
    }
  }
  return true;
}

// Blocks that the tokens up to `tok` of the chunk see.
__device__ inline int blocks_seen(const SeqInfo& si, int tok) {
  return si.n_hist_pages + (si.live_head + si.n_live - si.t + tok) / PS + 1;
}

// Whether a step (blocks [b0, b0 + PAGES)) has slots that some row of the item starting at token t0 does
// not see: a partly filled page, pages past the end, keys behind the item's first token.
__device__ inline bool is_edge(const SeqInfo& si, int t0, int b0) {
  const int nhp = si.n_hist_pages;
  const int first = nhp + (si.live_head + si.n_live - si.t + t0) / PS;  // block of the first token
  if (b0 + PAGES > first) return true;
  const int b_hist = (si.n_hist % PS) ? nhp - 1 : -1, b_live = si.live_head ? nhp : -1;
  return (b_hist >= b0 && b_hist < b0 + PAGES) || (b_live >= b0 && b_live < b0 + PAGES);
}

// Slots [lo, hi) of block b that hold a position with index <= q_log.
__device__ inline uint32_t slots_seen(const SeqInfo& si, int b, int n_blocks, int q_log) {
  if (b >= n_blocks) return 0;
  const BlockRange br = block_range(si, b);
  const int hi = min(br.hi, q_log - br.base + 1);
  return hi <= br.lo ? 0u : ((1u << hi) - 1u) & ~((1u << br.lo) - 1u);
}

// Query rows of tokens [t0, t0 + TOKENS) of one KV head by the 128 threads `ts`: rotated, scaled and
// rounded into the swizzled tile at `to`; PIECES = 2: what rounding left, rounded too, into the tile
// behind it.  Rows past the chunk are zero.  `free` waits until the tile may be written (false: give up).
// A thread takes 16-byte chunks c and c + 8 (which rotate together) of a token's G rows.
template <int PIECES, typename FreeFn>
__device__ inline void stage_q(const Dev& d, const SeqInfo& si, int head, int t0, const __nv_bfloat16* q,
                               float qk_scale, uint8_t* to, int ts, FreeFn free) {
  const int c = ts & 7;
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    const int tl = (ts >> 3) + 16 * h, tok = t0 + tl;
    uint4 a[G], b[G];
    float4 cs[4];
    const bool in = tok < si.t;
    if (in) {
      const uint4* row = reinterpret_cast<const uint4*>(
          q + ((size_t)(si.q_row0 + tok) * d.q_heads + head * G) * D) + c;
      const float4* t4 = reinterpret_cast<const float4*>(d.rope + (size_t)(si.pos_first + tok) * (D / 2) + c * 8);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        a[g] = row[g * 16];
        b[g] = row[g * 16 + 8];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) cs[e] = t4[e];
    }
    if (h == 0 && !free()) return;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      uint32_t ya[PIECES][4] = {}, yb[PIECES][4] = {};
      if (in) {
        const uint32_t ua[4] = {a[g].x, a[g].y, a[g].z, a[g].w};
        const uint32_t ub[4] = {b[g].x, b[g].y, b[g].z, b[g].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a0 = bf16lo(ua[e]), a1 = bf16hi(ua[e]), b0 = bf16lo(ub[e]), b1 = bf16hi(ub[e]);
          const float x0 = fmaf(a0, cs[e].x, -b0 * cs[e].y) * qk_scale;
          const float x1 = fmaf(a1, cs[e].z, -b1 * cs[e].w) * qk_scale;
          const float y0 = fmaf(b0, cs[e].x, a0 * cs[e].y) * qk_scale;
          const float y1 = fmaf(b1, cs[e].z, a1 * cs[e].w) * qk_scale;
          ya[0][e] = pack_bf16(x0, x1);
          yb[0][e] = pack_bf16(y0, y1);
          if constexpr (PIECES == 2) {
            ya[1][e] = pack_bf16(x0 - bf16lo(ya[0][e]), x1 - bf16hi(ya[0][e]));
            yb[1][e] = pack_bf16(y0 - bf16lo(yb[0][e]), y1 - bf16hi(yb[0][e]));
          }
        }
      }
      const int r = tl * G + g;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        uint8_t* at = to + p * SLOT + r * 128 + ((c ^ (r & 7)) << 4);
        *reinterpret_cast<uint4*>(at) = make_uint4(ya[p][0], ya[p][1], ya[p][2], ya[p][3]);
        *reinterpret_cast<uint4*>(at + PANEL) = make_uint4(yb[p][0], yb[p][1], yb[p][2], yb[p][3]);
      }
    }
  }
}

// First item of each session, and the number of all behind the last: sums of count(session) (one warp).
template <typename CountFn>
__device__ inline void first_items(int n_seq, int lane, int* first, CountFn count) {
  int sum = 0;
  for (int i0 = 0; i0 < n_seq; i0 += 32) {
    const int i = i0 + lane, n = i < n_seq ? count(i) : 0;
    int x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(FULL, x, o);
      if (lane >= o) x += y;
    }
    if (i < n_seq) first[i] = sum + x - n;
    sum += __shfl_sync(FULL, x, 31);
  }
  if (lane == 0) first[n_seq] = sum;
}

// Session that item `at` belongs to.
__device__ inline int session_of(int n_seq, const int* first, int at) {
  int lo = 0, hi = n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= at) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Boxes of a tile of up to PAGES pages (16 rows x 64 columns each) by lanes 0 .. 15 of a warp: lane
// 2 pg + h has half h of page pg, whose id it is given.
__device__ inline void load_tile(const Dev& d, int layer, int kv, int head, int page, int n_pg, uint8_t* to,
                                 const CUtensorMap* map, uint64_t* bar, int lane) {
  const int pg = lane >> 1 & 7;
  if (lane < 16 && pg < n_pg)
    tma_load_2d(to + (lane & 1) * PANEL + pg * 2048, map, 0,
                (((page * d.layers + layer) * 2 + kv) * d.kv_heads + head) * PS, bar);
}

}  // namespace

}  // namespace kvc
