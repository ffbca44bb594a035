// What the tensor-core kernels of whole prompts share: tiles of 128 rows (32 tokens x 4 query heads of a
// KV head, or 128 keys) by 128 dims, their products, waits, masks and work lists.
#pragma once

#include "kvc_prefill_tc.cuh"
#include "kvc_prompt_list.cuh"

namespace kvc {

namespace {

constexpr int KEYS = 128, PAGES = KEYS / PS;       // of a step
constexpr int TOKENS = 32;                         // of a tile
constexpr int SLOT = KEYS * D * 2;                 // a tile: 32 KiB
// A tile is 16 groups of 8 rows; a group holds columns 0-63, then 64-127 of its rows, 1 KiB each with
// 128-byte swizzle: what one copy brings of a page (16 rows) is then 4 KiB of the tile as it stands.
constexpr int ATOM = 1024, ROW_GROUP = 2 * ATOM;
// Byte offset in a tile of 16-byte chunk c (0 .. 15) of row r.
__device__ inline uint32_t tile_at(int r, int c) {
  return (r >> 3) * ROW_GROUP + (c >> 3) * ATOM + (r & 7) * 128 + (((c & 7) ^ (r & 7)) << 4);
}
// Descriptors of a tile as an operand whose K dimension is its columns (K-major), and whose K dimension
// is its rows (MN-major); the 16 columns or rows of a step lie step_columns(kk) or 2 ROW_GROUP kk on.
__device__ inline uint64_t desc_columns(uint32_t tile) { return smem_desc(tile, 0, ROW_GROUP); }
__device__ inline uint64_t desc_rows(uint32_t tile) { return smem_desc(tile, ATOM, ROW_GROUP); }
__host__ __device__ constexpr uint32_t step_columns(int kk) { return (kk >> 2) * ATOM + (kk & 3) * 32; }
__device__ inline void tc_mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                 uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// 32 columns of this thread's tensor-memory lane on their way into r, and there.
__device__ inline void tmem_ld32_begin(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ inline void tmem_ld32_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
// 16 columns on their way to tensor memory, and all of them there.
__device__ inline void tmem_st16_begin(uint32_t taddr, const uint32_t (&w)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11]), "r"(w[12]), "r"(w[13]), "r"(w[14]), "r"(w[15])
               : "memory");
}
__device__ inline void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ inline void tma_load_tile(void* dst, const CUtensorMap* map, int group, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %2, %2, %3}], [%4];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(group), "r"(smem_u32(bar))
      : "memory");
}
// Bounded wait that also ends when another warp has given up.  Its loop is out of line: a role's code has to
// stay in the instruction caches (16,384 tokens 1,657 us with the loop at each wait, 1,617 without).
__device__ __noinline__ bool keep_waiting(const Dev& d, uint64_t* bar, uint32_t parity, volatile int* stop) {
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
__device__ inline bool wait_or_stop(const Dev& d, uint64_t* bar, uint32_t parity, volatile int* stop) {
  if (mbar_try_wait(bar, parity)) return true;
  return keep_waiting(d, bar, parity, stop);
}

// Steps (of PAGES blocks) with slots that some row of the item starting at token t0 does not see: a
// partly filled page, pages past the end, keys behind the item's first token.
struct EdgeSteps {
  int diag, hist, live;
  __device__ bool at(int j) const { return j >= diag || j == hist || j == live; }
  // Counted from a step on (those before it are below 0).
  __device__ void from(int j) {
    diag -= j;
    hist -= j;
    live -= j;
  }
};
__device__ inline EdgeSteps edge_steps(const SeqInfo& si, int t0) {
  const int nhp = si.n_hist_pages;
  return {(nhp + (si.live_head + si.n_live - si.t + t0) / PS) / PAGES,
          (si.n_hist % PS) ? (nhp - 1) / PAGES : -1, si.live_head ? nhp / PAGES : -1};
}

// Query rows of tokens [t0, t0 + TOKENS) of one KV head by the N threads `ts`: rotated, scaled and
// rounded into the swizzled tile at `to`; PIECES = 2: what rounding left, rounded too, into the tile
// behind it.  Rows past the chunk are zero.  `free` waits until the tile may be written (false: give up).
// A thread takes 16-byte chunks c and c + 8 (which rotate together) of a token's G rows.
template <int PIECES, int N, typename FreeFn>
__device__ inline void stage_q(const Dev& d, const SeqInfo& si, int head, int t0, const __nv_bfloat16* q,
                               float qk_scale, uint8_t* to, int ts, FreeFn free) {
  const int c = ts & 7;
#pragma unroll 1
  for (int step = 0; step < TOKENS * 8 / N; ++step) {
    const int tl = (ts >> 3) + N / 8 * step, tok = t0 + tl;
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
    if (step == 0 && !free()) return;
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
        uint8_t* at = to + p * SLOT + tile_at(r, c);
        *reinterpret_cast<uint4*>(at) = make_uint4(ya[p][0], ya[p][1], ya[p][2], ya[p][3]);
        *reinterpret_cast<uint4*>(at + ATOM) = make_uint4(yb[p][0], yb[p][1], yb[p][2], yb[p][3]);
      }
    }
  }
}

// A tile of up to PAGES pages by lanes 0 .. 7 of a warp, which have the id of a page each.
__device__ inline void load_tile(const Dev& d, int layer, int kv, int head, int page, int n_pg, uint8_t* to,
                                 const CUtensorMap* map, uint64_t* bar, int lane) {
  if (lane < n_pg)
    tma_load_tile(to + lane * PS * D * 2, map,
                  (((page * d.layers + layer) * 2 + kv) * d.kv_heads + head) * (PS / 8), bar);
}

}  // namespace

}  // namespace kvc
