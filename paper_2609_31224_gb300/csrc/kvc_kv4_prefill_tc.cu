// Chunked-prefill attention over a cache held in 4 bits (KVC_KV4), bfloat16 calls, on the
// 5th-generation tensor cores (tcgen05 + TMEM).
//
// The T * G query rows of a (session, KV head) pair (T <= 32 tokens, G = 4 heads) are the M = 128
// rows of the products S = Q K^T and O += P V, 128 keys (8 pages) a stage.  Operands are binary16:
// K and V exactly the numbers that the codes stand for (over 16, kvc_kv4.h), q and P rounded to 11
// bits; accumulation and softmax in binary32.  Rounding and masks are those of kvc_kv4_decode.cu:
// q rows over a power of two, P = exp2(s - m + 8) with a lagging reference m, masked keys of weight
// 0, invalid slots of value 0.  A V group that stands for NaN and that not every row sees is held as
// 0 and its first place noted; the rows that see it get NaN when they are written.
//
// Each pair's pages are cut into k slices of whole stages, one CTA each; the k CTAs of a pair are a
// thread-block cluster and merge their partial rows through distributed shared memory.
//
// Warps of a CTA (608 threads, one CTA per SM):
//   0-7    softmax: warps w and w + 4 own TMEM lanes 32 w .. 32 w + 31, a query row per lane; warp
//          w takes the first 64 keys of a stage, warp w + 4 the others.  They rotate the rows into
//          TMEM, then turn rows of S into rows of P (written over them), keep maximum and sum, and
//          write the output.  The two threads of a row share its reference m: a vote of their warps
//          tells each stage whether it still holds;
//   8-15   operands: warp 8 + i unpacks page i of a stage, K and V, into 128-byte-swizzled tiles.
//          Dims and nibbles keep their stored order (the query's dims take K's, the output's are put
//          back in order), so that a word of eight codes becomes one 16-byte store; the order of the
//          stores of a warp is chosen so that eight lanes in a row hit all banks;
//   16     copies the raw pages (18 D bytes each, K and V) into a ring of 3 stages;
//   17, 18 issue S = Q K^T (Q from TMEM) and O += P V (P from TMEM, V read along its keys).
// Every wait is bounded; a timeout records KVC_DERR_WAIT and the CTA stops.
//
// What bounds it: 64 sessions of 4,096 positions and 17 tokens read 47 us of bytes, the products are
// 73 us at the measured rate (68 of their 128 rows are tokens), and about 6,000 warp instructions a stage,
// 2,000 of them the unpacking, 1,300 the weights, hold 53 % of the issue slots: 1.15 us a stage.  Measured
// 169 us a layer (233 as first written; 168 over bfloat16 rows, whose operands need no unpacking), one
// session 15.7 us (12.5), 9 sessions 30 us (30).  Few sessions take 2 to 3 us more than over bfloat16
// rows whatever their length (one of 100 positions 7.6 and 5.8, of 8,000 18.9 and 16.3): not the stages,
// but what each CTA does once.  Larger stages pay: at 96 keys the hops between the roles cost
// 15 % more; softmax warps of 64 columns each beat four of 128 by a seventh.
#include <cuda.h>

#include <algorithm>

#include "kvc_kv4.cuh"
#include "kvc_prefill_tc.cuh"

namespace kvc {

namespace {

using namespace kv4;

constexpr int KEYS = 128;                       // of a stage
constexpr int PAGES = KEYS / PS;
constexpr int PAGE = 18 * D;                    // raw bytes of a page of one head, K and V
constexpr int PANEL = KEYS * 128;               // 128 rows of 64 binary16 numbers
constexpr int TILE = 2 * PANEL;                 // K or V of a stage
constexpr int RAW = 3;                          // raw stages in the ring
constexpr int SM_WARPS = 8, OP_WARPS = PAGES, SM_THREADS = 32 * SM_WARPS;
constexpr int W_OP = SM_WARPS, W_LOAD = W_OP + OP_WARPS, W_S = W_LOAD + 1, W_PV = W_S + 1;
constexpr int THREADS = (W_PV + 1) * 32;
constexpr float P_SHIFT = 8.f;                   // as in the decode kernel

// Tensor memory: S of even and odd stages (128 fp32 columns each; P of each 64 keys, 32 columns of
// pairs, over their first half), O (128), Q (64).
constexpr int TMEM_COLS = 512, S_COL = 0, O_COL = 256, Q_COL = 384;

enum {
  B_RAW_FULL = 0,                  // [RAW] raw pages of a stage copied
  B_RAW_EMPTY = B_RAW_FULL + RAW,  // [RAW] ... and unpacked
  B_K_FULL = B_RAW_EMPTY + RAW,    // [2] K tile of a stage written
  B_K_EMPTY = B_K_FULL + 2,        // [2] ... and read by S = Q K^T
  B_V_FULL = B_K_EMPTY + 2,
  B_V_EMPTY = B_V_FULL + 2,
  B_S_FULL = B_V_EMPTY + 2,        // [2] scores complete
  B_P_FULL = B_S_FULL + 2,         // [2] weights written
  B_PV = B_P_FULL + 2,             // [2] O += P V complete (and S, P of the stage free)
  B_Q = B_PV + 2,                  // query rows in TMEM
  B_FINAL = B_Q + 1,               // [2] the products of an issuer complete
  N_BARS = B_FINAL + 2
};
// Shared memory from a 1024-aligned base: K tiles, V tiles, raw ring, barriers.  The partial rows of
// a slice take the place of the tiles when its products are complete.
constexpr int OFF_K = 0, OFF_V = OFF_K + 2 * TILE, OFF_RAW = OFF_V + 2 * TILE;
// Query rows on their way to TMEM (padded: 8 lanes read 8 rows without a conflict).
constexpr int Q_PITCH = 2 * D + 16;
constexpr int OFF_Q = OFF_RAW + RAW * PAGES * PAGE;
constexpr int OFF_ROW = OFF_Q + M * Q_PITCH;    // [M] softmax scales, then [2][M] exchanged values
constexpr int OFF_BAR = OFF_ROW + 3 * M * 4;
constexpr int OFF_TMEM = OFF_BAR + N_BARS * 8;
constexpr int OFF_NAN = OFF_TMEM + 8;           // [D / GROUP] first retained index of a NaN group
constexpr int SMEM = 1024 + OFF_NAN + D / GROUP * 4;
constexpr int ROW_PITCH = (D + 4) * 4;          // a partial row: D values, then (m, l, c)
static_assert(OFF_BAR % 8 == 0 && PAGE % 16 == 0 && M * ROW_PITCH <= 4 * TILE, "layout");
static_assert(SMEM <= 227 * 1024 - 256, "fits");

// Instruction descriptor, kind::f16: D fp32, A and B binary16, A K-major, B K- or MN-major.
__host__ __device__ constexpr uint32_t f16_desc(int n, int m, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}

__device__ inline void sts128(uint32_t at, const uint32_t (&v)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3])
               : "memory");
}

// The pages of a slice: blocks [blk0, blk0 + nblk) of a pair.
struct Slice {
  SeqInfo si;
  int seq, head, blk0, nblk;
  __device__ int stages() const { return (nblk + PAGES - 1) / PAGES; }
  __device__ int last0() const { return si.n_hist + si.n_live - si.t; }  // of the first token
  __device__ int first_new() const { return si.n_hist_pages + (si.live_head + si.n_live - si.t) / PS; }
  // Whether every row sees every slot of pages [b, b + n) of the pair: full pages of the history, or
  // full pages of the live part up to the first token's key.
  __device__ bool open(int b, int n) const {
    const int first = si.n_hist_pages;
    if (b + n <= first) return (b + n) * PS <= min(si.n_hist, last0() + 1);
    return b >= first && block_range(si, b).lo == 0 && block_range(si, b + n - 1).base + PS - 1 <= last0();
  }
};

// K tile rows of page i of a stage from its raw tile (shared addresses): lane (x, t) takes words
// [4 t, 4 t + 4) of rows r and r + 8.
__device__ inline void unpack_k(uint32_t raw, uint32_t tile, int i, bool open, const BlockRange& br,
                                int lane) {
  const int x = lane >> 2, t = lane & 3;
  const int r0 = (x & 4) | (x & 1) << 1 | (x >> 1 & 1);  // rows two apart side by side
  const int turn = t >> 1;                               // this lane's words in the places w ^ turn
  const __half2 m72 = __float2half2_rn(-72.f);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = r0 + 8 * j;
    uint32_t w[4], m[2];
    lds(raw + k_codes(D, row, 8 * t), w);
    lds(raw + k_scale(D, row, 0), m);
    if (!open && (row < br.lo || row >= br.hi)) m[0] = m[1] = 0u;
    const uint32_t to = tile + turn * PANEL + (PS * i + row) * 128;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const __half2 mm = s & 1 ? __high2half2(bits_h2(m[s / 2])) : __low2half2(bits_h2(m[s / 2]));
      uint32_t v[4];
      pairs_of(w[s], mm, __hmul2(mm, m72), v);
      sts128(to + (((4 * (t & 1) + (s ^ turn)) ^ (row & 7)) << 4), v);
    }
  }
}

// V tile rows of page i of a stage: lane (g, t) takes piece g of rows 2t, 2t + 1 (+ 8).
__device__ inline void unpack_v(uint32_t raw, uint32_t tile, int i, bool open, const BlockRange& br,
                                int last0, int* nan_at, int lane) {
  const int g = lane >> 2, t = lane & 3, turn = g & 1;   // this lane's words in the places s ^ turn
  const __half2 m72 = __float2half2_rn(-72.f);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row0 = 2 * t + 8 * h, group = g * (D / 8) / GROUP;
    uint32_t w[4], m;
    lds(raw + v_piece(D, row0, g), w);
    lds(raw + v_scale(D, row0, group), m);
    if (!open) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool valid = row0 + k >= br.lo && row0 + k < br.hi;
        const bool is_nan = (m >> (16 * k) & 0x7FFFu) > 0x7C00u;
        if (valid && is_nan && br.base + PS - 1 > last0) atomicMin(&nan_at[group], br.base + row0 + k);
        if (!valid || (is_nan && br.base + PS - 1 > last0)) m &= k ? 0x0000FFFFu : 0xFFFF0000u;
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = row0 + k;
      const __half2 mm = k ? __high2half2(bits_h2(m)) : __low2half2(bits_h2(m)), mb = __hmul2(mm, m72);
      const uint32_t to = tile + (g >> 2) * PANEL + (PS * i + row) * 128;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint32_t v[4];
        pairs_of(w[2 * k + s], mm, mb, v);
        sts128(to + (((2 * (g & 3) + (s ^ turn)) ^ (row & 7)) << 4), v);
      }
    }
  }
}

// The chunk's query rows into their staging rows: rotated, over a power of two (largest element in
// [1, 2); infinities and NaN pass through), dims in K's stored order; a row's softmax scale beside.
// Item (row, c): dims [8c, 8c + 8) and their rotate-half partners; 8 lanes a row.
__device__ inline void stage_queries(const Dev& d, const SeqInfo& si, int head,
                                     const __nv_bfloat16* q, uint8_t* rows, float* scale, int tid) {
  constexpr int HALF = D / 2, KC = D / 16, BATCH = 2;
  const int n = si.t * G * KC;
  for (int i0 = 0; i0 < n; i0 += BATCH * SM_THREADS) {
    uint4 a[BATCH], b[BATCH];
    float4 cs[BATCH][4];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int i = min(i0 + u * SM_THREADS + tid, n - 1), r = i / KC, c = i % KC;
      const uint4* row = reinterpret_cast<const uint4*>(
          q + ((size_t)(si.q_row0 + r / G) * d.q_heads + head * G + r % G) * D);
      a[u] = row[c];
      b[u] = row[c + KC];
      const float4* t4 = reinterpret_cast<const float4*>(d.rope + (size_t)(si.pos_first + r / G) * HALF + 8 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) cs[u][e] = t4[e];
    }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int i = i0 + u * SM_THREADS + tid, r = min(i, n - 1) / KC, c = min(i, n - 1) % KC;
      float x1[8], x2[8], y1[8], y2[8];
      Chunk16<__nv_bfloat16>::unpack(a[u], x1);
      Chunk16<__nv_bfloat16>::unpack(b[u], x2);
      uint32_t most = 0;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float4 t = cs[u][e / 2];
        turn_pair(x1[e], x2[e], make_float2(t.x, t.y), y1[e], y2[e]);
        turn_pair(x1[e + 1], x2[e + 1], make_float2(t.z, t.w), y1[e + 1], y2[e + 1]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, max(abs_bits(y1[e]), abs_bits(y2[e])));
      // (Rows are whole within a warp, and n is a multiple of 32: lanes past it repeat the last
      // item together.)
#pragma unroll
      for (int o = 1; o < KC; o <<= 1) most = max(most, __shfl_xor_sync(FULL, most, o));
      int e = (int)(most >> 23) - 127;
      e = e > 126 ? (e == 128 ? 0 : 126) : max(e, -126);
      const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
      if (i >= n) continue;
      // 16: scales are stored over 16; the softmax takes exponents of 2.
      if (c == 0)
        scale[r] = 16.f * LOG2E * 0.08838834764831845f * __uint_as_float((uint32_t)(127 + e) << 23);
      uint32_t u1[4], u2[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        u1[p] = h2_bits(__floats2half2_rn(y1[p] * inv, y1[p + 4] * inv));
        u2[p] = h2_bits(__floats2half2_rn(y2[p] * inv, y2[p + 4] * inv));
      }
      // Dims 8 c are word w = c / 4 of t = c % 4, the partners word w + 2.
      // (In the places of unpack_k: w ^ (t / 2); the partner's place differs in bit 1.)
      const int place = 4 * (c % 4) + ((c / 4) ^ (c % 4 / 2));
      uint8_t* to = rows + r * Q_PITCH + place * 16;
      *reinterpret_cast<uint4*>(to) = make_uint4(u1[0], u1[1], u1[2], u1[3]);
      *reinterpret_cast<uint4*>(rows + r * Q_PITCH + (place ^ 2) * 16) = make_uint4(u2[0], u2[1], u2[2], u2[3]);
    }
  }
}

// Weight of a state with reference m against the reference m2 of several.
__device__ inline float weight2(float m, float m2, float c) {
  return m == -INFINITY ? 0.f : ex2((m - m2) * c);
}

__device__ inline void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ inline void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ inline uint32_t cluster_map(uint32_t saddr, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ inline float4 ld_cluster(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(at)
               : "memory");
  return v;
}

// Dims [8 c, 8 c + 8) of an output row from its columns in the tiles' order.
__device__ inline void in_order(const float* o, float f, float (&y)[8]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    y[p] = o[2 * p] * f;
    y[p + 4] = o[2 * p + 1] * f;
  }
}

__global__ void __launch_bounds__(THREADS, 1) prefill_kv4_kernel(
    Dev d, int layer, const __nv_bfloat16* __restrict__ q, __nv_bfloat16* __restrict__ out,
    int pair0, int k_slices, Early early) {
  extern __shared__ uint8_t smem_raw[];
  // (The same offset in every CTA, so that cluster_map() of an address finds the peer's.)
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_TMEM);
  int* nan_at = reinterpret_cast<int*>(smem + OFF_NAN);
  __shared__ int s_abort_flag;
  volatile int& s_abort = s_abort_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // The first call after an append waits for it (and lets nothing else start before that).
  if (early == EARLY_NONE) pdl_wait();
  if (d.g->n_units == 0) {  // the append failed: nothing to do for any CTA
    pdl_wait();
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < RAW; ++i) {
      mbar_init(&bars[B_RAW_FULL + i], 1);
      mbar_init(&bars[B_RAW_EMPTY + i], OP_WARPS);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars[B_K_FULL + i], OP_WARPS);
      mbar_init(&bars[B_K_EMPTY + i], 1);
      mbar_init(&bars[B_V_FULL + i], OP_WARPS);
      mbar_init(&bars[B_V_EMPTY + i], 1);
      mbar_init(&bars[B_S_FULL + i], 1);
      mbar_init(&bars[B_P_FULL + i], SM_WARPS);
      mbar_init(&bars[B_PV + i], 1);
      mbar_init(&bars[B_FINAL + i], 1);
    }
    mbar_init(&bars[B_Q], SM_WARPS);
    fence_mbar_init();
    s_abort = 0;
  }
  if (tid < D / GROUP) nan_at[tid] = 1 << 30;
  __syncwarp();
  if (warp == W_S) tmem_alloc(tmem_slot, TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();
  const uint32_t sbase = smem_u32(smem);

  Slice sl;
  const int pair = pair0 + blockIdx.x / k_slices, slice = blockIdx.x % k_slices;
  sl.seq = pair / d.kv_heads;
  sl.head = pair % d.kv_heads;
  sl.si = d.seq[sl.seq];
  const SeqInfo& si = sl.si;
  {
    const int all = (si.n_blocks + PAGES - 1) / PAGES;
    sl.blk0 = min(si.n_blocks, PAGES * (int)((int64_t)slice * all / k_slices));
    sl.nblk = min(si.n_blocks, PAGES * (int)((int64_t)(slice + 1) * all / k_slices)) - sl.blk0;
  }
  const int n_st = sl.stages(), last0 = sl.last0(), R = si.t * G;
  // A wait that gives up stops its warp; the others follow when their own waits do.
  auto wait = [&](int bar, uint32_t parity) {
    const bool ok = __all_sync(FULL, mbar_wait(d, &bars[bar], parity & 1));
    if (!ok && lane == 0) s_abort = 1;
    return ok;
  };
  // This thread's partial row: reference, sum of its keys, softmax scale (softmax warps).
  float m = -INFINITY, l = 0.f, c = 0.f;
  bool dead = false;
  const int quarter = warp & 3, half = warp >> 2 & 1;
  float* s_row = reinterpret_cast<float*>(smem + OFF_ROW);
  // The two warps of a quarter (named barriers 1-4), all softmax warps (5).
  auto sync_quarter = [&] {
    __syncwarp();
    asm volatile("bar.sync %0, 64;" ::"r"(1 + quarter) : "memory");
  };

  // ... and whether a thread of either has x.
  auto quarter_any = [&](bool x) {
    uint32_t any;
    __syncwarp();
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "bar.red.or.pred q, %2, 64, p;\n"
        "selp.u32 %0, 1, 0, q;\n"
        "}"
        : "=r"(any)
        : "r"((uint32_t)x), "r"(1 + quarter)
        : "memory");
    return any != 0;
  };

  if (warp < SM_WARPS) {
    // ---------------- softmax ----------------
    const int r = 32 * quarter + lane;
    const bool live = r < R, idle = 32 * quarter >= R;
    const uint32_t trow = tmem + ((uint32_t)(32 * quarter) << 16);
    pdl_wait();
    stage_queries(d, si, sl.head, q, smem + OFF_Q, s_row, tid);
    __syncwarp();
    asm volatile("bar.sync 5, %0;" ::"n"(SM_THREADS) : "memory");
    {
      // This thread's half of its row's 64 columns of pairs; padding rows are zeros.
      uint32_t u[32];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const uint4 w = live ? *reinterpret_cast<const uint4*>(smem + OFF_Q + r * Q_PITCH + 128 * half + 16 * x)
                             : make_uint4(0, 0, 0, 0);
        u[4 * x] = w.x;
        u[4 * x + 1] = w.y;
        u[4 * x + 2] = w.z;
        u[4 * x + 3] = w.w;
      }
      __syncwarp();
      tmem_st32(trow + Q_COL + 32 * half, u);
      c = live ? s_row[r] : 0.f;
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars[B_Q]);
    const int last = last0 + r / G;  // retained index of the last key that the row sees
    constexpr int HK = KEYS / 2, HP = PAGES / 2;
    for (int i = 0; i < n_st; ++i) {
      const int b = i & 1;
      dead = dead || !wait(B_S_FULL + b, i >> 1);
      tc_fence_after();
      if (idle) {  // padding rows: whatever their P is, it stays in their rows of O
        if (dead) break;
        if (lane == 0) mbar_arrive(&bars[B_P_FULL + b]);
        continue;
      }
      const uint32_t ts = trow + S_COL + KEYS * b + HK * half;
      const int b0 = sl.blk0 + PAGES * i + HP * half, npg = sl.nblk - PAGES * i - HP * half;
      const bool open = npg >= HP && sl.open(b0, HP);
      // Slots of page pg that the row sees.
      auto seen = [&](int pg, int& lo, int& hi) {
        const BlockRange br = block_range(si, b0 + pg);
        lo = br.lo;
        hi = pg < npg ? min(br.hi, last - br.base + 1) : 0;
      };
      uint32_t pw[HK / 2];
      float sum = 0.f;
      auto weigh = [&] {
        float2 rs[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        const float2 c2 = make_float2(c, c), sh = make_float2(P_SHIFT, P_SHIFT);
        const float2 nm = make_float2(-m, -m);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          float s[32];
          tmem_ld32(ts + 32 * part, s);
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            const float2 a = __ffma2_rn(__fadd2_rn(make_float2(s[k], s[k + 1]), nm), c2, sh);
            s[k] = a.x;
            s[k + 1] = a.y;
          }
          if (!open) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              int lo, hi;
              seen(2 * part + h, lo, hi);
#pragma unroll
              for (int k = 0; k < PS; ++k)
                if (k < lo || k >= hi) s[PS * h + k] = -INFINITY;
            }
          }
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            const float2 p = make_float2(ex2(s[k]), ex2(s[k + 1]));
            rs[(k / 2) & 1] = __fadd2_rn(rs[(k / 2) & 1], p);
            pw[16 * part + k / 2] = h2_bits(__floats2half2_rn(p.x, p.y));
          }
        }
        sum = (rs[0].x + rs[1].x) + (rs[0].y + rs[1].y);
      };
      // A new reference where the weights' sum passes 2^15 (so no weight passes what binary16 holds;
      // under a reference that is the largest score the 64 weights are at most 2^14 together), and at
      // the first stage: a test of the sum in place of a maximum of 64 scores.  Both
      // warps take every barrier of a stage, and leave together when a wait of either gave up.
      bool need = false;
      if (i > 0 && !dead) {
        weigh();
        need = live && sum > 32768.f;
      }
      const bool any = quarter_any(dead || need);
      if (any) dead = quarter_any(dead);
      if (dead) break;
      const bool fresh = i == 0 || any;
      if (fresh) {
        float mx = -INFINITY;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          float s[32];
          tmem_ld32(ts + 32 * part, s);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            int lo, hi;
            seen(2 * part + h, lo, hi);
#pragma unroll
            for (int k = 0; k < PS; ++k)
              if (k >= lo && k < hi) mx = fmaxf(mx, s[PS * h + k]);
          }
        }
        s_row[M * (1 + half) + r] = mx;
        sync_quarter();
        const float mn = fmaxf(m, fmaxf(mx, s_row[M * (2 - half) + r]));
        const float f = weight2(m, mn, c);
        if (i > 0) {
          // The products so far are complete: this thread's half of the row's columns is scaled.
          dead = !wait(B_PV + (b ^ 1), (i - 1) >> 1);
          tc_fence_after();
          if (!dead) {
#pragma unroll 1
            for (int x = 0; x < D / 32; ++x) {
              float o[16];
              tmem_ld16(trow + O_COL + D / 2 * half + 16 * x, o);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] *= f;
              tmem_st16(trow + O_COL + D / 2 * half + 16 * x, o);
            }
          }
        }
        l *= f;
        m = mn;
        if (!dead) weigh();
        // (Both have read the other's maximum before either writes one again.)
        dead = quarter_any(dead);
        if (dead) break;
      }
      l += sum;
      __syncwarp();
      tmem_st32(ts, pw);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_P_FULL + b]);
    }
    if (n_st > 0 && !dead) dead = !wait(B_PV + ((n_st - 1) & 1), (n_st - 1) >> 1);
    tc_fence_after();
    s_row[M * (1 + half) + r] = l;
  } else if (warp < W_LOAD) {
    // ---------------- operands ----------------
    const int pg = warp - W_OP;
    for (int i = 0; i < n_st; ++i) {
      const int slot = i % RAW, b = i & 1;
      if (!wait(B_RAW_FULL + slot, i / RAW)) break;
      const uint32_t raw = sbase + OFF_RAW + (slot * PAGES + pg) * PAGE;
      const int blk = sl.blk0 + PAGES * i + pg;
      const bool here = blk < sl.blk0 + sl.nblk;
      const BlockRange br = block_range(si, here ? blk : sl.blk0);
      const bool open = here && sl.open(blk, 1);
      if (i >= 2 && !wait(B_K_EMPTY + b, (i >> 1) - 1)) break;
      // (A page that is not there: its scores are masked whatever K holds.)
      if (here) unpack_k(raw, sbase + OFF_K + b * TILE, pg, open, br, lane);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_K_FULL + b]);
      if (i >= 2 && !wait(B_V_EMPTY + b, (i >> 1) - 1)) break;
      if (here) {
        unpack_v(raw + 9 * D, sbase + OFF_V + b * TILE, pg, open, br, last0, nan_at, lane);
      } else {
        // Weight 0 times what the tile held must be 0.
        const uint32_t zero[4] = {0u, 0u, 0u, 0u};
        const uint32_t at = sbase + OFF_V + b * TILE + PS * pg * 128 + lane * 16;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          sts128(at + x * 512, zero);
          sts128(at + PANEL + x * 512, zero);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&bars[B_V_FULL + b]);
        mbar_arrive(&bars[B_RAW_EMPTY + slot]);
      }
    }
  } else if (warp == W_LOAD) {
    // ---------------- raw pages ----------------
    const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
    const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
    const uint8_t* tiles = d.pool + tile_at(D, d.layers, d.kv_heads, 0, layer, sl.head, 0);
    const size_t stride = page_bytes(D, d.layers, d.kv_heads);
    const uint64_t policy = evict_first_policy();
    // Page ids, one to a lane, asked for 32 at a time a whole group ahead of the copies that use them.
    auto ids_at = [&](int b) { return b < sl.nblk ? block_page(si, hrow, lrow, sl.blk0 + b) : 0; };
    constexpr int PER = 32 / PAGES;
    int done = 0, ids = ids_at(lane), ahead = ids_at(32 + lane);
    {
      // The query rows (1 KiB a token) and rotary rows (512 B) into L2 ahead of the softmax warps.
      const char* qb = reinterpret_cast<const char*>(q + ((size_t)si.q_row0 * d.q_heads + sl.head * G) * D);
      const char* rb = reinterpret_cast<const char*>(d.rope + (size_t)si.pos_first * (D / 2));
      for (int x = lane; x < si.t * 12; x += 32) {
        const int t = x / 12, line = x % 12;
        prefetch_l2(line < 8 ? qb + (size_t)t * d.q_heads * D * 2 + line * 128
                             : rb + (size_t)t * 512 + (line - 8) * 128);
      }
    }
    for (int i = 0; i < n_st; ++i) {
      const int slot = i % RAW, npg = min(PAGES, sl.nblk - PAGES * i);
      if (i > 0 && i % PER == 0) {
        ids = ahead;
        ahead = ids_at(PAGES * i + 32 + lane);
      }
      const int page = __shfl_sync(FULL, ids, PAGES * (i % PER) + lane % PAGES);
      if (early == EARLY_OLD && sl.blk0 + PAGES * i + npg > sl.first_new()) pdl_wait();
      if (i >= RAW && !wait(B_RAW_EMPTY + slot, i / RAW - 1)) break;
      if (lane == 0) mbar_arrive_expect_tx(&bars[B_RAW_FULL + slot], npg * PAGE);
      __syncwarp();
      if (lane < npg) {
        fence_proxy_async_smem();
        bulk_g2s_hint(smem + OFF_RAW + (slot * PAGES + lane) * PAGE, tiles + page * stride, PAGE,
                      &bars[B_RAW_FULL + slot], policy);
      }
      done = i + 1;
    }
    // No copy may still be in flight when the CTA ends.
    for (int i = max(0, done - RAW); i < done; ++i)
      mbar_wait(d, &bars[B_RAW_FULL + i % RAW], i / RAW & 1);
  } else if (lane == 0) {
    // ---------------- MMA issuers ----------------
    bool ok = true;
    if (warp == W_S) {
      constexpr uint32_t ID = f16_desc(KEYS, M, false);
      ok = mbar_wait(d, &bars[B_Q], 0);
      for (int i = 0; i < n_st && ok; ++i) {
        const int b = i & 1;
        ok = mbar_wait(d, &bars[B_K_FULL + b], i >> 1 & 1) &&
             (i < 2 || mbar_wait(d, &bars[B_PV + b], (i >> 1) - 1 & 1));
        if (!ok) break;
        tc_fence_after();
        const uint64_t k_desc = smem_desc(sbase + OFF_K + b * TILE, 0, 1024);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          tc_mma_ts(tmem + S_COL + KEYS * b, tmem + Q_COL + 8 * kk,
                    desc_at(k_desc, (kk >> 2) * PANEL + (kk & 3) * 32), ID, kk > 0);
        tc_commit(&bars[B_S_FULL + b]);
        tc_commit(&bars[B_K_EMPTY + b]);
      }
    } else {
      constexpr uint32_t ID = f16_desc(D, M, true);
      for (int i = 0; i < n_st && ok; ++i) {
        const int b = i & 1;
        ok = mbar_wait(d, &bars[B_V_FULL + b], i >> 1 & 1) &&
             mbar_wait(d, &bars[B_P_FULL + b], i >> 1 & 1);
        if (!ok) break;
        tc_fence_after();
        const uint64_t v_desc = smem_desc(sbase + OFF_V + b * TILE, PANEL, 1024);
#pragma unroll
        for (int kk = 0; kk < KEYS / 16; ++kk)
          tc_mma_ts(tmem + O_COL, tmem + S_COL + KEYS * b + (kk >> 2) * (KEYS / 2) + (kk & 3) * 8,
                    desc_at(v_desc, kk * 16 * 128), ID, i > 0 || kk > 0);
        tc_commit(&bars[B_PV + b]);
        tc_commit(&bars[B_V_EMPTY + b]);
      }
    }
    if (!ok) s_abort = 1;
    // No MMA may still be running when the tensor memory is released.
    tc_commit(&bars[B_FINAL + (warp - W_S)]);
    mbar_wait(d, &bars[B_FINAL + (warp - W_S)], 0);
  }
  __syncwarp();
  if (warp >= SM_WARPS) pdl_wait();
  tc_fence_before();
  __syncthreads();  // every product and copy is complete
  tc_fence_after();

  // ---------------- output ----------------
  if (warp < SM_WARPS && 32 * quarter < R) {
    const int r = 32 * quarter + lane;
    const bool live = r < R;
    const uint32_t trow = tmem + ((uint32_t)(32 * quarter) << 16) + O_COL;
    const int last = last0 + r / G;
    l = s_row[M + r] + s_row[2 * M + r];
    const float f = k_slices == 1 ? 16.f / l : 1.f;
    __nv_bfloat16* orow =
        out + ((size_t)(si.q_row0 + r / G) * d.q_heads + sl.head * G + r % G) * D;
    float* prow = reinterpret_cast<float*>(smem + OFF_K + r * ROW_PITCH);
#pragma unroll 1
    for (int x = 2 * half; x < 2 * half + 2; ++x) {  // this thread's half of the row
      float o[32];
      __syncwarp();
      if (n_st > 0) {
        tmem_ld32(trow + GROUP * x, o);
      } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = 0.f;
      }
      if (!live || s_abort) continue;
      const bool is_nan = last >= nan_at[x];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = j < 2 ? j : 5 - j;  // unpack_v's places: words of odd pieces change sides
        float y[8];
        in_order(o + 8 * j, is_nan ? __uint_as_float(0x7FC00000u) : f, y);
        if (k_slices == 1) {
          Eight<__nv_bfloat16>::store(orow + GROUP * x + 8 * at, y);
        } else {
          float* to = prow + GROUP * x + 8 * at;
          *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<float4*>(to + 4) = make_float4(y[4], y[5], y[6], y[7]);
        }
      }
    }
    if (live && k_slices > 1 && half == 0)
      *reinterpret_cast<float4*>(prow + D) = make_float4(dead ? -INFINITY : m, l, c, 0.f);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == W_S) tmem_dealloc(tmem, TMEM_COLS);
  if (k_slices == 1) return;

  // Rows [slice R / k, (slice + 1) R / k) of the pair are this CTA's to merge and write.
  __syncwarp();
  cluster_arrive();
  cluster_wait();  // every part is in its CTA's shared memory
  const int k = k_slices, r0 = slice * R / k, n_rows = (slice + 1) * R / k - r0;
  for (int i = tid; i < n_rows * (D / 4); i += THREADS) {
    const int r = r0 + i / (D / 4), x = i % (D / 4);
    const uint32_t at = sbase + OFF_K + r * ROW_PITCH;
    float4 ml[PF_MAX_SLICES], o[PF_MAX_SLICES];
#pragma unroll
    for (int p = 0; p < PF_MAX_SLICES; ++p) {
      if (p >= k) break;
      const uint32_t there = cluster_map(at, p);
      ml[p] = ld_cluster(there + D * 4);
      o[p] = ld_cluster(there + x * 16);
    }
    float mx = -INFINITY, L = 0.f;
#pragma unroll
    for (int p = 0; p < PF_MAX_SLICES; ++p)
      if (p < k) mx = fmaxf(mx, ml[p].x);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int p = 0; p < PF_MAX_SLICES; ++p) {
      if (p >= k) break;
      const float w = weight2(ml[p].x, mx, ml[p].z);
      L += ml[p].y * w;
      a.x = fmaf(o[p].x, w, a.x);
      a.y = fmaf(o[p].y, w, a.y);
      a.z = fmaf(o[p].z, w, a.z);
      a.w = fmaf(o[p].w, w, a.w);
    }
    const float f = 16.f / L;
    __nv_bfloat16* to = out + ((size_t)(si.q_row0 + r / G) * d.q_heads + sl.head * G + r % G) * D + 4 * x;
    *reinterpret_cast<uint2*>(to) =
        make_uint2(pack_bf16(a.x * f, a.y * f), pack_bf16(a.z * f, a.w * f));
  }
  __syncwarp();
  cluster_arrive();
  cluster_wait();  // no CTA still reads this one's rows
}

}  // namespace

cudaError_t kv4_prefill_tc_limits(Limits* lim) {
  cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(&prefill_kv4_kernel),
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
  if (e != cudaSuccess) return e;
  for (int k = 1; k <= PF_MAX_SLICES; ++k) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(k);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = k;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, &prefill_kv4_kernel, &cfg);
    lim->kv4_clusters[k] = e == cudaSuccess ? n : 0;
    if (e != cudaSuccess) cudaGetLastError();  // (a size that the device does not take: no error)
  }
  return cudaSuccess;
}

cudaError_t launch_prefill_kv4_tc(const Dev& d, const Limits& lim, int layer, const void* q,
                                  void* out, int n_pairs, int64_t units, Early early,
                                  cudaStream_t s, int64_t* launches) {
  // How the pairs are cut, by what was measured: a CTA takes 9 us beside its stages of 1.15 us, a merge
  // 1 us.  (31 stages: one session 45 us in one slice, 28 in 2, 19 in 4, 15.7 in 8; 9 sessions 46, 30, 42
  // and 81 us; 64 sessions 183 in one, 207 in 2.)  Whole waves of uncut pairs may go first, the rest
  // in slices of its own behind them, where one more wave would find most SMs without a pair.
  const int pages = (int)std::max<int64_t>(1, (units + n_pairs - 1) / n_pairs);
  const int stages = (pages + PAGES - 1) / PAGES, per_wave = lim.kv4_clusters[1];
  auto cut = [&](int n, float* least) {
    int k = 1;
    *least = n > 0 ? 1e30f : 0.f;
    for (int x = 1; n > 0 && x <= std::min(PF_MAX_SLICES, stages); ++x) {
      if (lim.kv4_clusters[x] < 1) continue;
      const int waves = (n + lim.kv4_clusters[x] - 1) / lim.kv4_clusters[x];
      const float t = waves * (9.f + 1.15f * ((stages + x - 1) / x)) + (x > 1 ? 1.f : 0.f);
      if (t < *least) {
        *least = t;
        k = x;
      }
    }
    return k;
  };
  float t_all, t_rest;
  int first = 0, k = cut(n_pairs, &t_all);
  if (per_wave > 0 && n_pairs > per_wave) {
    const int waves = n_pairs / per_wave, k_rest = cut(n_pairs - waves * per_wave, &t_rest);
    if (k_rest > 1 && waves * (9.f + 1.15f * stages) + t_rest < t_all) {
      first = waves * per_wave;
      k = k_rest;
    }
  }
  for (int part = first > 0 ? 0 : 1; part < 2; ++part) {
    const int kp = part == 0 ? 1 : k, n = part == 0 ? first : n_pairs - first;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n * kp);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int a = 0;
    if (kp > 1) {
      attr[a].id = cudaLaunchAttributeClusterDimension;
      attr[a].val.clusterDim.x = kp;
      attr[a].val.clusterDim.y = 1;
      attr[a].val.clusterDim.z = 1;
      ++a;
    }
    attr[a].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[a].val.programmaticStreamSerializationAllowed = 1;
    ++a;
    cfg.attrs = attr;
    cfg.numAttrs = a;
    // (The second launch starts when the first has waited for the append, if it had to.)
    const cudaError_t e = cudaLaunchKernelEx(&cfg, &prefill_kv4_kernel, d, layer,
                                             static_cast<const __nv_bfloat16*>(q),
                                             static_cast<__nv_bfloat16*>(out), part == 0 ? 0 : first, kp,
                                             part == 1 && first > 0 && early == EARLY_NONE ? EARLY_ALL : early);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

}  // namespace kvc
