// Chunked-prefill attention over a cache held in 4 bits (KVC_KV4), bfloat16 calls, on the
// 5th-generation tensor cores (tcgen05 + TMEM).
//
// The T * G query rows of a (session, KV head) pair (T <= 32 tokens, G = 4 heads) are the M = 128
// rows of the products S = Q K^T and O += P V, 96 keys (6 pages) a stage.  Operands are binary16:
// K and V exactly the numbers that the codes stand for (over 16, kvc_kv4.h), q and P rounded to 11
// bits; accumulation and softmax in binary32.  Rounding and masks are those of kvc_kv4_decode.cu:
// q rows over a power of two, P = exp2(s - m + 8) with a lagging reference m, masked keys of weight
// 0, invalid slots of value 0.  A V group that stands for NaN and that not every row sees is held as
// 0 and its first place noted; the rows that see it get NaN when they are written.
//
// Two ways to spread the pages.  Cluster: each pair's pages are cut into k slices of whole stages, one
// CTA each; the k CTAs of a pair are a thread-block cluster and merge their partial rows through
// distributed shared memory.  Stream-K: the call's (session, KV head, page) units are cut evenly over
// a grid of one CTA per SM; a CTA's range covers segments, the parts of pairs inside it, and the last
// CTA of a pair to finish merges the parts from global memory.  Every role walks the segments by
// itself, so that pages are copied and unpacked for the next one while this one's rows are written.
//
// Warps of a CTA (512 threads, one CTA per SM):
//   0-3, 4-7  softmax, two groups that take the stages in turn: a thread owns a TMEM lane, that is a
//          query row; turns its row of S into one of P (written over it).  Both groups weigh against
//          one reference per row, so that their products share O: a stage's weights are formed with
//          the reference at hand, and published when the stage before has been, formed again if that
//          one moved it.  The groups also rotate the queries into TMEM and write the output;
//   8-13   operands: unpack the pages of a stage, K and V, into 128-byte-swizzled tiles, a page each.
//          Dims and nibbles keep their stored order (the query's dims take K's, the output's are put
//          back in order), so that a word of eight codes becomes one 16-byte store; the order of the
//          stores of a warp is chosen so that eight lanes in a row hit all banks;
//   14     copies the raw pages (18 D bytes each, K and V) into a ring of 3 stages;
//   15     issues S = Q K^T (Q from TMEM) two stages ahead of O += P V (P from TMEM, V read along its
//          keys); three S tiles, so that neither waits for the other.
// Every wait is bounded; a timeout records KVC_DERR_WAIT and the CTA stops.
#include <cuda.h>

#include <algorithm>

#include "kvc_kv4.cuh"
#include "kvc_prefill_tc.cuh"

namespace kvc {

namespace {

using namespace kv4;

constexpr int PAGES = 6, KEYS = PAGES * PS;     // of a stage
constexpr int PAGE = 18 * D;                    // raw bytes of a page of one head, K and V
constexpr int PANEL = KEYS * 128;               // rows of 64 binary16 numbers
constexpr int TILE = 2 * PANEL;                 // K or V of a stage
constexpr int BUF = 3;                          // stages of raw pages, K, V and S
constexpr int SM_WARPS = 8, OP_WARPS = PAGES, SM_THREADS = 32 * SM_WARPS;
constexpr int W_OP = SM_WARPS, W_LOAD = W_OP + OP_WARPS, W_MMA = W_LOAD + 1;
constexpr int THREADS = (W_MMA + 1) * 32;
constexpr float P_SHIFT = 8.f, P_LAG = 6.f;     // as in the decode kernel

// Tensor memory: three S tiles (96 fp32 columns; P, 48 columns of pairs, over the first half), Q
// (64), O (128).
constexpr int TMEM_COLS = 512, S_COL = 0, Q_COL = BUF * KEYS, O_COL = 384;
static_assert(Q_COL + D / 2 <= O_COL && O_COL + D <= TMEM_COLS, "tensor memory");

enum {
  B_RAW_FULL = 0,                  // [BUF] raw pages of a stage copied
  B_RAW_EMPTY = B_RAW_FULL + BUF,  // [BUF] ... and unpacked
  B_K_FULL = B_RAW_EMPTY + BUF,    // [BUF] K tile of a stage written
  B_K_EMPTY = B_K_FULL + BUF,      // [BUF] ... and read by S = Q K^T
  B_V_FULL = B_K_EMPTY + BUF,
  B_V_EMPTY = B_V_FULL + BUF,
  B_S_FULL = B_V_EMPTY + BUF,      // [BUF] scores complete
  B_P_FULL = B_S_FULL + BUF,       // [BUF] weights written
  B_PV = B_P_FULL + BUF,           // [BUF] O += P V complete (and S, P of the stage free)
  B_TURN = B_PV + BUF,             // [4 quarters][2 groups] a stage's weights published
  B_Q = B_TURN + 8,                // query rows in TMEM
  B_FINAL = B_Q + 1,               // every product complete
  N_BARS = B_FINAL + 1
};
// Shared memory from a 1024-aligned base: K tiles, V tiles, raw ring, query rows on their way to TMEM
// (padded: 8 lanes read 8 rows without a conflict), row values, barriers.  The partial rows of a slice
// take the place of the tiles when its products are complete.
constexpr int OFF_K = 0, OFF_V = OFF_K + BUF * TILE, OFF_RAW = OFF_V + BUF * TILE;
constexpr int Q_PITCH = 2 * D + 16;
constexpr int OFF_Q = OFF_RAW + BUF * PAGES * PAGE;
constexpr int OFF_ROW = OFF_Q + M * Q_PITCH;    // [M] softmax scale, [M] reference, [2][M] sums
constexpr int OFF_BAR = OFF_ROW + 4 * M * 4;
constexpr int OFF_TMEM = OFF_BAR + N_BARS * 8;
// First retained index of a NaN in each group: of 8 segments, since pages of up to three segments ahead
// are unpacked while a segment's rows are written.
constexpr int OFF_NAN = OFF_TMEM + 8, NAN_SEGS = 8, NG = D / GROUP, NO_NAN = 1 << 30;
constexpr int SMEM = 1024 + OFF_NAN + NAN_SEGS * NG * 4;
constexpr int ROW_PITCH = (D + 4) * 4;          // a partial row: D values, then (m, l, c)
static_assert(OFF_BAR % 8 == 0 && PAGE % 16 == 0 && M * ROW_PITCH <= OFF_RAW, "layout");
static_assert(PANEL % 1024 == 0 && SMEM <= 227 * 1024 - 256, "fits");

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

// K tile rows of page i of a stage from its raw tile (shared addresses): lane (x, t) takes words
// [4 t, 4 t + 4) of rows r and r + 8.
__device__ inline void unpack_k(uint32_t raw, uint32_t tile, int i, bool open, const BlockRange& br,
                                int lane) {
  const int x = lane >> 2, t = lane & 3;
  const int r0 = (x & 4) | (x & 1) << 1 | (x >> 1 & 1);  // rows two apart side by side
  const int turn = t >> 1;                               // this lane's words in the order w ^ turn
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
      // (w ^ turn of a register array would go through memory: both are picked.)
      const uint32_t word = turn ? w[s ^ 1] : w[s];
      const uint32_t mm = __byte_perm(m[s / 2], 0, (s & 1) != turn ? 0x3232u : 0x1010u);
      uint32_t v[4];
      pairs_of(word, bits_h2(mm), __hmul2(bits_h2(mm), m72), v);
      sts128(to + (((4 * (t & 1) + (s ^ turn)) ^ (row & 7)) << 4), v);
    }
  }
}

// V tile rows of page i of a stage: lane (g, t) takes piece g of rows 2t, 2t + 1 (+ 8).
__device__ inline void unpack_v(uint32_t raw, uint32_t tile, int i, bool open, const BlockRange& br,
                                int last0, int* nan_at, int lane) {
  const int g = lane >> 2, t = lane & 3, turn = g & 1;   // this lane's rows in the order k ^ turn
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
      const int row = row0 + (k ^ turn);
      const uint32_t mm = __byte_perm(m, 0, k != turn ? 0x3232u : 0x1010u);
      const uint32_t to = tile + (g >> 2) * PANEL + (PS * i + row) * 128;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint32_t v[4];
        pairs_of(turn ? w[2 * (k ^ 1) + s] : w[2 * k + s], bits_h2(mm), __hmul2(bits_h2(mm), m72), v);
        sts128(to + (((2 * (g & 3) + s) ^ (row & 7)) << 4), v);
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
      uint8_t* to = rows + r * Q_PITCH + (4 * (c % 4) + c / 4) * 16;
      *reinterpret_cast<uint4*>(to) = make_uint4(u1[0], u1[1], u1[2], u1[3]);
      *reinterpret_cast<uint4*>(to + 32) = make_uint4(u2[0], u2[1], u2[2], u2[3]);
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

// The session of the call that holds unit u (one warp; one round trip for 32 sessions each).
__device__ inline int session_of_unit(const Dev& d, int u, int lane) {
  const int n_seq = d.g->n_seq;
  int n = 0;
  for (int i = lane; i < n_seq + lane; i += 32)
    n += __popc(__ballot_sync(FULL, i < n_seq && d.seq[i].unit_base <= u));
  return n - 1;
}

// A segment: units [u, end) of a pair.
struct Seg {
  SeqInfo si;
  int seq, head, pair_start, pair_end, u, end;
  __device__ int blk0() const { return u - pair_start; }
  __device__ int nblk() const { return end - u; }
  __device__ int stages() const { return (end - u + PAGES - 1) / PAGES; }
  __device__ int last0() const { return si.n_hist + si.n_live - si.t; }  // of the first token
  __device__ bool whole() const { return u == pair_start && end == pair_end; }
  __device__ void set(int s, int h, int u0, int u_end) {
    seq = s;
    head = h;
    pair_start = si.unit_base + h * si.n_blocks;
    pair_end = pair_start + si.n_blocks;
    u = u0;
    end = min(u_end, pair_end);
  }
  // The segment behind this one (which ends at its pair's end): the session's next head or the next
  // session's first.
  __device__ void step(const Dev& d, int u_end) {
    const int at = end;
    int h = head + 1, s = seq;
    if (h == d.kv_heads) {
      h = 0;
      si = d.seq[++s];
    }
    set(s, h, at, u_end);
  }
};

// Dims [8 c, 8 c + 8) of an output row from its columns in the tiles' order.
__device__ inline void in_order(const float* o, float f, float (&y)[8]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    y[p] = o[2 * p] * f;
    y[p + 4] = o[2 * p + 1] * f;
  }
}

template <bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 1) prefill_kv4_kernel(
    Dev d, int layer, const __nv_bfloat16* __restrict__ q, __nv_bfloat16* __restrict__ out,
    int k_slices, int early) {
  extern __shared__ uint8_t smem_raw[];
  // (The same offset in every CTA, so that cluster_map() of an address finds the peer's.)
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_TMEM);
  int* nan_at = reinterpret_cast<int*>(smem + OFF_NAN);
  __shared__ int s_abort_flag, s_last, s_stop;
  volatile int& s_abort = s_abort_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = d.kv_heads;
  // The first call after an append waits for it (and lets nothing else start before that).
  if (!early) pdl_wait();
  if (CLUSTER && d.g->n_units == 0) {  // the append failed: nothing to do for any CTA
    pdl_wait();
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < BUF; ++i) {
      mbar_init(&bars[B_RAW_FULL + i], 1);
      mbar_init(&bars[B_RAW_EMPTY + i], PAGES);
      mbar_init(&bars[B_K_FULL + i], PAGES);
      mbar_init(&bars[B_K_EMPTY + i], 1);
      mbar_init(&bars[B_V_FULL + i], PAGES);
      mbar_init(&bars[B_V_EMPTY + i], 1);
      mbar_init(&bars[B_S_FULL + i], 1);
      mbar_init(&bars[B_P_FULL + i], SM_WARPS / 2);
      mbar_init(&bars[B_PV + i], 1);
    }
    for (int i = 0; i < 8; ++i) mbar_init(&bars[B_TURN + i], 1);
    mbar_init(&bars[B_Q], SM_WARPS);
    mbar_init(&bars[B_FINAL], 1);
    fence_mbar_init();
    s_abort = 0;
    s_stop = 0;
  }
  if (tid < NAN_SEGS * NG) nan_at[tid] = NO_NAN;
  // This CTA's units, and its first segment.
  UnitSplit us = {};
  Seg seg;
  int u_begin = 0, u_end = 0;
  const int cta = blockIdx.x;
  if constexpr (CLUSTER) {
    const int pair = cta / k_slices, slice = cta % k_slices, s = pair / H;
    seg.si = d.seq[s];
    const int nb = seg.si.n_blocks, all = (nb + PAGES - 1) / PAGES;
    const int from = min(nb, PAGES * (int)((int64_t)slice * all / k_slices));
    const int to = min(nb, PAGES * (int)((int64_t)(slice + 1) * all / k_slices));
    const int base = seg.si.unit_base + pair % H * nb;
    seg.set(s, pair % H, base + from, base + to);
    u_begin = seg.u;
    u_end = seg.end;
  } else {
    us = unit_split(d, gridDim.x, PAGES, 1 << 16);
    if (cta < us.n_cta) {
      u_begin = us.start_of(cta);
      u_end = us.start_of(cta + 1);
    }
    if (u_begin < u_end) {
      const int s = session_of_unit(d, u_begin, lane);
      seg.si = d.seq[s];
      seg.set(s, (u_begin - seg.si.unit_base) / seg.si.n_blocks, u_begin, u_end);
    }
  }
  __syncwarp();
  if (warp == W_MMA) tmem_alloc(tmem_slot, TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();
  const uint32_t sbase = smem_u32(smem);

  // A wait that gives up stops its warp; the others follow when their own waits do.
  auto wait = [&](int bar, uint32_t parity) {
    const bool ok = __all_sync(FULL, mbar_wait(d, &bars[bar], parity & 1));
    if (!ok && lane == 0) s_abort = 1;
    return ok;
  };
  // Phases: a stage's number n over all segments (it has the (n % BUF)-th tiles, the (n / BUF)-th time),
  // a segment's number g.
  if (warp < SM_WARPS) {
    // ---------------- softmax ----------------
    const int quarter = warp & 3, grp = warp >> 2;
    const int r = 32 * quarter + lane;
    const uint32_t trow = tmem + ((uint32_t)(32 * quarter) << 16);
    float* s_row = reinterpret_cast<float*>(smem + OFF_ROW);
    volatile float* s_m = s_row + M;
    auto sync_all = [] {
      __syncwarp();
      asm volatile("bar.sync 5, %0;" ::"n"(SM_THREADS) : "memory");
    };
    pdl_wait();
    int n = 0;
    for (int u = u_begin, g = 0; u < u_end; ++g) {
      if (g > 0) seg.step(d, u_end);
      u = seg.end;
      const SeqInfo& si = seg.si;
      const int n_st = seg.stages(), last0 = seg.last0(), R = si.t * G, nblk = seg.nblk();
      const bool live = r < R, idle = 32 * quarter >= R;
      stage_queries(d, si, seg.head, q, smem + OFF_Q, s_row, tid);
      if (grp == 0) s_m[r] = -INFINITY;
      sync_all();
      {
        // This thread's half of its row's 64 columns of pairs; padding rows are zeros.
        uint32_t w[32];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const uint4 v = live ? *reinterpret_cast<const uint4*>(smem + OFF_Q + r * Q_PITCH + 128 * grp + 16 * x)
                               : make_uint4(0, 0, 0, 0);
          w[4 * x] = v.x;
          w[4 * x + 1] = v.y;
          w[4 * x + 2] = v.z;
          w[4 * x + 3] = v.w;
        }
        __syncwarp();
        tmem_st32(trow + Q_COL + 32 * grp, w);
      }
      const float c = live ? s_row[r] : 0.f;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_Q]);
      // The sum of the weights of this thread's keys, and the reference that they were formed with.
      float m = -INFINITY, l = 0.f;
      bool dead = false;
      const int last = last0 + r / G;  // retained index of the last key that the row sees
      for (int i = 0; i < n_st && !dead; ++i, ++n) {
        if ((n & 1) != grp) continue;
        const int b = n % BUF;
        dead = !wait(B_S_FULL + b, n / BUF);
        if (dead) break;
        tc_fence_after();
        if (idle) {  // padding rows: whatever their P is, it stays in their rows of O
          if (lane == 0) {
            mbar_arrive(&bars[B_P_FULL + b]);
            mbar_arrive(&bars[B_TURN + 2 * quarter + grp]);
          }
          continue;
        }
        const uint32_t ts = trow + S_COL + KEYS * b;
        const int b0 = seg.blk0() + PAGES * i, npg = nblk - PAGES * i;
        // Pages of the stage with a key that some row must not see.
        unsigned edge = 0;
#pragma unroll
        for (int pg = 0; pg < PAGES; ++pg) {
          const BlockRange br = block_range(si, b0 + min(pg, npg - 1));
          if (pg >= npg || br.lo > 0 || br.hi < PS || br.base + PS - 1 > last0) edge |= 1u << pg;
        }
        // Slots of page pg that the row sees.
        auto seen = [&](int pg, int& lo, int& hi) {
          const BlockRange br = block_range(si, b0 + pg);
          lo = br.lo;
          hi = pg < npg ? min(br.hi, last - br.base + 1) : 0;
        };
        uint32_t pw[KEYS / 2];
        float sum = 0.f, most = -INFINITY;
        auto weigh = [&](float ref) {
          most = -INFINITY;
          float2 rs[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float2 c2 = make_float2(c, c), sh = make_float2(P_SHIFT, P_SHIFT);
          const float2 nm = make_float2(-ref, -ref);
#pragma unroll
          for (int part = 0; part < PAGES / 2; ++part) {
            float s[32];
            tmem_ld32(ts + 32 * part, s);
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float2 a = __ffma2_rn(__fadd2_rn(make_float2(s[k], s[k + 1]), nm), c2, sh);
              s[k] = a.x;
              s[k + 1] = a.y;
            }
            if (edge >> (2 * part) & 3u) {
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
              most = fmaxf(most, fmaxf(s[k], s[k + 1]));
              const float2 p = make_float2(ex2(s[k]), ex2(s[k + 1]));
              rs[(k / 2) & 1] = __fadd2_rn(rs[(k / 2) & 1], p);
              pw[16 * part + k / 2] = h2_bits(__floats2half2_rn(p.x, p.y));
            }
          }
          sum = (rs[0].x + rs[1].x) + (rs[0].y + rs[1].y);
        };
        // The stage before has published its weights, and with them the reference.
        auto turn = [&] {
          return wait(B_TURN + 2 * quarter + (grp ^ 1), (n - 1) >> 1);
        };
        float ref = -INFINITY;
        if (i > 1) {
          ref = s_m[r];  // (perhaps not the last one yet)
          weigh(ref);
        }
        if (i > 0) {
          dead = !turn();
          if (dead) break;
        }
        const float now = i > 0 ? s_m[r] : -INFINITY;
        // Formed again where the reference moved or a weight passes 2^(P_SHIFT + P_LAG), and at a
        // segment's first two stages.
        if (i < 2 || __any_sync(FULL, live && (now != ref || most > P_SHIFT + P_LAG))) {
          float mx = -INFINITY;
#pragma unroll
          for (int part = 0; part < PAGES / 2; ++part) {
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
          ref = now;
          if (mx > now && !((mx - now) * c <= P_LAG)) ref = mx;
          if (i > 0 && __any_sync(FULL, live && ref != now)) {
            // The products so far are complete: the row of O is scaled.
            dead = !wait(B_PV + (n - 1) % BUF, (n - 1) / BUF);
            if (dead) break;
            tc_fence_after();
            const float f = ref == now ? 1.f : weight2(now, ref, c);
#pragma unroll 1
            for (int x = 0; x < D / 16; ++x) {
              float o[16];
              tmem_ld16(trow + O_COL + 16 * x, o);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] *= f;
              tmem_st16(trow + O_COL + 16 * x, o);
            }
          }
          weigh(ref);
        }
        if (m != ref) l *= weight2(m, ref, c);
        m = ref;
        l += sum;
        s_m[r] = ref;
        __syncwarp();
        tmem_st16(ts, pw);
        tmem_st16(ts + 16, pw + 16);
        tmem_st16(ts + 32, pw + 32);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars[B_P_FULL + b]);
          mbar_arrive(&bars[B_TURN + 2 * quarter + grp]);
        }
      }
      // Every product of the segment complete; the sums of a row's two threads.
      if (!dead) dead = !wait(B_PV + (n - 1) % BUF, (n - 1) / BUF);
      tc_fence_after();
      // (All softmax warps stop together: only they set this, before the barrier.)
      if (dead && lane == 0) s_stop = 1;
      sync_all();
      const bool stop = *static_cast<volatile int*>(&s_stop) != 0;
      const float m_end = s_m[r];
      s_row[M * (2 + grp) + r] = m == m_end ? l : l * weight2(m, m_end, c);
      m = m_end;
      sync_all();
      l = s_row[2 * M + r] + s_row[3 * M + r];
      const bool whole = CLUSTER ? k_slices == 1 : seg.whole();
      const float f = whole ? 16.f / l : 1.f;
      __nv_bfloat16* orow =
          out + ((size_t)(si.q_row0 + r / G) * d.q_heads + seg.head * G + r % G) * D;
      const int slot = 2 * cta + (seg.u == u_begin ? 0 : 1);
      // Rows of a partial slot: [D / 4 chunks][M rows] of 16 bytes, so that the threads of a warp, a
      // row each, access them side by side.
      auto part_row = [&](int sl) { return reinterpret_cast<float4*>(d.pf_part_o + (size_t)sl * (M * D)) + r; };
      if (!idle) {
#pragma unroll 1
        for (int x = 2 * grp; x < 2 * grp + 2; ++x) {  // this thread's half of the row
          float o[32];
          __syncwarp();
          tmem_ld32(trow + O_COL + GROUP * x, o);
          if (!live || stop) continue;
          const bool is_nan = last >= nan_at[(g % NAN_SEGS) * NG + x];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float y[8];
            in_order(o + 8 * j, is_nan ? __uint_as_float(0x7FC00000u) : f, y);
            const float4 lo = make_float4(y[0], y[1], y[2], y[3]), hi = make_float4(y[4], y[5], y[6], y[7]);
            if (whole) {
              Eight<__nv_bfloat16>::store(orow + GROUP * x + 8 * j, y);
            } else if constexpr (CLUSTER) {
              float* to = reinterpret_cast<float*>(smem + OFF_K + r * ROW_PITCH) + GROUP * x + 8 * j;
              *reinterpret_cast<float4*>(to) = lo;
              *reinterpret_cast<float4*>(to + 4) = hi;
            } else {
              part_row(slot)[(8 * x + 2 * j) * M] = lo;
              part_row(slot)[(8 * x + 2 * j + 1) * M] = hi;
            }
          }
        }
        if (live && !whole && grp == 0) {
          if constexpr (CLUSTER)
            *reinterpret_cast<float4*>(smem + OFF_K + r * ROW_PITCH + D * 4) =
                make_float4(stop ? -INFINITY : m, l, c, 0.f);
          else
            d.pf_part_ml[(size_t)slot * M + r] = make_float2(m, l);
        }
      }
      tc_fence_before();
      sync_all();
      if (stop) break;
      if (tid < NG) nan_at[(g % NAN_SEGS) * NG + tid] = NO_NAN;
      if (!CLUSTER && !whole) {
        // The last CTA of the pair to arrive merges.
        const int cf = us.owner(seg.pair_start), parts = us.owner(seg.pair_end - 1) - cf + 1;
        int* counter = &d.pf_count[seg.seq * H + seg.head];
        if (tid == 0) s_last = arrive_acq_rel(counter, parts);
        sync_all();
        if (s_last) {
          const int first_slot = us.slot_of(cf, cf, seg.pair_start);
          auto slot_of = [&](int p) { return p ? 2 * (cf + p) : first_slot; };
          if (live) {
            float mx = -INFINITY, L = 0.f;
            for (int p = 0; p < parts; ++p)
              mx = fmaxf(mx, __ldcg(&d.pf_part_ml[(size_t)slot_of(p) * M + r]).x);
            for (int p = 0; p < parts; ++p) {
              const float2 ml = __ldcg(&d.pf_part_ml[(size_t)slot_of(p) * M + r]);
              L += ml.y * weight2(ml.x, mx, c);
            }
            const float inv = 16.f / L;
#pragma unroll 1
            for (int x = 2 * grp; x < 2 * grp + 2; ++x) {
              float4 a[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) a[j] = make_float4(0.f, 0.f, 0.f, 0.f);
              for (int p = 0; p < parts; ++p) {
                const float w = weight2(__ldcg(&d.pf_part_ml[(size_t)slot_of(p) * M + r]).x, mx, c) * inv;
                float4 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = __ldcg(part_row(slot_of(p)) + (8 * x + j) * M);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  a[j].x = fmaf(v[j].x, w, a[j].x);
                  a[j].y = fmaf(v[j].y, w, a[j].y);
                  a[j].z = fmaf(v[j].z, w, a[j].z);
                  a[j].w = fmaf(v[j].w, w, a[j].w);
                }
              }
#pragma unroll
              for (int j = 0; j < 8; j += 2) {
                const float y[8] = {a[j].x, a[j].y, a[j].z, a[j].w,
                                    a[j + 1].x, a[j + 1].y, a[j + 1].z, a[j + 1].w};
                Eight<__nv_bfloat16>::store(orow + GROUP * x + 4 * j, y);
              }
            }
          }
          if (tid == 0) *counter = 0;
        }
      }
    }
  } else if (warp < W_LOAD) {
    // ---------------- operands ----------------
    const int pg = warp - W_OP;
    bool ok = true;
    int n = 0;
    for (int u = u_begin, g = 0; u < u_end && ok; ++g) {
      if (g > 0) seg.step(d, u_end);
      u = seg.end;
      const SeqInfo& si = seg.si;
      const int n_st = seg.stages(), last0 = seg.last0(), nblk = seg.nblk(), blk0 = seg.blk0();
      int* nans = nan_at + (g % NAN_SEGS) * NG;
      for (int i = 0; i < n_st; ++i, ++n) {
        const int b = n % BUF, time = n / BUF;
        if (!(ok = wait(B_RAW_FULL + b, time))) break;
        const uint32_t raw = sbase + OFF_RAW + (b * PAGES + pg) * PAGE;
        const bool here = PAGES * i + pg < nblk;
        const BlockRange br = block_range(si, blk0 + (here ? PAGES * i + pg : 0));
        const bool open = br.lo == 0 && br.hi == PS && br.base + PS - 1 <= last0;
        if (n >= BUF && !(ok = wait(B_K_EMPTY + b, time - 1))) break;
        // (A page that is not there: its scores are masked whatever K holds.)
        if (here) unpack_k(raw, sbase + OFF_K + b * TILE, pg, open, br, lane);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_K_FULL + b]);
        if (n >= BUF && !(ok = wait(B_V_EMPTY + b, time - 1))) break;
        if (here) {
          unpack_v(raw + 9 * D, sbase + OFF_V + b * TILE, pg, open, br, last0, nans, lane);
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
          mbar_arrive(&bars[B_RAW_EMPTY + b]);
        }
      }
    }
  } else if (warp == W_LOAD) {
    // ---------------- raw pages ----------------
    const size_t stride = page_bytes(D, d.layers, H);
    const uint64_t policy = evict_first_policy();
    bool ok = true;
    int n = 0;
    for (int u = u_begin, g = 0; u < u_end && ok; ++g) {
      if (g > 0) seg.step(d, u_end);
      u = seg.end;
      const SeqInfo& si = seg.si;
      const int n_st = seg.stages(), nblk = seg.nblk(), blk0 = seg.blk0();
      const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
      const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
      const uint8_t* tiles = d.pool + tile_at(D, d.layers, H, 0, layer, seg.head, 0);
      auto page_at = [&](int b) {
        return lane < PAGES && b < nblk ? block_page(si, hrow, lrow, blk0 + b) : 0;
      };
      int page = page_at(lane);
      {
        // The query rows (1 KiB a token) and rotary rows (512 B) into L2 ahead of the softmax warps.
        const char* qb = reinterpret_cast<const char*>(q + ((size_t)si.q_row0 * d.q_heads + seg.head * G) * D);
        const char* rb = reinterpret_cast<const char*>(d.rope + (size_t)si.pos_first * (D / 2));
        for (int x = lane; x < si.t * 12; x += 32) {
          const int t = x / 12, line = x % 12;
          prefetch_l2(line < 8 ? qb + (size_t)t * d.q_heads * D * 2 + line * 128
                               : rb + (size_t)t * 512 + (line - 8) * 128);
        }
      }
      for (int i = 0; i < n_st; ++i, ++n) {
        const int b = n % BUF, npg = min(PAGES, nblk - PAGES * i);
        const int next = page_at(PAGES * (i + 1) + lane);
        if (n >= BUF && !(ok = wait(B_RAW_EMPTY + b, n / BUF - 1))) break;
        if (lane == 0) mbar_arrive_expect_tx(&bars[B_RAW_FULL + b], npg * PAGE);
        __syncwarp();
        if (lane < npg) {
          fence_proxy_async_smem();
          bulk_g2s_hint(smem + OFF_RAW + (b * PAGES + lane) * PAGE, tiles + page * stride, PAGE,
                        &bars[B_RAW_FULL + b], policy);
        }
        page = next;
      }
    }
    // No copy may still be in flight when the CTA ends.
    for (int i = max(0, n - BUF); i < n; ++i)
      mbar_wait(d, &bars[B_RAW_FULL + i % BUF], i / BUF & 1);
  } else if (lane == 0) {
    // ---------------- MMA issuer ----------------
    constexpr uint32_t ID_S = f16_desc(KEYS, M, false), ID_PV = f16_desc(D, M, true);
    constexpr int AHEAD = 2;
    bool ok = true;
    int n = 0;  // first stage of the segment
    for (int u = u_begin, g = 0; u < u_end && ok; ++g) {
      if (g > 0) seg.step(d, u_end);
      u = seg.end;
      const int n_st = seg.stages();
      ok = mbar_wait(d, &bars[B_Q], g & 1);
      for (int i = 0; i < n_st + AHEAD && ok; ++i) {
        if (i < n_st) {
          const int at = n + i, b = at % BUF, time = at / BUF;
          ok = mbar_wait(d, &bars[B_K_FULL + b], time & 1) &&
               (at < BUF || mbar_wait(d, &bars[B_PV + b], (time - 1) & 1));
          if (!ok) break;
          tc_fence_after();
          const uint64_t k_desc = smem_desc(sbase + OFF_K + b * TILE, 0, 1024);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            tc_mma_ts(tmem + S_COL + KEYS * b, tmem + Q_COL + 8 * kk,
                      desc_at(k_desc, (kk >> 2) * PANEL + (kk & 3) * 32), ID_S, kk > 0);
          tc_commit(&bars[B_S_FULL + b]);
          tc_commit(&bars[B_K_EMPTY + b]);
        }
        if (i >= AHEAD) {
          const int at = n + i - AHEAD, b = at % BUF, time = at / BUF;
          ok = mbar_wait(d, &bars[B_V_FULL + b], time & 1) &&
               mbar_wait(d, &bars[B_P_FULL + b], time & 1);
          if (!ok) break;
          tc_fence_after();
          const uint64_t v_desc = smem_desc(sbase + OFF_V + b * TILE, PANEL, 1024);
#pragma unroll
          for (int kk = 0; kk < KEYS / 16; ++kk)
            tc_mma_ts(tmem + O_COL, tmem + S_COL + KEYS * b + 8 * kk, desc_at(v_desc, kk * 16 * 128),
                      ID_PV, i > AHEAD || kk > 0);
          tc_commit(&bars[B_PV + b]);
          tc_commit(&bars[B_V_EMPTY + b]);
        }
      }
      n += n_st;
    }
    if (!ok) s_abort = 1;
    // No MMA may still be running when the tensor memory is released.
    tc_commit(&bars[B_FINAL]);
    mbar_wait(d, &bars[B_FINAL], 0);
  }
  __syncwarp();
  if (warp >= SM_WARPS) pdl_wait();
  tc_fence_before();
  __syncthreads();  // every product and copy is complete
  tc_fence_after();
  if (warp == W_MMA) tmem_dealloc(tmem, TMEM_COLS);
  if constexpr (CLUSTER) {
    if (k_slices == 1) return;
    // Rows [slice R / k, (slice + 1) R / k) of the pair are this CTA's to merge and write.
    const SeqInfo& si = seg.si;
    const int k = k_slices, slice = cta % k, R = si.t * G;
    for (int r = tid; u_begin == u_end && r < R; r += THREADS)  // no page: weighs nothing
      *reinterpret_cast<float4*>(smem + OFF_K + r * ROW_PITCH + D * 4) = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    __syncwarp();
    cluster_arrive();
    cluster_wait();  // every part is in its CTA's shared memory
    const int r0 = slice * R / k, n_rows = (slice + 1) * R / k - r0;
    for (int i = tid; i < n_rows * (D / 4); i += THREADS) {
      const int r = r0 + i / (D / 4), x = i % (D / 4);
      const uint32_t at = sbase + OFF_K + r * ROW_PITCH;
      float4 ml[PF_MAX_SLICES], o[PF_MAX_SLICES];
#pragma unroll
      for (int p = 0; p < PF_MAX_SLICES; ++p) {
        const uint32_t there = cluster_map(at, min(p, k - 1));
        ml[p] = ld_cluster(there + D * 4);
        o[p] = ld_cluster(there + x * 16);
      }
      float mx = -INFINITY, L = 0.f;
#pragma unroll
      for (int p = 0; p < PF_MAX_SLICES; ++p) mx = fmaxf(mx, ml[p].x);
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int p = 0; p < PF_MAX_SLICES; ++p) {
        if (p >= k || ml[p].x == -INFINITY) continue;  // (a part without a key of this row)
        const float w = weight2(ml[p].x, mx, ml[p].z);
        L += ml[p].y * w;
        a.x = fmaf(o[p].x, w, a.x);
        a.y = fmaf(o[p].y, w, a.y);
        a.z = fmaf(o[p].z, w, a.z);
        a.w = fmaf(o[p].w, w, a.w);
      }
      const float f = 16.f / L;
      __nv_bfloat16* to =
          out + ((size_t)(si.q_row0 + r / G) * d.q_heads + seg.head * G + r % G) * D + 4 * x;
      *reinterpret_cast<uint2*>(to) =
          make_uint2(pack_bf16(a.x * f, a.y * f), pack_bf16(a.z * f, a.w * f));
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();  // no CTA still reads this one's rows
  }
}

}  // namespace

cudaError_t kv4_prefill_tc_limits(const Dev& d, Limits* lim) {
  const void* fns[2] = {reinterpret_cast<const void*>(&prefill_kv4_kernel<false>),
                        reinterpret_cast<const void*>(&prefill_kv4_kernel<true>)};
  for (const void* fn : fns) {
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
  }
  // One CTA per SM; each may leave two partial states.
  lim->kv4_prefill_stream_k = std::min(lim->sms, d.pf_slots / 2);
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
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, &prefill_kv4_kernel<true>, &cfg);
    lim->kv4_clusters[k] = e == cudaSuccess ? n : 0;
    if (e != cudaSuccess) cudaGetLastError();  // (a size that the device does not take: no error)
  }
  return cudaSuccess;
}

cudaError_t launch_prefill_kv4_tc(const Dev& d, const Limits& lim, int layer, const void* q,
                                  void* out, int n_pairs, int64_t units, bool early,
                                  cudaStream_t s) {
  const int pages = (int)std::max<int64_t>(1, (units + n_pairs - 1) / n_pairs);
  const int stages = (pages + PAGES - 1) / PAGES;
  int k = 0;
  float least = n_pairs < lim.sms ? 1e30f : 8.f + 0.9f * n_pairs * stages / lim.sms + 3.f * n_pairs / lim.sms;
  for (int x = 1; x <= std::min(PF_MAX_SLICES, stages); ++x) {
    if (lim.kv4_clusters[x] < 1) continue;
    const int waves = (n_pairs + lim.kv4_clusters[x] - 1) / lim.kv4_clusters[x];
    const float t = waves * (5.5f + 0.9f * ((stages + x - 1) / x)) + (x > 1 ? 2.f : 0.f);
    if (t < least) {
      least = t;
      k = x;
    }
  }
  if (getenv("KV4_PK")) k = atoi(getenv("KV4_PK"));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(k > 0 ? n_pairs * k : lim.kv4_prefill_stream_k);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (k > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = k;
    attr[n].val.clusterDim.y = 1;
    attr[n].val.clusterDim.z = 1;
    ++n;
  }
  attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[n].val.programmaticStreamSerializationAllowed = 1;
  ++n;
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, k > 0 ? &prefill_kv4_kernel<true> : &prefill_kv4_kernel<false>, d,
                            layer, static_cast<const __nv_bfloat16*>(q),
                            static_cast<__nv_bfloat16*>(out), k, (int)early);
}

}  // namespace kvc
