// Whole prompts of binary32 sessions: attention (kvc_attn_prompt) and attention weights
// (kvc_attn_weights), on the tensor cores (mma.sync m16n8k8, TF32 operands, binary32 sums).
//
// A TF32 operand has 11 significant bits.  Each operand x is taken as two: x_up = x rounded to TF32 and
// x - x_up, which is exact, cut to TF32 by the product; a b = a_up b_up + (a_up b_low + a_low b_up) leaves
// out less than 2^-21 of |a b|.  The tensor cores round their sums towards zero, so the large products and
// the two small ones have accumulators of their own (the small ones' roundings do not count), and what a
// tile of 64 keys adds to an output comes into its binary32 sum in one rounded addition.
// Three products for one: a third of the TF32 rate of mma.sync (300 TFLOP/s measured), 100 against the
// 76 TFLOP/s of the FMA pipes, which a kernel on them reaches a quarter to a half of.
//
// A tile is rows of 64 floats in shared memory.  A warp has 16 rows as the A operand, whose pieces lie
// in shared memory, and meets a tile of 64 rows as B, which it takes apart itself.  Dims are taken in an
// order that makes every fragment a 16-byte load: dims 16 c + 4 t .. + 3 of a row are lane t's for the
// steps 2c (first two) and 2c + 1 of the products; of P V the keys 8 s + 2 t, + 1 are lane t's for step
// s, as the scores' fragments hold them, and output dims 32 h + 4 g .. + 3 are column g of four products.
//
// Measured: three prompts of up to 1,501 tokens, 4 KV heads, 198 us a layer (531 on the FMA pipes); bound
// by the products and the operands' taking apart (16 rows a warp leave each B row's pieces to be formed by
// eight warps), and by items: 32 tokens of a KV head, last ones first, on 152 SMs.  Weights of three units
// of 17 tokens behind 1,100 positions 30 us a layer (102 on the FMA pipes), which is three launches and
// their chains of latencies; one after the other instead of together, the nine parts of a row's statistics
// were 3 us of it.  Weights of long chunks: the three prompts 234 us a layer, 4,099 tokens 855 (15 and
// 20 TFLOP/s of scores formed once; they are formed twice).
//
// Tiles with a number that is not finite, or whose upper piece is not (in a slot that holds nothing as well), go a
// slow way in plain binary32 arithmetic, where a key that a row does not see takes no part.
#include <algorithm>
#include <cmath>

#include "kvc_prompt.h"
#include "kvc_prompt_merge.cuh"
#include "kvc_rope.cuh"
#include "kvc_weights_plain.cuh"

namespace kvc {

namespace {

constexpr int G = 4, D = 64;
constexpr int WARPS = 8, THREADS = WARPS * 32;
constexpr int CTAS = 1;                          // of an SM
constexpr int ROWS = 16 * WARPS;                 // of an item's A operand
constexpr int TOKENS = ROWS / G;
constexpr int KT = 64, PAGES = KT / PS, NT = KT / 8;  // keys of a tile, eight a product
constexpr int TILE = KT * D;                     // floats
constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr float LOG2E = 1.4426950408889634f;

__device__ inline void cp_async16(float* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ inline void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ inline void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Float offset of 16-byte chunk c of row r: rows that are K or Q (a warp loads eight rows, four chunks at a
// time: odd rows swap the halves of 128 bytes), and of V (four pairs of rows, two chunks).
__device__ inline int at_k(int r, int c) { return r * D + ((c ^ ((r & 1) << 2)) << 2); }
__device__ inline int at_v(int r, int c) { return r * D + ((c ^ ((r >> 1 & 3) << 1)) << 2); }

struct Pieces {
  uint32_t up, low;
};
__device__ inline Pieces pieces(float x) {
  Pieces p;
  // (Half a unit of the last place that stays, then cut: 10 % faster than the conversion instruction.)
  p.up = (__float_as_uint(x) + 0x1000u) & 0xFFFFE000u;
  p.low = __float_as_uint(x - __uint_as_float(p.up));
  return p;
}
__device__ inline void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Products of the 16 rows from `rows` on (both pieces, in shared memory; the lower ones `low` floats behind)
// with the rows 8 n .. 8 n + 7, n < NT, of a tile: s[n][0, 1] of row g and columns 8 n + 2 t, + 1; s[n][2, 3]
// of row g + 8.
__device__ inline void products(const float* rows, int low, int r0, const float* tile, int lane,
                                float (&s)[NT][4]) {
  const int g = lane >> 2, t = lane & 3;
  float small[NT][4] = {};
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[n][i] = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint4 u0 = *reinterpret_cast<const uint4*>(rows + at_k(r0 + g, 4 * c + t));
    const uint4 u1 = *reinterpret_cast<const uint4*>(rows + at_k(r0 + g + 8, 4 * c + t));
    const uint4 l0 = *reinterpret_cast<const uint4*>(rows + low + at_k(r0 + g, 4 * c + t));
    const uint4 l1 = *reinterpret_cast<const uint4*>(rows + low + at_k(r0 + g + 8, 4 * c + t));
    const uint32_t up[2][4] = {{u0.x, u1.x, u0.y, u1.y}, {u0.z, u1.z, u0.w, u1.w}};
    const uint32_t dn[2][4] = {{l0.x, l1.x, l0.y, l1.y}, {l0.z, l1.z, l0.w, l1.w}};
    // (An accumulator's products lie four apart.)
#pragma unroll
    for (int n0 = 0; n0 < NT; n0 += 4) {
      Pieces p[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float4 x = *reinterpret_cast<const float4*>(tile + at_k(8 * (n0 + n) + g, 4 * c + t));
        p[n][0] = pieces(x.x);
        p[n][1] = pieces(x.y);
        p[n][2] = pieces(x.z);
        p[n][3] = pieces(x.w);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int n = 0; n < 4; ++n) mma(s[n0 + n], up[i], p[n][2 * i].up, p[n][2 * i + 1].up);
#pragma unroll
        for (int n = 0; n < 4; ++n) mma(small[n0 + n], up[i], p[n][2 * i].low, p[n][2 * i + 1].low);
#pragma unroll
        for (int n = 0; n < 4; ++n) mma(small[n0 + n], dn[i], p[n][2 * i].up, p[n][2 * i + 1].up);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[n][i] += small[n][i];
}

// A chunk of a row into its pieces' places.
__device__ inline void put_pieces(float4 x, float* to, int low) {
  const Pieces a = pieces(x.x), b = pieces(x.y), c = pieces(x.z), d = pieces(x.w);
  *reinterpret_cast<uint4*>(to) = make_uint4(a.up, b.up, c.up, d.up);
  *reinterpret_cast<uint4*>(to + low) = make_uint4(a.low, b.low, c.low, d.low);
}

// The same in plain arithmetic (slow): a row of `rows` (the sum of its pieces is exact) with one of the tile.
__device__ __noinline__ float plain_product(const float* rows, int low, int r, const float* tile, int k) {
  float s = 0.f;
  for (int c = 0; c < D / 4; ++c) {
    float4 a = *reinterpret_cast<const float4*>(rows + at_k(r, c));
    const float4 l = *reinterpret_cast<const float4*>(rows + low + at_k(r, c));
    a = make_float4(a.x + l.x, a.y + l.y, a.z + l.z, a.w + l.w);
    const float4 b = *reinterpret_cast<const float4*>(tile + at_k(k, c));
    s = fmaf(a.x, b.x, s);
    s = fmaf(a.y, b.y, s);
    s = fmaf(a.z, b.z, s);
    s = fmaf(a.w, b.w, s);
  }
  return s;
}

// Query rows of tokens [t0, t0 + ROWS_ / G) of one KV head, rotated and scaled, into a tile (low: in pieces,
// the lower ones that many floats behind; 0: as they are); rows past the chunk are zero.
template <int ROWS_>
__device__ inline void stage_rows(const Dev& d, const SeqInfo& si, int head, int t0, const float* __restrict__ q,
                                  float scale, float* tile, int low) {
  constexpr int PER = ROWS_ * 8 / THREADS;  // 16-byte chunks c and c + 8 (which rotate together) of a row
  const int c = threadIdx.x & 7;
  float4 a[PER], b[PER], c0[PER], c1[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = (threadIdx.x >> 3) + i * (THREADS / 8), tok = t0 + r / G;
    a[i] = b[i] = c0[i] = c1[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tok < si.t) {
      const float* row = q + ((size_t)(si.q_row0 + tok) * d.q_heads + head * G + r % G) * D + c * 4;
      const float4* cs = reinterpret_cast<const float4*>(d.rope + (size_t)(si.pos_first + tok) * (D / 2) + c * 4);
      a[i] = *reinterpret_cast<const float4*>(row);
      b[i] = *reinterpret_cast<const float4*>(row + D / 2);
      c0[i] = cs[0];
      c1[i] = cs[1];
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = (threadIdx.x >> 3) + i * (THREADS / 8);
    float4 ya, yb;
    rope_pair(a[i].x, b[i].x, make_float2(c0[i].x, c0[i].y), ya.x, yb.x);
    rope_pair(a[i].y, b[i].y, make_float2(c0[i].z, c0[i].w), ya.y, yb.y);
    rope_pair(a[i].z, b[i].z, make_float2(c1[i].x, c1[i].y), ya.z, yb.z);
    rope_pair(a[i].w, b[i].w, make_float2(c1[i].z, c1[i].w), ya.w, yb.w);
    ya = make_float4(ya.x * scale, ya.y * scale, ya.z * scale, ya.w * scale);
    yb = make_float4(yb.x * scale, yb.y * scale, yb.z * scale, yb.w * scale);
    if (low) {
      put_pieces(ya, tile + at_k(r, c), low);
      put_pieces(yb, tile + at_k(r, 8 + c), low);
    } else {
      *reinterpret_cast<float4*>(tile + at_k(r, c)) = ya;
      *reinterpret_cast<float4*>(tile + at_k(r, 8 + c)) = yb;
    }
  }
}

// Pages of blocks b0 .. b0 + N - 1 of a session, -1 from block nb on.
template <int N>
__device__ inline void look_up(const Dev& d, const SeqInfo& si, int b0, int nb, int (&pages)[N]) {
  const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
  const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
#pragma unroll
  for (int p = 0; p < N; ++p) pages[p] = b0 + p < nb ? block_page(si, hrow, lrow, b0 + p) : -1;
}

// Those pages (zeros for -1) into a tile of K and one of V (or none), asynchronously: a thread has chunk
// tid % 16 of some slots of each page.
template <int N>
__device__ inline void load_pages(const Dev& d, int layer, int head, const int (&pages)[N], float* k, float* v) {
  const int c = threadIdx.x & 15;
#pragma unroll
  for (int p = 0; p < N; ++p) {
    const int page = pages[p];
#pragma unroll
    for (int slot = threadIdx.x >> 4; slot < PS; slot += THREADS / 16) {
      const int r = p * PS + slot;
      if (page >= 0) {
        const float* src = reinterpret_cast<const float*>(d.pool) +
                           pool_offset_elems(d, page, layer, 0, head, slot) + c * 4;
        cp_async16(k + at_k(r, c), src);
        if (v) cp_async16(v + at_v(r, c), src + (size_t)d.kv_heads * PS * D);
      } else {
        *reinterpret_cast<float4*>(k + at_k(r, c)) = make_float4(0.f, 0.f, 0.f, 0.f);
        if (v) *reinterpret_cast<float4*>(v + at_v(r, c)) = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
  }
}

// Whether one of the numbers that this thread brought is not finite, or so large that rounded to TF32 it is not
// (its upper piece would be infinite, the product NaN).
__device__ inline bool odd_pages(int n_pg, const float* k, const float* v) {
  const int c = threadIdx.x & 15;
  bool odd = false;
  auto look = [&](const float* x) {
    const uint4 w = *reinterpret_cast<const uint4*>(x);
    const uint32_t e = 0x7FFFFFFFu, most = 0x7F7FEFFFu;
    odd |= (w.x & e) > most || (w.y & e) > most || (w.z & e) > most || (w.w & e) > most;
  };
#pragma unroll 4
  for (int r = threadIdx.x >> 4; r < n_pg * PS; r += THREADS / 16) {
    look(k + at_k(r, c));
    if (v) look(v + at_v(r, c));
  }
  return odd;
}

// An item, as every thread has it: one of `parts` of one of those that count() counts.
struct Item {
  int seq, in;  // session of the call, and which of its items; seq < 0: no more
  int at;       // of all
};
template <typename CountFn>
__device__ inline Item next_item(const Dev& d, int n_seq, int parts, const int* s_group, Item* s_item,
                                 CountFn count) {
  __syncthreads();
  if (threadIdx.x < 32) {
    int at = 0, in = 0;
    if (threadIdx.x == 0) at = take_item(d);
    at = __shfl_sync(FULL, at, 0);
    const int seq =
        at < s_group[GROUPS] * parts ? find_item(n_seq, threadIdx.x, s_group, at / parts, count, &in) : -1;
    if (threadIdx.x == 0) *s_item = {seq, in * parts + at % parts, at};
  }
  __syncthreads();
  return *s_item;
}

// ---------------------------------------------------------------------------
// Attention, and (STATS) the rows' (max, sum) alone.  An item is 32 tokens of one session and KV head,
// the last ones first, against (a part of) the keys that they see; a warp has four tokens' rows.
// ---------------------------------------------------------------------------
constexpr int PROMPT_SMEM = (2 * ROWS * D + 4 * TILE) * 4;
constexpr int STAT_SMEM = (2 * ROWS * D + 2 * TILE) * 4;

template <bool STATS>
__global__ void __launch_bounds__(THREADS, CTAS) prompt_f32_kernel(Dev d, int layer, const float* __restrict__ q,
                                                             float* __restrict__ out, float scale, int most_parts,
                                                             float2* __restrict__ stats) {
  extern __shared__ __align__(16) float sm[];
  __shared__ int s_group[GROUPS + 1];
  __shared__ Item s_item;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, H = d.kv_heads;
  float *s_q = sm, *s_k = sm + 2 * ROWS * D, *s_v = s_k + 2 * TILE;
  pdl_wait();
  pdl_launch_dependents();
  const int n_seq = d.g->total_tokens > 0 ? d.g->n_seq : 0;  // (no tokens: the append failed)
  auto items_of = [&](int i) { return (d.seq[i].t + TOKENS - 1) / TOKENS * H; };
  if (warp == 0) list_items(n_seq, lane, s_group, items_of);
  __syncthreads();
  const int parts =
      STATS ? stat_parts(d, most_parts, d.g->total_tokens) : parts_now(d, most_parts, s_group[GROUPS]);
  for (;;) {
    const Item it = next_item(d, n_seq, parts, s_group, &s_item, items_of);
    if (it.seq < 0) break;
    const SeqInfo si = d.seq[it.seq];
    const int part = it.in % parts, head = it.in / parts % H;
    const int t0 = ((si.t + TOKENS - 1) / TOKENS - 1 - it.in / parts / H) * TOKENS;
    const int nb = blocks_seen(si, min(t0 + TOKENS, si.t) - 1), all = (nb + PAGES - 1) / PAGES;
    const int j0 = (int)((int64_t)all * part / parts), j1 = (int)((int64_t)all * (part + 1) / parts);
    int pages[PAGES];  // of the next tile to load
    look_up(d, si, PAGES * j0, nb, pages);
    auto load = [&](int j) {
      load_pages(d, layer, head, pages, s_k + (j & 1) * TILE, STATS ? nullptr : s_v + (j & 1) * TILE);
      cp_async_commit();
      look_up(d, si, PAGES * (j + 1), nb, pages);
    };
    if (j0 < j1) load(j0);
    stage_rows<ROWS>(d, si, head, t0, q, scale, s_q, ROWS * D);
    // This lane's rows: 16 warp + g and + 8, of tokens two apart.
    const int tok0 = t0 + 4 * warp + g / G, q_log0 = si.n_hist + si.n_live - si.t;
    const int q_log[2] = {q_log0 + tok0, q_log0 + tok0 + 2};
    const int q_first = q_log0 + t0 + 4 * warp;            // the warp's first token
    const int nb_warp = blocks_seen(si, min(t0 + 4 * warp + 3, si.t - 1));
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float o[8][4] = {};                                     // [4 h + j]: see above
    for (int j = j0; j < j1; ++j) {
      const float *kt = s_k + (j & 1) * TILE, *vt = s_v + (j & 1) * TILE;
      cp_async_wait_all();
      const bool odd = __syncthreads_or(odd_pages(PAGES, kt, STATS ? nullptr : vt));
      if (j + 1 < j1) load(j + 1);
      if (PAGES * j >= nb_warp) continue;                   // behind all tokens of the warp
      float s[NT][4];
      if (!odd) {
        products(s_q, ROWS * D, 16 * warp, kt, lane, s);
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s[n][i] = plain_product(s_q, ROWS * D, 16 * warp + g + (i >> 1) * 8, kt, 8 * n + 2 * t + (i & 1));
      }
      uint32_t seen[2][PAGES];                              // slots of the pages that the rows see
      bool whole = true;
#pragma unroll
      for (int p = 0; p < PAGES; ++p) {
        whole = whole && slots_seen(si, PAGES * j + p, nb, q_first) == 0xFFFFu;
        seen[0][p] = seen[1][p] = 0xFFFFu;
      }
      if (!whole) {
#pragma unroll
        for (int p = 0; p < PAGES; ++p)
#pragma unroll
          for (int h = 0; h < 2; ++h) seen[h][p] = slots_seen(si, PAGES * j + p, nb, q_log[h]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(seen[i >> 1][n >> 1] >> (8 * (n & 1) + 2 * t + (i & 1)) & 1)) s[n][i] = -INFINITY;
      }
      float al[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < NT; ++n) mx = fmaxf(mx, fmaxf(s[n][2 * h], s[n][2 * h + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 2));
        const float mn = fmaxf(m[h], mx), ref = mn == -INFINITY ? 0.f : mn;
        al[h] = exp2_safe(m[h], ref);
        m[h] = mn;
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            s[n][2 * h + e] = ex2(s[n][2 * h + e] - ref);
            sum += s[n][2 * h + e];
          }
        l[h] = l[h] * al[h] + sum;  // (this lane's keys; the others' are added at the end)
      }
      if constexpr (!STATS) {
        if (!odd) {
          Pieces p[NT][4];  // A: rows g, g + 8 of key 2 t, then of key 2 t + 1
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) p[n][i] = pieces(s[n][(i & 1) * 2 + (i >> 1)]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 32 dims
            float big[4][4] = {}, small[4][4] = {};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const float4 a = *reinterpret_cast<const float4*>(vt + at_v(8 * n + 2 * t, 8 * h + g));
              const float4 b = *reinterpret_cast<const float4*>(vt + at_v(8 * n + 2 * t + 1, 8 * h + g));
              const Pieces p0[4] = {pieces(a.x), pieces(a.y), pieces(a.z), pieces(a.w)};
              const Pieces p1[4] = {pieces(b.x), pieces(b.y), pieces(b.z), pieces(b.w)};
              const uint32_t up[4] = {p[n][0].up, p[n][1].up, p[n][2].up, p[n][3].up};
              const uint32_t dn[4] = {p[n][0].low, p[n][1].low, p[n][2].low, p[n][3].low};
#pragma unroll
              for (int i = 0; i < 4; ++i) mma(big[i], up, p0[i].up, p1[i].up);
#pragma unroll
              for (int i = 0; i < 4; ++i) mma(small[i], up, p0[i].low, p1[i].low);
#pragma unroll
              for (int i = 0; i < 4; ++i) mma(small[i], dn, p0[i].up, p1[i].up);
            }
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[4 * h + n][i] = fmaf(o[4 * h + n][i], al[i >> 1], big[n][i] + small[n][i]);
          }
        } else {
#pragma unroll
          for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][i] *= al[i >> 1];
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
              const int from = (lane & ~3) | (k >> 1), slot = 8 * (n & 1) + k;
              float p[2];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float x = __shfl_sync(FULL, s[n][2 * h], from), y = __shfl_sync(FULL, s[n][2 * h + 1], from);
                p[h] = (k & 1) ? y : x;
              }
#pragma unroll
              for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int dim = 32 * (i >> 2) + 4 * (2 * t + (e & 1)) + (i & 3), h = e >> 1;
                  if (seen[h][n >> 1] >> slot & 1)
                    o[i][e] = fmaf(p[h], vt[at_v(8 * n + k, dim >> 2) + (dim & 3)], o[i][e]);
                }
            }
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(FULL, l[h], 1);
      l[h] += __shfl_xor_sync(FULL, l[h], 2);
      const int tok = tok0 + 2 * h;
      if (tok >= si.t) continue;
      const size_t row = (size_t)(si.q_row0 + tok) * d.q_heads + head * G + g % G;
      if constexpr (STATS) {
        if (t == 0) stats[(size_t)part * d.g->total_tokens * d.q_heads + row] = make_float2(m[h], l[h]);
      } else {
        if (parts > 1) {
          const int r = 16 * warp + g + 8 * h;
          float4* to = part_rows<D>(d, it.at) + r;
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              to[(2 * t + 8 * c + e) * PART_ROWS] = make_float4(o[4 * c][2 * h + e], o[4 * c + 1][2 * h + e],
                                                                o[4 * c + 2][2 * h + e], o[4 * c + 3][2 * h + e]);
          if (t == 0) part_sums<D>(d, it.at)[r] = make_float2(m[h], l[h]);
          continue;
        }
        const float inv = 1.f / l[h];
        float4* to = reinterpret_cast<float4*>(out + row * D + 8 * t);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            to[8 * c + e] = make_float4(o[4 * c][2 * h + e] * inv, o[4 * c + 1][2 * h + e] * inv,
                                        o[4 * c + 2][2 * h + e] * inv, o[4 * c + 3][2 * h + e] * inv);
      }
    }
  }
  if (tid == 0) leave_counters(d);
}

// ---------------------------------------------------------------------------
// Sums by key: an item is 128 keys of one session and KV head, 16 a warp, and a share of the chunk's
// tokens, 16 (64 rows) at a time.
// ---------------------------------------------------------------------------
constexpr int KEYS = 16 * WARPS, KEY_PAGES = KEYS / PS;
constexpr int STEP_TOKENS = KT / G;
constexpr int SUMS_SMEM = (2 * KEYS * D + 2 * TILE) * 4;

__global__ void __launch_bounds__(THREADS, CTAS) weights_sums_f32_kernel(Dev d, int layer,
                                                                   const float* __restrict__ q, float scale,
                                                                   int most_parts, int shares, WeightsWork work) {
  extern __shared__ __align__(16) float sm[];
  __shared__ int s_group[GROUPS + 1];
  __shared__ Item s_item;
  __shared__ __align__(8) float s_lse[2][KT];
  static_assert(KT <= THREADS, "a thread a row");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, H = d.kv_heads;
  float *s_k = sm, *s_q = sm + 2 * KEYS * D;
  pdl_wait();
  pdl_launch_dependents();
  const int n_seq = d.g->total_tokens > 0 ? d.g->n_seq : 0;
  const int total = d.g->total_tokens, parts = stat_parts(d, most_parts, total);
  auto items_of = [&](int i) { return (d.seq[i].n_blocks + KEY_PAGES - 1) / KEY_PAGES * H * shares; };
  if (warp == 0) list_items(n_seq, lane, s_group, items_of);
  for (;;) {
    const Item it = next_item(d, n_seq, 1, s_group, &s_item, items_of);
    if (it.seq < 0) break;
    const SeqInfo si = d.seq[it.seq];
    const int head = it.in % H, share = it.in / H % shares, b0 = it.in / H / shares * KEY_PAGES;
    const int steps = (si.t + STEP_TOKENS - 1) / STEP_TOKENS, q_log0 = si.n_hist + si.n_live - si.t;
    const int first = max(0, block_range(si, b0).base - q_log0) / STEP_TOKENS;
    const int i0 = first + (int)((int64_t)(steps - first) * share / shares);
    const int i1 = first + (int)((int64_t)(steps - first) * (share + 1) / shares);
    auto stage = [&](int i) {
      stage_rows<KT>(d, si, head, i * STEP_TOKENS, q, scale, s_q + (i & 1) * TILE, 0);
      if (tid < KT) {  // rows past the chunk draw nothing
        const int tok = i * STEP_TOKENS + tid / G;
        float lse = INFINITY;
        if (tok < si.t)
          lse = row_lse(work.stats + (size_t)(si.q_row0 + tok) * d.q_heads + head * G + tid % G,
                        (size_t)total * d.q_heads, parts);
        s_lse[i & 1][tid] = lse;
      }
    };
    if (i0 < i1) {
      int pages[KEY_PAGES];
      look_up(d, si, b0, si.n_blocks, pages);
      load_pages(d, layer, head, pages, s_k, nullptr);
      cp_async_commit();
      stage(i0);
      cp_async_wait_all();
      // Into pieces: each thread what it brought.
      for (int r = tid >> 4; r < KEYS; r += THREADS / 16) {
        float* at = s_k + at_k(r, tid & 15);
        put_pieces(*reinterpret_cast<const float4*>(at), at, KEYS * D);
      }
    }
    // This lane's keys: 16 warp + g and + 8, and the first token that sees each.
    const int blk = b0 + warp;
    const BlockRange br = blk < si.n_blocks ? block_range(si, blk) : BlockRange{0, 0, 0};
    int from[2];
    bool in[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      in[h] = g + 8 * h >= br.lo && g + 8 * h < br.hi;
      from[h] = br.base + g + 8 * h - q_log0;
    }
    float sum[2] = {0.f, 0.f}, rest[2] = {0.f, 0.f};  // (rest: what additions to the sums rounded off)
    for (int i = i0; i < i1; ++i) {
      const float* tile = s_q + (i & 1) * TILE;
      if (i > i0) stage(i);
      __syncthreads();
      float s[NT][4], add[2] = {0.f, 0.f};
      products(s_k, KEYS * D, 16 * warp, tile, lane, s);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 lse = *reinterpret_cast<const float2*>(&s_lse[i & 1][8 * n + 2 * t]);
        const int tok = i * STEP_TOKENS + (8 * n + 2 * t) / G;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (tok >= from[h]) add[h] += ex2(s[n][2 * h] - lse.x) + ex2(s[n][2 * h + 1] - lse.y);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float a = add[h] + rest[h], to = sum[h] + a;
        rest[h] = a - (to - sum[h]);
        sum[h] = to;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sum[h] += __shfl_xor_sync(FULL, sum[h], 1);
      sum[h] += __shfl_xor_sync(FULL, sum[h], 2);
      if (t != 0 || !in[h]) continue;
      const int page = block_page(si, d.hist_pt + (size_t)si.sid * d.max_pages_per_session,
                                  d.live_pt + (size_t)si.sid * d.max_pages_per_session, blk);
      if (isnan(sum[h])) {
        const Dev dev = d;  // (copies, so that only this branch has them in memory)
        const SeqInfo info = si;
        sum[h] = plain_sum<float, D>(dev, info, layer, head, page, g + 8 * h, max(i0 * STEP_TOKENS, from[h]),
                                     min(i1 * STEP_TOKENS, si.t), q, scale, work.stats, parts);
      }
      work.scores[((size_t)(head * shares + share) * d.n_pages + page) * PS + g + 8 * h] = sum[h];
    }
  }
  if (tid == 0) leave_counters(d);
}

__global__ void __launch_bounds__(MERGE_THREADS) prompt_merge_f32_kernel(Dev d, float* out, int parts) {
  merge_parts<float, D, 1>(d, out, parts, [](const SeqInfo&, int, int, int) { return false; });
}

template <typename K>
cudaError_t most_smem(K* kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

float score_scale() { return LOG2E / sqrtf((float)D); }

}  // namespace

cudaError_t prompt_f32_attributes() {
  cudaError_t e = most_smem(prompt_f32_kernel<false>, PROMPT_SMEM);
  if (e == cudaSuccess) e = most_smem(prompt_f32_kernel<true>, STAT_SMEM);
  return e != cudaSuccess ? e : most_smem(weights_sums_f32_kernel, SUMS_SMEM);
}

cudaError_t launch_prompt_f32(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int parts,
                              int64_t items, cudaStream_t s, int64_t* launches) {
  float* to = static_cast<float*>(out);
  cudaError_t e = launch_ex(&prompt_f32_kernel<false>, dim3(lim.sms * CTAS), dim3(THREADS), PROMPT_SMEM, s, true,
                            d, layer, static_cast<const float*>(q), to, score_scale(), parts,
                            static_cast<float2*>(nullptr));
  *launches += e == cudaSuccess;
  if (e != cudaSuccess || parts == 1) return e;
  e = launch_ex(&prompt_merge_f32_kernel, dim3(merge_grid(items, D)), dim3(MERGE_THREADS), 0, s, true, d, to,
                parts);
  *launches += e == cudaSuccess;
  return e;
}

cudaError_t launch_weights_f32(const Dev& d, const Limits& lim, int layer, const void* q,
                               const WeightsWork& work, int parts, int shares, cudaStream_t s,
                               int64_t* launches) {
  const float* qf = static_cast<const float*>(q);
  cudaError_t e = launch_ex(&prompt_f32_kernel<true>, dim3(lim.sms * CTAS), dim3(THREADS), STAT_SMEM, s, true, d,
                            layer, qf, static_cast<float*>(nullptr), score_scale(), parts, work.stats);
  *launches += e == cudaSuccess;
  if (e != cudaSuccess) return e;
  e = launch_ex(&weights_sums_f32_kernel, dim3(lim.sms * CTAS), dim3(THREADS), SUMS_SMEM, s, true, d, layer, qf,
                score_scale(), parts, shares, work);
  *launches += e == cudaSuccess;
  return e;
}

}  // namespace kvc
