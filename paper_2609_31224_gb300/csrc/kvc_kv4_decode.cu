// Single-token decode attention over a cache held in 4 bits (KVC_KV4).
//
// For each session of the last append (one token each), KV head and its G = 4 query heads:
// out = softmax(RoPE(q) . k / sqrt(D)) v over every resident key, k and v the numbers that the codes
// stand for.
//
// A warp takes a page of 16 keys at a time, as one step of mma.sync m16n8k16 (binary16 in, binary32
// accumulate) with the keys as M:
//   S^T [16 keys x 8] = K [16 x D] . Q^T [D x 8],   O^T [D x 8] += V^T [D x 16] . P^T [16 x 8].
// The eight columns are two binary16 pieces of each of the four heads (column 2h: q rounded, 2h + 1:
// what the rounding left), so that lane (g, t) ends with both pieces of head t for keys g and g + 8:
// their sum is a score with about 22 bits of q, one softmax state per lane, no lane idle.  binary32
// calls split P the same way; for bfloat16 the rounding of P to 11 bits stays.
//
// What bounds it: 18 D bytes a page (44 us for 64 sessions of 4,096 positions) against about 280
// warp instructions, 80 for the scores, 125 for P V (most of both the way from nibble to operand) and
// the rest ring, masks and softmax.  K's nibbles go in as they are (an AND each: bits 0..3 and 4..7 of
// a half are binary16 numbers n 2^-24 and n 2^-20) with scale and zero behind the product, which a
// group of 32 dims does not cross; V's take an AND-OR and one or two products each.  The rest is kept
// small: the query's operands stay in registers, the softmax reference lags (it moves only when a
// score passes it by 2^6), two pages make a step, page lists are looked up 32 at a time, and only
// pages with masked slots look at their range.  64 sessions: 60.9 us (72 % of the bytes' rate; 105 us
// as first written, 517 instructions), against 159 us for bfloat16 rows; issue is at 55 %, and 16 warps
// an SM is what 128 registers leave.  One session: 5.7 us against 0.7 us for its bytes, a chain (release
// by the launch before 0.9, query 0.5, two pages a warp 1.3, the CTA's merge 0.9, arrival 0.7, the pair's
// merge 1.3), in which the number of instructions one after the other is what counts.
#include <algorithm>

#include "kvc_kv4.cuh"
#include "kvc_kv4_cuts.h"

namespace kvc {

namespace {

using namespace kv4;

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int G = 4;               // query heads per KV head
constexpr float LOG2E = 1.4426950408889634f;
constexpr float P_SHIFT = 8.f;     // log2 of the weight P of a key at the reference
constexpr float P_LAG = 6.f;       // and of how far above it a weight may be: 2^14 in all

// Shape of a CTA: WARPS warps, each with its own ring of STAGES pairs of pages.
template <typename T_, int D_, int WARPS_, int STAGES_>
struct Cfg {
  using T = T_;
  static constexpr int D = D_, WARPS = WARPS_, STAGES = STAGES_, THREADS = 32 * WARPS_;
  static constexpr bool SPLIT_P = sizeof(T) == 4;  // P in two binary16 pieces
  static constexpr bool SCALE_BEHIND = !SPLIT_P;   // K's scales come in behind the product
  static constexpr int PAGE = 18 * D;              // bytes of a page of one head, K and V
  static constexpr int KW = D / 32;                // 32-bit words of K codes per lane and row
  static constexpr int VW = D / 64;                // and of V codes per lane and row
  static constexpr int MT = D / 16;                // row tiles of O^T
  // Shared memory: rings, the warps' states, weights of parts, barriers.
  static constexpr int RING = WARPS * STAGES * 2 * PAGE;
  static constexpr int STATE_O = RING;                          // [WARPS][G][D] floats
  static constexpr int STATE_ML = STATE_O + WARPS * G * D * 4;  // [WARPS][G] (m, l)
  static constexpr int PARTS_ROOM = 96;                         // parts and a batch past them
  static constexpr int WEIGHT = STATE_ML + WARPS * G * 8;       // [PARTS_ROOM][G], of parts
  static constexpr int BARS = WEIGHT + PARTS_ROOM * G * 4;
  static_assert(PARTS_ROOM >= DECODE_MAX_PARTS + 20, "room for zeros");
  static constexpr int SMEM = BARS + WARPS * STAGES * 8;
  static_assert(PAGE % 16 == 0 && RING % 16 == 0 && BARS % 8 == 0, "alignment");
};

__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Weight of a state with reference m against the reference M of several, 0 where it has no key.
// References are of the raw products S, c is the row's softmax scale: S - m is rounded before c
// comes in, so that logits of any size leave exponents that are exact near 0.
__device__ inline float weight2(float m, float M, float c) {
  return m == -INFINITY ? 0.f : ex2((m - M) * c);
}

// The query of a pair in this warp's registers.
template <class C>
struct Query {
  // Lane (n, t) holds, for column n (head n / 2, piece n % 2), the pairs (p, p + 4) of dims
  // [32 w + 8 t, 32 w + 8 t + 8); where the scales come in behind the product, pairs 1 and 3 (whose
  // nibbles are read 16 times too large) over 16.
  uint32_t b[C::KW][4];
  float c;        // softmax scale of head t
  float zero[C::KW];  // -8 times the sum of a group's dims of head t: takes the 8 off its nibbles
};

constexpr int Q_EXP = 9;        // a row's largest element is in [2^9, 2^10)
constexpr int RAW_EXP = -24;    // a nibble's bits 0..3 as a binary16 number are n 2^-24

// The query of a pair as it is staged for all warps of a CTA.
template <class C>
struct StagedQuery {
  uint32_t b[C::KW][32][4];
  float zero[G][C::KW];
  float c[G];
};

// Head h of the pair, by one warp: lane (w, t, p) takes dims a = 32 w + 8 t + p and a + 4 and the
// rotate-half partners of both, which are pair p of words w and w + D / 64.  (Every warp for itself took
// 450 instructions before its first page.)
template <class C>
__device__ inline void stage_query(const Dev& d, const SeqInfo& si, int head, int h,
                                   const typename C::T* q, int lane, StagedQuery<C>& sq) {
  constexpr int D = C::D, KW = C::KW, HALF = D / 2;
  const int w = lane / 16 % (KW / 2), t = lane / 4 % 4, p = lane % 4, a = GROUP * w + 8 * t + p;
  const typename C::T* row = q + ((size_t)si.q_row0 * d.q_heads + head * G + h) * D + a;
  const float x[4] = {to_float<typename C::T>(row[0]), to_float<typename C::T>(row[4]),
                      to_float<typename C::T>(row[HALF]), to_float<typename C::T>(row[HALF + 4])};
  const float2* cs = d.rope + (size_t)si.pos_first * HALF + a;
  float y[2][2];  // [word w, its partner][dim a, dim a + 4]
  turn_pair(x[0], x[2], cs[0], y[0][0], y[1][0]);
  turn_pair(x[1], x[3], cs[4], y[0][1], y[1][1]);
  uint32_t most = max(max(abs_bits(y[0][0]), abs_bits(y[0][1])), max(abs_bits(y[1][0]), abs_bits(y[1][1])));
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) most = max(most, __shfl_xor_sync(FULL, most, o));
  // The row over 2^e.  Infinities and NaN pass through.
  int e = (int)(most >> 23) - 127 - Q_EXP;
  e = most >= 0x7F800000u ? 0 : max(e, -126);
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  float sum[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float y0 = y[i][0] * inv, y1 = y[i][1] * inv;
    const __half2 hi = __floats2half2_rn(y0, y1);
    const __half2 lo = __floats2half2_rn(y0 - __low2float(hi), y1 - __high2float(hi));
    // (Where the scales come in behind the product; exact but for the last bits of small numbers.)
    const bool over16 = C::SCALE_BEHIND && (p & 1);
    const __half2 f = __float2half2_rn(over16 ? 0.0625f : 1.f), vh = __hmul2(hi, f), vl = __hmul2(lo, f);
    sum[i] = ((__low2float(vh) + __high2float(vh)) + (__low2float(vl) + __high2float(vl))) *
             (over16 ? 16.f : 1.f);
    sq.b[w + i * (KW / 2)][8 * h + t][p] = h2_bits(vh);
    sq.b[w + i * (KW / 2)][8 * h + 4 + t][p] = h2_bits(vl);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) sum[i] += __shfl_xor_sync(FULL, sum[i], o);
  if (lane % 16 == 0)
#pragma unroll
    for (int i = 0; i < 2; ++i) sq.zero[h][w + i * (KW / 2)] = sum[i] * (-8.f / (float)(1 << -RAW_EXP));
  // 16: scales are stored over 16; and the softmax takes exponents of 2.  (Beyond binary32 it is large
  // enough to single out a maximum.)
  const float scale = 16.f * LOG2E * (D == 128 ? 0.08838834764831845f : 0.125f);
  const float c = scale * __uint_as_float((uint32_t)(127 + e) << 23) *
                  (C::SCALE_BEHIND ? (float)(1 << -RAW_EXP) : 1.f);
  if (lane == 0) sq.c[h] = fminf(c, 3.4e38f);
}

template <class C>
__device__ inline void load_query(const StagedQuery<C>& sq, int lane, Query<C>& qr) {
#pragma unroll
  for (int w = 0; w < C::KW; ++w) {
    const uint4 v = *reinterpret_cast<const uint4*>(sq.b[w][lane]);
    qr.b[w][0] = v.x;
    qr.b[w][1] = v.y;
    qr.b[w][2] = v.z;
    qr.b[w][3] = v.w;
    qr.zero[w] = sq.zero[lane & 3][w];
  }
  qr.c = sq.c[lane & 3];
}

// Which pages of a session need no look at their slots: full pages of the compacted region and live
// pages between the consumed front and the partly filled end.
struct OpenPages {
  int hist_full, live_first, live_last;
  __device__ explicit OpenPages(const SeqInfo& si) {
    hist_full = si.n_hist / PS;
    live_first = si.n_hist_pages + (si.live_head + PS - 1) / PS;
    live_last = si.n_hist_pages + (si.live_head + si.n_live) / PS - 1;
  }
  // Blocks b to e (those of a warp among them).
  __device__ bool has(int b, int e) const {
    return e < hist_full || (b >= live_first && e <= live_last);
  }
};

// A warp's running state: head t, this lane's keys (l) and its 16 (8) dims of piece g (o).
template <class C>
struct State {
  float o[C::MT][4];
  float m, l;
};

// Scores of keys g and g + 8 of a page for head t.
template <class C>
__device__ inline void page_scores(uint32_t kt, const Query<C>& qr, int lane, float& s0, float& s1) {
  constexpr int D = C::D, KW = C::KW;
  const int g = lane >> 2, t = lane & 3;
  uint32_t wa[KW], wb[KW], ma[KW / 2], mb[KW / 2];
  lds(kt + g * (D / 2) + t * (D / 8), wa);
  lds(kt + (g + 8) * (D / 2) + t * (D / 8), wb);
  lds(kt + k_scale(D, g, 0), ma);
  lds(kt + k_scale(D, g + 8, 0), mb);
  float x[KW][4];
  const __half2 m72 = __float2half2_rn(-72.f);
  if constexpr (C::SCALE_BEHIND) {
    const float none[4] = {0.f, 0.f, 0.f, 0.f};
    // Nibbles as they are: bits 0..3 of a half are n 2^-24, bits 4..7 n 2^-20.
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const uint32_t ha = wa[w] >> 8, hb = wb[w] >> 8;
      mma_f16(x[w], wa[w] & 0x000F000Fu, wb[w] & 0x000F000Fu, wa[w] & 0x00F000F0u,
              wb[w] & 0x00F000F0u, qr.b[w][0], qr.b[w][1], none);
      mma_f16(x[w], ha & 0x000F000Fu, hb & 0x000F000Fu, ha & 0x00F000F0u, hb & 0x00F000F0u,
              qr.b[w][2], qr.b[w][3]);
    }
    float2 z0 = make_float2(0.f, 0.f), z1 = z0;
#pragma unroll
    for (int w = 0; w < KW; w += 2) {
      const float2 a = __half22float2(bits_h2(ma[w / 2])), b = __half22float2(bits_h2(mb[w / 2]));
      const float2 zero = make_float2(qr.zero[w], qr.zero[w + 1]);
      z0 = __ffma2_rn(__fadd2_rn(make_float2(x[w][0] + x[w][1], x[w + 1][0] + x[w + 1][1]), zero), a, z0);
      z1 = __ffma2_rn(__fadd2_rn(make_float2(x[w][2] + x[w][3], x[w + 1][2] + x[w + 1][3]), zero), b, z1);
    }
    s0 = z0.x + z0.y;
    s1 = z1.x + z1.y;
  } else {
    // Exact values of the keys, and a sum for every 16 dims: the tensor cores cut off what they
    // add to an accumulator.
    float z[KW][4];
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const uint32_t da = __byte_perm(ma[w / 2], 0, w % 2 ? 0x3232u : 0x1010u);
      const uint32_t db = __byte_perm(mb[w / 2], 0, w % 2 ? 0x3232u : 0x1010u);
      uint32_t a[4], b[4];
      pairs_of(wa[w], bits_h2(da), __hmul2(bits_h2(da), m72), a);
      pairs_of(wb[w], bits_h2(db), __hmul2(bits_h2(db), m72), b);
      x[w][0] = x[w][1] = x[w][2] = x[w][3] = z[w][0] = z[w][1] = z[w][2] = z[w][3] = 0.f;
      mma_f16(x[w], a[0], b[0], a[1], b[1], qr.b[w][0], qr.b[w][1]);
      mma_f16(z[w], a[2], b[2], a[3], b[3], qr.b[w][2], qr.b[w][3]);
    }
    s0 = s1 = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      s0 += x[w][1] + z[w][1];
      s1 += x[w][3] + z[w][3];
    }
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      s0 += x[w][0] + z[w][0];
      s1 += x[w][2] + z[w][2];
    }
  }
}

// O^T += V^T P^T of a page; b0, b1: P^T of rows 2t, 2t + 1 and 2t + 8, 2t + 9 for column g.
template <class C>
__device__ inline void page_values(uint32_t vt, uint32_t b0, uint32_t b1, bool open,
                                   const BlockRange& br, State<C>& st, int lane) {
  constexpr int D = C::D, VW = C::VW;
  const int g = lane >> 2, t = lane & 3;
  const __half2 m72 = __float2half2_rn(-72.f);
  // V^T: lane (g, t) takes piece g of rows 2t, 2t + 1 (lo) and 2t + 8, 2t + 9 (hi).
  uint32_t lo[2 * VW], hi[2 * VW], sl, sh;  // [row of the pair][word]
  lds(vt + lane * (D / 8), lo);
  lds(vt + D * 4 + lane * (D / 8), hi);
  const uint32_t sc = vt + v_scale(D, 2 * t, g * (D / 8) / GROUP);
  lds(sc, sl);
  lds(sc + 16, sh);
  if (!open) {
    // Invalid slots stand for 0, whatever the page held there before.
    const int i = 2 * t;
    if (i < br.lo || i >= br.hi) sl &= 0xFFFF0000u;
    if (i + 1 < br.lo || i + 1 >= br.hi) sl &= 0x0000FFFFu;
    if (i + 8 < br.lo || i + 8 >= br.hi) sh &= 0xFFFF0000u;
    if (i + 9 < br.lo || i + 9 >= br.hi) sh &= 0x0000FFFFu;
  }
  const __half2 ml = bits_h2(sl), mh = bits_h2(sh);
  const __half2 nl = __hmul2(ml, m72), nh = __hmul2(mh, m72);
#pragma unroll
  for (int w = 0; w < VW; ++w)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      // Dims 8 w + 4 half + 0..3 of the piece: nibble p of both halves of a word, the pair's rows.
      const uint32_t sel = half ? 0x7632u : 0x5410u;
      uint32_t a[4], b[4];
      pairs_of(__byte_perm(lo[w], lo[VW + w], sel), ml, nl, a);
      pairs_of(__byte_perm(hi[w], hi[VW + w], sel), mh, nh, b);
      const int mt = 4 * w + 2 * half;
      if constexpr (C::SPLIT_P) {
        // A page's sums by themselves, then added rounded (as above).
        float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16(x, a[0], a[1], b[0], b[1], b0, b1);
        mma_f16(y, a[2], a[3], b[2], b[3], b0, b1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          st.o[mt][j] += x[j];
          st.o[mt + 1][j] += y[j];
        }
      } else {
        mma_f16(st.o[mt], a[0], a[1], b[0], b[1], b0, b1);
        mma_f16(st.o[mt + 1], a[2], a[3], b[2], b[3], b0, b1);
      }
    }
}

// Weights of two keys (g and g + 8 of a page) as the B operand of page_values; adds them to l.
template <class C>
__device__ inline void weights_of(float a0, float a1, float& l, uint32_t& b0, uint32_t& b1) {
  const float p0 = ex2(a0), p1 = ex2(a1);
  l += p0 + p1;
  if constexpr (C::SPLIT_P) {
    const float h0 = __half2float(__float2half_rn(p0)), h1 = __half2float(__float2half_rn(p1));
    b0 = transpose8(h2_bits(__floats2half2_rn(h0, p0 - h0)));
    b1 = transpose8(h2_bits(__floats2half2_rn(h1, p1 - h1)));
  } else {
    b0 = transpose8(h2_bits(__floats2half2_rn(p0, 0.f)));
    b1 = transpose8(h2_bits(__floats2half2_rn(p1, 0.f)));
  }
}

// N pages (in shared memory at `at`, blocks blk and blk + WARPS): scores, running softmax, P V.
template <class C, int N>
__device__ inline void pages_step(uint32_t at, const Query<C>& qr, const OpenPages& pages,
                                  const SeqInfo& si, int blk, State<C>& st, int lane) {
  const int g = lane >> 2;
  float s[N][2];
  const bool open = pages.has(blk, blk + (N - 1) * C::WARPS);
  BlockRange br[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    page_scores<C>(at + i * C::PAGE, qr, lane, s[i][0], s[i][1]);
    if (!open) {
      br[i] = block_range(si, blk + i * C::WARPS);
      if (g < br[i].lo || g >= br[i].hi) s[i][0] = -INFINITY;
      if (g + 8 < br[i].lo || g + 8 >= br[i].hi) s[i][1] = -INFINITY;
    }
  }
  float a[N][2], most = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      a[i][j] = fmaf(s[i][j] - st.m, qr.c, P_SHIFT);
      most = fmaxf(most, a[i][j]);
    }
  // (At the first page m is -infinity: every valid key asks for a new reference.)
  if (__any_sync(FULL, most > P_SHIFT + P_LAG)) {
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) mx = fmaxf(mx, fmaxf(s[i][0], s[i][1]));
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, off));
    const float mn = fmaxf(st.m, mx);
    const float alpha = weight2(st.m, mn, qr.c);
    st.l *= alpha;
#pragma unroll
    for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j) st.o[mt][j] *= alpha;
    st.m = mn;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) a[i][j] = fmaf(s[i][j] - mn, qr.c, P_SHIFT);
  }
  uint32_t b[N][2];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (!open) {
      // (Where no key was valid so far s - m is no number.)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (s[i][j] == -INFINITY) a[i][j] = -INFINITY;
    }
    weights_of<C>(a[i][0], a[i][1], st.l, b[i][0], b[i][1]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    page_values<C>(at + i * C::PAGE + 9 * C::D, b[i][0], b[i][1], open, br[i], st, lane);
}

// The new token's K (rotated at its position) and V of this layer and head, from the caller's rows,
// into their slot of the pool and of the page just loaded from it (whose copy may be older), as the
// write kernel would have them.  By the warp that has the pair's last block.
template <class C>
__device__ void write_new_row(const Dev& d, int layer, const SeqInfo& si, int head,
                              const typename C::T* nk, const typename C::T* nv, uint8_t* page,
                              int lane) {
  using T = typename C::T;
  constexpr int D = C::D, HALF = D / 2, E = D / 32, LANES = GROUP / E;  // elements, lanes of a group
  const int gs = d.tok_slot[si.q_row0], slot = gs % PS, d0 = lane * E;
  const size_t row = ((size_t)si.q_row0 * d.kv_heads + head) * D;
  float x[E], partner[E], y[2][E];
  float2 cs[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = to_float<T>(nk[row + d0 + e]);
    partner[e] = to_float<T>(nk[row + (d0 ^ HALF) + e]);
    y[1][e] = to_float<T>(nv[row + d0 + e]);
    cs[e] = d.rope[(size_t)si.pos_first * HALF + (d0 & (HALF - 1)) + e];
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    float other;
    if (d0 < HALF) turn_pair(x[e], partner[e], cs[e], y[0][e], other);
    else turn_pair(partner[e], x[e], cs[e], other, y[0][e]);
  }
  uint8_t* tiles = d.pool + tile_at(D, d.layers, d.kv_heads, gs / PS, layer, head, 0);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint32_t most = most_of(y[kv]);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) most = max(most, __shfl_xor_sync(FULL, most, o));
    const float s = scale_of(most);
    const Divisor div(s);
    if (div.passes(most)) hold_codes(y[kv], div.by);
    const uint32_t codes = codes_of(y[kv], div.inv, div.rest);
    const int at = kv * 9 * D + (kv ? v_codes(D, slot, d0 & ~7) : k_codes(D, slot, d0 & ~7)) +
                   d0 % 8 / 2;
    if constexpr (E == 4) {
      *reinterpret_cast<uint16_t*>(tiles + at) = (uint16_t)codes;
      *reinterpret_cast<uint16_t*>(page + at) = (uint16_t)codes;
    } else {
      tiles[at] = page[at] = (uint8_t)codes;
    }
    if (lane % LANES == 0) {
      const int group = lane / LANES;
      const int sc = kv * 9 * D + (kv ? v_scale(D, slot, group) : k_scale(D, slot, group));
      *reinterpret_cast<__half*>(tiles + sc) = stored_scale(s);
      *reinterpret_cast<__half*>(page + sc) = stored_scale(s);
    }
  }
  __syncwarp();
}

// The pages of one warp and segment (every WARPS-th block), through the warp's ring.  What is looked at
// once in 16 steps stays in the warp's copy of the segment in shared memory: the registers of the main
// loop are all taken (with 20 of these in registers instead, spills were 25 instructions a page).
template <class C>
struct Ring {
  uint8_t* slots;
  uint64_t* full;
  const uint8_t* tiles;      // of the layer and head in page 0
  const UnitSeg* seg;
  int first, n_my, win, pid;

  __device__ void open(const Dev& d, int layer, const UnitSeg* s, int warp) {
    seg = s;
    tiles = d.pool + tile_at(C::D, d.layers, d.kv_heads, 0, layer, s->head, 0);
    first = s->blk_begin() + warp;
    const int n = s->end - s->u;
    n_my = n > warp ? (n - warp + C::WARPS - 1) / C::WARPS : 0;
    win = -32;
    pid = 0;
  }
  __device__ int steps() const { return (n_my + 1) / 2; }
  // Copy the warp's k-th pair of pages in, as its n-th of the launch; the whole warp.
  __device__ void issue(const Dev& d, int k, uint32_t n, int lane) {
    if (2 * k >= win + 32) {
      win = (2 * k) & ~31;
      const int j = win + lane, b = first + j * C::WARPS, nh = seg->si.n_hist_pages;
      const size_t row = (size_t)seg->si.sid * d.max_pages_per_session;
      pid = j < n_my ? (b < nh ? d.hist_pt[row + b] : d.live_pt[row + b - nh]) : 0;
    }
    const int p0 = __shfl_sync(FULL, pid, 2 * k - win), p1 = __shfl_sync(FULL, pid, 2 * k + 1 - win);
    if (lane == 0) {
      const uint32_t st = n % C::STAGES;
      const size_t stride = page_bytes(C::D, d.layers, d.kv_heads);
      const uint64_t policy = evict_first_policy();
      uint8_t* to = slots + st * 2 * C::PAGE;
      const bool two = 2 * k + 1 < n_my;
      fence_proxy_async_smem();
      mbar_arrive_expect_tx(&full[st], two ? 2 * C::PAGE : C::PAGE);
      bulk_g2s_hint(to, tiles + p0 * stride, C::PAGE, &full[st], policy);
      if (two) bulk_g2s_hint(to + C::PAGE, tiles + p1 * stride, C::PAGE, &full[st], policy);
    }
  }
};

// N floats as one access (N = 1, 2 or 4).
template <int N>
struct Floats {
  float v[N];
  __device__ static Floats load(const float* p) {  // of global memory, past L1
    Floats f;
    if constexpr (N == 4) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(p));
      f.v[0] = x.x; f.v[1] = x.y; f.v[2] = x.z; f.v[3] = x.w;
    } else if constexpr (N == 2) {
      const float2 x = __ldcg(reinterpret_cast<const float2*>(p));
      f.v[0] = x.x; f.v[1] = x.y;
    } else {
      f.v[0] = __ldcg(p);
    }
    return f;
  }
  __device__ static Floats load_shared(const float* p) {
    Floats f;
    if constexpr (N == 4) {
      const float4 x = *reinterpret_cast<const float4*>(p);
      f.v[0] = x.x; f.v[1] = x.y; f.v[2] = x.z; f.v[3] = x.w;
    } else if constexpr (N == 2) {
      const float2 x = *reinterpret_cast<const float2*>(p);
      f.v[0] = x.x; f.v[1] = x.y;
    } else {
      f.v[0] = *p;
    }
    return f;
  }
  __device__ void store(float* p) const {
    if constexpr (N == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else if constexpr (N == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
    else *p = v[0];
  }
  template <typename T>
  __device__ void store_row(T* p) const {
    if constexpr (sizeof(T) == 4) {
      store(reinterpret_cast<float*>(p));
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2)
        *reinterpret_cast<__nv_bfloat162*>(p + i) = __floats2bfloat162_rn(v[i], v[i + 1]);
    }
  }
};

// Rows of a pair from the parts that cover it, by every thread of the last CTA to arrive: part 0 is in
// slot `first`, part i in next + step i; [G][D] outputs and (m, l) per head.  A thread takes EPT elements
// side by side; parts that are not there have weight 0 (the chain of instructions is what this costs).
template <class C>
__device__ void merge_parts(const float* part_o, const float2* part_ml, int parts, int first, int next,
                            int step, const float* scale, float* weight, typename C::T* out, int tid) {
  constexpr int D = C::D, E = G * D, EPT = E / C::THREADS;
  // Parts whose loads are in flight together: more than the 17 that one session's pairs are cut into.
  constexpr int BATCH = C::WARPS == 8 ? 20 : 32 / EPT;
  const int lane = tid & 31, warp = tid >> 5, e0 = tid * EPT, h = e0 / D;
  const float* p = part_o + (size_t)next * E + e0;
  const uint32_t stride = step * E;
  const Floats<EPT> x0 = Floats<EPT>::load(part_o + (size_t)first * E + e0);
  Floats<EPT> x[BATCH];
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      x[i] = {};
      if (i0 + i < parts) x[i] = Floats<EPT>::load(p + (i0 + i) * stride);
    }
  };
  load(1);
  if (warp < G) {
    constexpr int PL = C::PARTS_ROOM / 32;
    float2 ml[PL];
    float M = -INFINITY, L = 0.f, w[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const int k = lane + 32 * i;
      ml[i] = k < parts ? __ldcg(&part_ml[(size_t)(k ? next + step * k : first) * G + warp])
                        : make_float2(-INFINITY, 0.f);
      M = fmaxf(M, ml[i].x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(FULL, M, o));
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      w[i] = weight2(ml[i].x, M, scale[warp]);
      L += ml[i].y * w[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(FULL, L, o);
    const float inv = 16.f / L;
#pragma unroll
    for (int i = 0; i < PL; ++i) weight[(lane + 32 * i) * G + warp] = w[i] * inv;
  }
  __syncthreads();
  const float* w = weight + h;
  Floats<EPT> acc;
#pragma unroll
  for (int k = 0; k < EPT; ++k) acc.v[k] = x0.v[k] * w[0];
  for (int i0 = 1;;) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
#pragma unroll
      for (int k = 0; k < EPT; ++k) acc.v[k] += x[i].v[k] * w[(i0 + i) * G];
    i0 += BATCH;
    if (i0 >= parts) break;
    load(i0);
  }
  acc.store_row(out + e0);
}

// How a call's pages reach the CTAs: slices >= 1 cuts each (session, KV head) pair into as many
// slices, one CTA each (no more than it has pages); 0 cuts the call's units evenly over the grid
// (stream-K), at least min_units to a CTA.
struct Cut {
  int slices, min_units;
};

// Query rows and rotary row of a pair into L2 (what later loads observe does not depend on it).
template <class C>
__device__ inline void prefetch_query(const Dev& d, const SeqInfo& si, int head,
                                      const typename C::T* q, int lane) {
  constexpr int QL = G * C::D * (int)sizeof(typename C::T) / 128, RL = C::D * 4 / 128;
  const uint8_t* qa = reinterpret_cast<const uint8_t*>(q + ((size_t)si.q_row0 * d.q_heads + head * G) * C::D);
  const uint8_t* ra = reinterpret_cast<const uint8_t*>(d.rope + (size_t)si.pos_first * (C::D / 2));
  if (lane < QL) prefetch_l2(qa + 128 * lane);
  else if (lane >= 16 && lane < 16 + RL) prefetch_l2(ra + 128 * (lane - 16));
}

template <class C, bool FUSED>
__global__ void __launch_bounds__(C::THREADS, 16 / C::WARPS) decode_kv4_kernel(
    Dev d, int layer, const typename C::T* __restrict__ q, typename C::T* __restrict__ out,
    const typename C::T* __restrict__ new_k, const typename C::T* __restrict__ new_v, Cut cut,
    int early) {
  using T = typename C::T;
  constexpr int D = C::D, E = G * D;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_last, s_abort;
  __shared__ UnitSeg s_seg[2][C::WARPS];
  __shared__ __align__(16) StagedQuery<C> s_query;
  const float* s_scale = s_query.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float* state_o = reinterpret_cast<float*>(smem + C::STATE_O);
  float2* state_ml = reinterpret_cast<float2*>(smem + C::STATE_ML);
  float* weight = reinterpret_cast<float*>(smem + C::WEIGHT);
  Ring<C> ring;
  ring.slots = smem + warp * C::STAGES * 2 * C::PAGE;
  ring.full = reinterpret_cast<uint64_t*>(smem + C::BARS) + warp * C::STAGES;
  if (lane == 0) {
    for (int i = 0; i < C::STAGES; ++i) mbar_init(&ring.full[i], 1);
    fence_mbar_init();
  }
  if (tid == 0) s_abort = 0;
  __syncthreads();
  // Before the wait below an early launch reads only what the append wrote (work list, page tables,
  // pages); q, outputs, partial states and counters come after it.
  if (!early) pdl_wait();
  pdl_launch_dependents();
  bool waited = false;

  const int H = d.kv_heads, cta = blockIdx.x;
  UnitSplit us = {};
  UnitSeg seg;  // (the one to come; the warp's copy of the current one is in shared memory)
  int u_begin, u_end, slices = 0, turn = 0;
  if (cut.slices > 0) {
    const int pair = cta / cut.slices, slice = cta % cut.slices;
    seg.seq = pair / H;
    seg.head = pair % H;
    seg.si = d.seq[seg.seq];
    const int nb = seg.si.n_blocks;
    slices = min(cut.slices, nb);
    // (The append failed: what d.seq holds is an older one's.)
    if (d.g->n_units == 0 || slice >= slices) {
      pdl_wait();
      return;
    }
    seg.pair_start = seg.si.unit_base + seg.head * nb;
    seg.pair_end = seg.pair_start + nb;
    seg.u = u_begin = seg.pair_start + (int)((int64_t)slice * nb / slices);
    seg.end = u_end = seg.pair_start + (int)((int64_t)(slice + 1) * nb / slices);
  } else {
    us = unit_split(d, gridDim.x, cut.min_units, DECODE_MAX_PARTS);
    if (cta >= us.n_cta) {
      pdl_wait();
      return;
    }
    u_begin = us.start_of(cta);
    u_end = us.start_of(cta + 1);
    if (u_begin >= u_end) return;
    seg = unit_segment(d, u_begin, u_end);
  }
  auto keep = [&] {
    __syncwarp();
    if (lane == 0) s_seg[turn][warp] = seg;
    __syncwarp();
    return &s_seg[turn][warp];
  };
  const uint32_t slots = smem_u32(ring.slots);
  uint32_t loads = 0;  // steps of this warp, over all segments before
  ring.open(d, layer, keep(), warp);
  for (int k = 0; k < min(C::STAGES, ring.steps()); ++k) ring.issue(d, k, k, lane);
  if (warp == 0) prefetch_query<C>(d, seg.si, seg.head, q, lane);

  for (;;) {
    const UnitSeg& cur = *ring.seg;
    const SeqInfo& si = cur.si;
    if (!waited) {
      pdl_wait();
      waited = true;
    }
    if (warp < G) stage_query<C>(d, si, cur.head, warp, q, lane, s_query);
    __syncthreads();
    Query<C> qr;
    load_query<C>(s_query, lane, qr);
    State<C> st;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int mt = 0; mt < C::MT; ++mt) st.o[mt][0] = st.o[mt][1] = st.o[mt][2] = st.o[mt][3] = 0.f;
    const OpenPages open(si);
    const int n_my = ring.n_my, n_steps = ring.steps();
    int failed_at = -1;
    for (int k = 0; k < n_steps; ++k) {
      const uint32_t n = loads + k, stage = n % C::STAGES;
      if (!__all_sync(FULL, mbar_wait(d, &ring.full[stage], (n / C::STAGES) & 1))) {
        failed_at = k;
        break;
      }
      const uint32_t at = slots + stage * 2 * C::PAGE;
      const int blk = ring.first + 2 * k * C::WARPS;
      if constexpr (FUSED) {
        const int last = si.n_blocks - 1;
        if (blk == last || (blk + C::WARPS == last && 2 * k + 1 < n_my))
          write_new_row<C>(d, layer, si, cur.head, new_k, new_v,
                           ring.slots + (stage * 2 + (blk != last)) * C::PAGE, lane);
      }
      if (2 * k + 1 < n_my) pages_step<C, 2>(at, qr, open, si, blk, st, lane);
      else pages_step<C, 1>(at, qr, open, si, blk, st, lane);
      __syncwarp();
      if (k + C::STAGES < n_steps) ring.issue(d, k + C::STAGES, n + C::STAGES, lane);
    }
    if (failed_at >= 0 && lane == 0) s_abort = 1;

    // This warp's state for the CTA's merge.
    {
      const int g = lane >> 2, t = lane & 3;
      float l = st.l;
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(FULL, l, off);
      if (g == 0) {
        state_ml[warp * G + t] = make_float2(st.m, l);
      }
      float* to = state_o + (warp * G + t) * D + g * (D / 8);
#pragma unroll
      for (int mt = 0; mt < C::MT; mt += 2) {
        float4 x = make_float4(st.o[mt][0], st.o[mt][2], st.o[mt + 1][0], st.o[mt + 1][2]);
        if constexpr (C::SPLIT_P)
          x = make_float4(x.x + st.o[mt][1], x.y + st.o[mt][3], x.z + st.o[mt + 1][1],
                          x.w + st.o[mt + 1][3]);
        *reinterpret_cast<float4*>(to + 2 * mt) = x;
      }
    }
    __syncthreads();
    if (s_abort) {
      // A wait gave up: each warp drains the copies that it still has in flight (bounded), then the
      // whole CTA stops.
      if (failed_at >= 0)
        for (int k = failed_at; k < min(n_steps, failed_at + C::STAGES); ++k)
          mbar_wait(d, &ring.full[(loads + k) % C::STAGES], ((loads + k) / C::STAGES) & 1);
      return;
    }
    loads += n_steps;
    const bool more = cur.end < u_end;
    // The next segment's first pages are on their way while this one is merged.
    if (more) {
      seg = unit_segment(d, cur.end, u_end);
      turn ^= 1;
      ring.open(d, layer, keep(), warp);
      for (int k = 0; k < min(C::STAGES, ring.steps()); ++k) ring.issue(d, k, loads + k, lane);
    }
    const bool whole = cur.whole();
    // Slots of a pair's parts: its slices one after the other, or two of each CTA of the split.
    const int slot = slices ? cta : 2 * cta + (cur.u == u_begin ? 0 : 1);
    T* orow = out + ((size_t)cur.si.q_row0 * d.q_heads + cur.head * G) * D;
    // The warps' states: each thread finds the weights of its elements' head by itself, which is sooner
    // done than handed out.
    // (The thread's number is hidden from the compiler, which would hold what follows from it in registers
    // throughout the pages' loop.)
    int id = tid;
    asm volatile("" : "+r"(id));
    constexpr int EPT = E / C::THREADS;
    const int e0 = id * EPT, h = e0 / D;
    float2 ml[C::WARPS];
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < C::WARPS; ++w) {
      ml[w] = state_ml[w * G + h];
      M = fmaxf(M, ml[w].x);
    }
    Floats<EPT> o = {};
#pragma unroll
    for (int w = 0; w < C::WARPS; ++w) {
      const float f = weight2(ml[w].x, M, s_scale[h]);
      const Floats<EPT> x = Floats<EPT>::load_shared(state_o + w * E + e0);
      L += ml[w].y * f;
#pragma unroll
      for (int k = 0; k < EPT; ++k) o.v[k] += x.v[k] * f;
    }
    if (whole) {
      const float inv = 16.f / L;
#pragma unroll
      for (int k = 0; k < EPT; ++k) o.v[k] *= inv;
      o.store_row(orow + e0);
    } else {
      o.store(d.dec_part_o + (size_t)slot * E + e0);
      if (e0 % D == 0) d.dec_part_ml[(size_t)slot * G + h] = make_float2(M, L);
      // The last CTA of the pair to arrive merges (stream-K: CTAs cf..cl own its units).
      const int cf = slices ? cta - cta % cut.slices : us.owner(cur.pair_start);
      const int parts = slices ? slices : us.owner(cur.pair_end - 1) - cf + 1;
      int* counter = &d.dec_count[cur.seq * H + cur.head];
      __syncthreads();
      if (tid == 0) s_last = arrive_acq_rel(counter, parts);
      __syncthreads();
      if (s_last) {
        const int first_slot = slices ? cf : us.slot_of(cf, cf, cur.pair_start);
        const int next_slot = slices ? cf : 2 * cf, step = slices ? 1 : 2;
        merge_parts<C>(d.dec_part_o, d.dec_part_ml, parts, first_slot, next_slot, step, s_scale, weight,
                       orow, id);
        if (tid == 0) *counter = 0;
      }
    }
    if (!more) break;
    __syncthreads();
  }
}

template <typename T, int D>
using Narrow = Cfg<T, D, 4, 2>;
template <typename T, int D>
using Wide = Cfg<T, D, 8, 2>;
// One CTA to an SM: the block scheduler fills an SM with several CTAs of a small grid while others
// stay empty (96 CTAs of 4 warps: 23.5 us against 14.2), so that these ask for more shared memory.
constexpr int ALONE_SMEM = 120 * 1024;

template <class C>
cudaError_t set_smem() {
  const int most = std::max(C::SMEM, ALONE_SMEM);
  const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(&decode_kv4_kernel<C, false>),
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(reinterpret_cast<const void*>(&decode_kv4_kernel<C, true>),
                              cudaFuncAttributeMaxDynamicSharedMemorySize, most);
}

// CTAs of the stream-K split: as many as run at once; each may write two partial states.
template <class C>
cudaError_t grid_of(int sms, int dec_slots, int* grid) {
  int per_sm = 0;
  cudaError_t e = set_smem<C>();
  if (e == cudaSuccess)
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(
        &per_sm, reinterpret_cast<const void*>(&decode_kv4_kernel<C, false>), C::THREADS, C::SMEM);
  *grid = std::min(per_sm * sms, dec_slots / 2);
  return e;
}

template <class C>
cudaError_t launch(const Dev& d, int layer, const void* q, void* out, const void* new_k,
                   const void* new_v, int grid, bool alone, Cut cut, bool early, cudaStream_t s) {
  using T = typename C::T;
  return launch_ex(new_k != nullptr ? &decode_kv4_kernel<C, true> : &decode_kv4_kernel<C, false>,
                   dim3(grid), dim3(C::THREADS), alone ? std::max(C::SMEM, ALONE_SMEM) : C::SMEM, s,
                   true, d, layer, static_cast<const T*>(q), static_cast<T*>(out),
                   static_cast<const T*>(new_k), static_cast<const T*>(new_v), cut, (int)early);
}

template <typename T, int D>
cudaError_t launch_any(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                       const void* new_k, const void* new_v, int n_pairs, int64_t units, bool early,
                       cudaStream_t s) {
  const DecodeCut c = decode_cut(lim.sms, n_pairs, units, d.esz);
  if (c.slices == 0)
    return launch<Narrow<T, D>>(d, layer, q, out, new_k, new_v, lim.kv4_decode, false, {0, 8}, early, s);
  const int grid = n_pairs * c.slices;
  const bool alone = grid <= lim.sms;
  return c.wide ? launch<Wide<T, D>>(d, layer, q, out, new_k, new_v, grid, alone, {c.slices, 0}, early, s)
                : launch<Narrow<T, D>>(d, layer, q, out, new_k, new_v, grid, alone, {c.slices, 0}, early, s);
}

template <typename T, int D>
cudaError_t limits_of(int dec_slots, Limits* lim) {
  const cudaError_t e = set_smem<Wide<T, D>>();
  return e != cudaSuccess ? e : grid_of<Narrow<T, D>>(lim->sms, dec_slots, &lim->kv4_decode);
}

}  // namespace

cudaError_t kv4_decode_limits(const Dev& d, Limits* lim) {
  return d.esz == 2 ? limits_of<__nv_bfloat16, 128>(d.dec_slots, lim)
                    : limits_of<float, 64>(d.dec_slots, lim);
}

cudaError_t launch_decode_kv4(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                              const void* new_k, const void* new_v, int n_pairs, int64_t units,
                              bool early, cudaStream_t s) {
  return d.esz == 2
             ? launch_any<__nv_bfloat16, 128>(d, lim, layer, q, out, new_k, new_v, n_pairs, units, early, s)
             : launch_any<float, 64>(d, lim, layer, q, out, new_k, new_v, n_pairs, units, early, s);
}

}  // namespace kvc
