// Attention over a cache held in 4 bits (KVC_KV4): single-token decode and chunked prefill.
//
// For each session of the last append, KV head and query row r (token tq, query head gq of the
// group): out = softmax(RoPE(q) . k / sqrt(D)) v over the resident keys up to the row's own
// position, k and v the numbers that the codes stand for.
//
// One page of 16 keys is one step of mma.sync m16n8k16 (binary16 in, binary32 accumulate) with the
// keys as M, eight query rows (a column tile) as N:
//   S^T [16 keys x 8 rows] = K [16 x D] . Q^T [D x 8],   O^T [D x 8 rows] += V^T [D x 16] . P^T.
// The A operands come out of the nibbles by one AND-OR and one fused multiply-add per pair, exact
// (kvc_kv4.h): only q and P are rounded, to 11 bits.  binary32 calls split q and P into two
// binary16 pieces each, so that their products keep about 22 bits.
//   - q rows are divided by a power of two first (largest element in [1, 2)), so that neither
//     large nor small rows leave binary16; the factor returns with the softmax scale.
//   - P is exp2(s - m + 8): 22 octaves below the row's largest weight stay normal numbers.
//   - Masked keys get weight 0, and an invalid slot's V scale is set to 0: what a page held before
//     cannot reach a row.  A V group that stands for NaN reaches exactly the rows that see its key.
//
// A CTA is WP page groups of WC warps.  A group takes every WP-th page of the segment through its
// own ring of bulk copies (18 D bytes: K and V tiles of a head); its warps share each page, warp
// wc taking column tiles [wc * NT, (wc + 1) * NT).  The groups' states merge in shared memory, the
// CTAs' (stream-K split over (session, KV head, page) units) in global memory, by the last CTA of
// a pair to arrive.
#include <algorithm>

#include "kvc_kv4.cuh"

namespace kvc {

namespace {

using namespace kv4;

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int G = 4;               // query heads per KV head
constexpr float LOG2E = 1.4426950408889634f;
constexpr float P_SHIFT = 8.f;     // log2 of the largest weight P

// Shape of one kernel: element type, head dim, column tiles per warp, ring depth.
template <typename T_, int D_, int NT_, int STAGES_>
struct Cfg {
  using T = T_;
  static constexpr int D = D_, NT = NT_, STAGES = STAGES_;
  static constexpr int PIECES = sizeof(T) == 4 ? 2 : 1;  // binary16 pieces of q and of P
  static constexpr int PAGE = 18 * D;                    // bytes of a page of one head, K and V
  static constexpr int WORDS = D / 32;                   // 32-bit words of K codes per lane and row
  static constexpr int MT = D / 16;                      // row tiles of O^T
  static constexpr int STATE = NT * (4 * MT + 4);        // floats of a lane's (o, m, l)
  static constexpr int MOST_THREADS = NT == 1 ? 128 : 384;
  // Bytes of one column tile's query fragments: WORDS uint4 per lane and piece.
  static constexpr int Q_TILE = PIECES * WORDS * 32 * 16;
};

// Shared memory of a CTA, in bytes from the start.
template <class C>
struct Layout {
  int ring, q, scale, merge, weight, bars, total;
  __host__ __device__ Layout(int wc, int wp, int parts) {
    const int tiles = wc * C::NT;
    ring = 0;
    q = ring + wp * C::STAGES * C::PAGE;
    scale = q + tiles * C::Q_TILE;                       // [tiles * 8] softmax scales of the columns
    merge = scale + tiles * 8 * 4;                       // [wp / 2 groups][wc][32 lanes][STATE]
    weight = merge + (wp / 2) * wc * 32 * C::STATE * 4;  // [parts][tiles * 8]
    bars = weight + parts * tiles * 8 * 4;               // [wp][STAGES] full, then empty
    bars = (bars + 7) & ~7;
    total = bars + wp * C::STAGES * 2 * 8;
  }
};

// Weight of a state with running maximum x against the maximum m of both, 0 where there is no key.
// Maxima are of the raw products S, c is the row's softmax scale: S - max is rounded before c comes
// in, so that logits of any size leave exponents that are exact near 0 and never positive.
__device__ inline float weight2(float x, float m, float c) {
  return m == -INFINITY ? 0.f : exp2f((x - m) * c);
}

// Query rows of a segment as B operands, in shared memory: item (column, c) rotates dims
// [8c, 8c + 8) and their partners; the KC threads of a column find its largest element.
// Columns past the chunk's rows are zero.
template <class C>
__device__ void build_queries(const Dev& d, const SeqInfo& si, int head, int n_cols,
                              const typename C::T* q, float scale, uint8_t* frag, float* col_scale,
                              int tid, int n_threads) {
  using T = typename C::T;
  constexpr int D = C::D, KC = D / 16;
  const int rows = si.t * G;
  for (int i0 = 0; i0 < n_cols * KC; i0 += n_threads) {
    const int i = i0 + tid, col = i / KC, c = i % KC;
    const bool real = i < n_cols * KC && col < rows;
    float x1[8] = {}, x2[8] = {}, ya[8], yb[8];
    if (real) {
      const T* row = q + ((size_t)(si.q_row0 + col / G) * d.q_heads + head * G + col % G) * D + c * 8;
      Eight<T> a, b;
      a.load(row);
      b.load(row + D / 2);
      a.get(x1);
      b.get(x2);
    }
    const int pos = real ? si.pos_first + col / G : 0;
    const float4* t4 = reinterpret_cast<const float4*>(d.rope + (size_t)pos * (D / 2) + c * 8);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float4 cs = t4[e / 2];
      turn_pair(x1[e], x2[e], make_float2(cs.x, cs.y), ya[e], yb[e]);
      turn_pair(x1[e + 1], x2[e + 1], make_float2(cs.z, cs.w), ya[e + 1], yb[e + 1]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, max(abs_bits(ya[e]), abs_bits(yb[e])));
#pragma unroll
    for (int o = 1; o < KC; o <<= 1) most = max(most, __shfl_xor_sync(FULL, most, o));
    if (i >= n_cols * KC) continue;
    // 2^e with the row's largest element in [2^e, 2^(e + 1)); infinities and NaN pass through.
    int e = (int)(most >> 23) - 127;
    e = e > 126 ? (e == 128 ? 0 : 126) : max(e, -126);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    if (c == 0) col_scale[col] = scale * __uint_as_float((uint32_t)(127 + e) << 23);
    const int tile = col / 8, n = col % 8;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int dim = half * (D / 2) + 8 * c;                // first of eight dims
      const int t = dim % GROUP / 8, w = dim / GROUP;        // lane (n, t), word w
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = (half ? yb[j] : ya[j]) * inv;
#pragma unroll
      for (int piece = 0; piece < C::PIECES; ++piece) {
        uint32_t u[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const __half2 v = __floats2half2_rn(y[p], y[p + 4]);
          u[p] = h2_bits(v);
          y[p] -= __low2float(v);
          y[p + 4] -= __high2float(v);
        }
        *reinterpret_cast<uint4*>(frag + (size_t)tile * C::Q_TILE +
                                  ((piece * C::WORDS + w) * 32 + n * 4 + t) * 16) =
            make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
  }
}

// A warp's running state: rows (columns of the MMAs) 8 nt + 2t, 2t + 1; dims D/8 of them from
// g * D / 8 (o[nt][mt][0..3]: dims 2 mt, 2 mt, 2 mt + 1, 2 mt + 1 of rows 2t, 2t + 1, 2t, 2t + 1).
template <class C>
struct State {
  float o[C::NT][C::MT][4];
  float m[C::NT][2], l[C::NT][2];  // l: this lane's keys only
  __device__ void clear() {
#pragma unroll
    for (int nt = 0; nt < C::NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
    }
  }
  // To and from shared memory, one lane's floats 32 apart.
  template <typename F>
  __device__ void each(F f) {
    int i = 0;
#pragma unroll
    for (int nt = 0; nt < C::NT; ++nt) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        f(i++, m[nt][j]);
        f(i++, l[nt][j]);
      }
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) f(i++, o[nt][mt][j]);
    }
  }
  // Add the state that another group's warp left at p (+ lane).  col_scale: of this lane's first column.
  __device__ void add(const float* p, const float* col_scale) {
#pragma unroll
    for (int nt = 0; nt < C::NT; ++nt) {
      const float* b = p + nt * (4 * C::MT + 4) * 32;
      const float2 c = *reinterpret_cast<const float2*>(col_scale + nt * 8);
      float mine[2], theirs[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float mo = b[2 * j * 32], lo = b[(2 * j + 1) * 32];
        const float mn = fmaxf(m[nt][j], mo);
        mine[j] = weight2(m[nt][j], mn, j ? c.y : c.x);
        theirs[j] = weight2(mo, mn, j ? c.y : c.x);
        l[nt][j] = l[nt][j] * mine[j] + lo * theirs[j];
        m[nt][j] = mn;
      }
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[nt][mt][j] = o[nt][mt][j] * mine[j & 1] + b[(4 + 4 * mt + j) * 32] * theirs[j & 1];
    }
  }
};

// One page: scores, running softmax, P V.  [lo, hi): its valid slots; base: retained index of
// slot 0; last0 + tq: retained index of token tq's own row, the last that it sees.
template <class C>
__device__ inline void page_step(const uint8_t* page, const uint8_t* frag, const float* col_scale,
                                 const BlockRange& br, int last0, int tile0, State<C>& st,
                                 int lane) {
  constexpr int D = C::D, NT = C::NT;
  const int g = lane >> 2, t = lane & 3;
  const uint8_t* kt = page;
  const uint8_t* vt = page + 9 * D;
  // Every key of the page is valid and seen by every row of the chunk.
  const bool open = br.lo == 0 && br.hi == PS && br.base + PS - 1 <= last0;

  float s[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
  {
    uint32_t wa[C::WORDS], wb[C::WORDS];  // rows g and g + 8
    if constexpr (D == 128) {
      const uint4 a = *reinterpret_cast<const uint4*>(kt + g * 64 + t * 16);
      const uint4 b = *reinterpret_cast<const uint4*>(kt + (g + 8) * 64 + t * 16);
      wa[0] = a.x; wa[1] = a.y; wa[2] = a.z; wa[3] = a.w;
      wb[0] = b.x; wb[1] = b.y; wb[2] = b.z; wb[3] = b.w;
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(kt + g * 32 + t * 8);
      const uint2 b = *reinterpret_cast<const uint2*>(kt + (g + 8) * 32 + t * 8);
      wa[0] = a.x; wa[1] = a.y;
      wb[0] = b.x; wb[1] = b.y;
    }
    const __half2 m72 = __float2half2_rn(-72.f);
#pragma unroll
    for (int w = 0; w < C::WORDS; ++w) {
      const __half2 ma = __half2half2(*reinterpret_cast<const __half*>(kt + k_scale(D, g, w)));
      const __half2 mb = __half2half2(*reinterpret_cast<const __half*>(kt + k_scale(D, g + 8, w)));
      const __half2 na = __hmul2(ma, m72), nb = __hmul2(mb, m72);
      uint32_t pa[4], pb[4];
      pairs_of(wa[w], ma, na, pa);
      pairs_of(wb[w], mb, nb, pb);
      const uint32_t a[8] = {pa[0], pb[0], pa[1], pb[1], pa[2], pb[2], pa[3], pb[3]};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint8_t* qf = frag + (size_t)(tile0 + nt) * C::Q_TILE + (w * 32 + lane) * 16;
        const uint4 b = *reinterpret_cast<const uint4*>(qf);
        if constexpr (C::PIECES == 1) {
          mma_f16(s[nt], a[0], a[1], a[2], a[3], b.x, b.y);
          mma_f16(s[nt], a[4], a[5], a[6], a[7], b.z, b.w);
        } else {
          // The sum of each 16 dims by itself, then added rounded: the tensor cores cut off what
          // they add to an accumulator.
          const uint4 b2 = *reinterpret_cast<const uint4*>(qf + C::WORDS * 32 * 16);
          float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
          mma_f16(x, a[0], a[1], a[2], a[3], b2.x, b2.y);
          mma_f16(y, a[4], a[5], a[6], a[7], b2.z, b2.w);
          mma_f16(x, a[0], a[1], a[2], a[3], b.x, b.y);
          mma_f16(y, a[4], a[5], a[6], a[7], b.z, b.w);
#pragma unroll
          for (int j = 0; j < 4; ++j) s[nt][j] += x[j] + y[j];
        }
      }
    }
  }

  uint32_t pb[NT][C::PIECES][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int col = (tile0 + nt) * 8 + 2 * t;
    const float2 cs = *reinterpret_cast<const float2*>(col_scale + col);
    if (!open) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int slot = g + 8 * (j >> 1), last = last0 + (col + (j & 1)) / G;
        if (slot < br.lo || slot >= br.hi || br.base + slot > last) s[nt][j] = -INFINITY;
      }
    }
    float p[4];
    bool moved = false;
    float alpha[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float c = j ? cs.y : cs.x;
      float mx = fmaxf(s[nt][j], s[nt][j + 2]);
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, off));
      const float mn = fmaxf(st.m[nt][j], mx);
      alpha[j] = weight2(st.m[nt][j], mn, c);
      const float ref = mn == -INFINITY ? 0.f : mn;
      p[j] = exp2f(fmaf(s[nt][j] - ref, c, P_SHIFT));
      p[j + 2] = exp2f(fmaf(s[nt][j + 2] - ref, c, P_SHIFT));
      st.l[nt][j] = st.l[nt][j] * alpha[j] + (p[j] + p[j + 2]);
      st.m[nt][j] = mn;
      moved = moved || alpha[j] != 1.f;
    }
    if (__any_sync(FULL, moved)) {
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) st.o[nt][mt][j] *= alpha[j & 1];
    }
#pragma unroll
    for (int piece = 0; piece < C::PIECES; ++piece)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const __half2 v = __floats2half2_rn(p[2 * j], p[2 * j + 1]);
        pb[nt][piece][j] = transpose8(h2_bits(v));
        p[2 * j] -= __low2float(v);
        p[2 * j + 1] -= __high2float(v);
      }
  }

  // V^T: lane (g, t) takes piece g of rows 2t, 2t + 1 (lo) and 2t + 8, 2t + 9 (hi).
  constexpr int VW = D / 64;  // words of a piece of one row
  uint32_t v[2][2][VW];       // [lo, hi][row of the pair][word]
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* at = vt + i * (D * 4) + lane * (D / 8);
    if constexpr (D == 128) {
      const uint4 w = *reinterpret_cast<const uint4*>(at);
      v[i][0][0] = w.x; v[i][0][1] = w.y;
      v[i][1][0] = w.z; v[i][1][1] = w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(at);
      v[i][0][0] = w.x;
      v[i][1][0] = w.y;
    }
  }
  const int group = g * (D / 8) / GROUP;
  uint32_t sc[2];
  sc[0] = *reinterpret_cast<const uint32_t*>(vt + v_scale(D, 2 * t, group));
  sc[1] = *reinterpret_cast<const uint32_t*>(vt + v_scale(D, 2 * t + 8, group));
  if (!open) {
    // Invalid slots stand for 0; NaN groups for 0 here and for NaN in the rows that see them.
    uint32_t nan = 0;  // bit 2 i + r: row 2t + 8 i + r of this lane's group
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int slot = 2 * t + 8 * i + r;
        const bool valid = slot >= br.lo && slot < br.hi;
        const bool is_nan = (sc[i] >> (16 * r) & 0x7FFFu) > 0x7C00u;
        if (!valid || is_nan) sc[i] &= r ? 0x0000FFFFu : 0xFFFF0000u;
        if (valid && is_nan) nan |= 1u << (2 * i + r);
      }
    if (__any_sync(FULL, nan != 0)) {
      for (int slot = 0; slot < PS; ++slot) {
        // The lane of this g that holds the slot's scale.
        const uint32_t held = __shfl_sync(FULL, nan, (lane & ~3) | ((slot & 7) >> 1));
        if (!(held >> (2 * (slot >> 3) + (slot & 1)) & 1)) continue;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            if (br.base + slot <= last0 + ((tile0 + nt) * 8 + 2 * t + j) / G)
#pragma unroll
              for (int mt = 0; mt < C::MT; ++mt)
                st.o[nt][mt][j] = st.o[nt][mt][j + 2] = __uint_as_float(0x7FC00000u);
      }
    }
  }
  const __half2 m72 = __float2half2_rn(-72.f);
  const __half2 ml = bits_h2(sc[0]), mh = bits_h2(sc[1]);
  const __half2 nl = __hmul2(ml, m72), nh = __hmul2(mh, m72);
#pragma unroll
  for (int w = 0; w < VW; ++w)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      // Dims 8 w + 4 half + 0..3 of the piece: nibble p of both halves of a word, the pair's rows.
      const uint32_t sel = half ? 0x7632u : 0x5410u;
      const uint32_t lo = __byte_perm(v[0][0][w], v[0][1][w], sel);
      const uint32_t hi = __byte_perm(v[1][0][w], v[1][1][w], sel);
      uint32_t pl[4], ph[4];
      pairs_of(lo, ml, nl, pl);
      pairs_of(hi, mh, nh, ph);
      const uint32_t a[8] = {pl[0], pl[1], ph[0], ph[1], pl[2], pl[3], ph[2], ph[3]};
      const int mt = 4 * w + 2 * half;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if constexpr (C::PIECES == 1) {
          mma_f16(st.o[nt][mt], a[0], a[1], a[2], a[3], pb[nt][0][0], pb[nt][0][1]);
          mma_f16(st.o[nt][mt + 1], a[4], a[5], a[6], a[7], pb[nt][0][0], pb[nt][0][1]);
        } else {
          // A page's sums by themselves, then added rounded: the tensor cores cut off what they
          // add, and the losses of many pages would all go the same way.
          float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int piece = C::PIECES - 1; piece >= 0; --piece) {
            mma_f16(x, a[0], a[1], a[2], a[3], pb[nt][piece][0], pb[nt][piece][1]);
            mma_f16(y, a[4], a[5], a[6], a[7], pb[nt][piece][0], pb[nt][piece][1]);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            st.o[nt][mt][j] += x[j];
            st.o[nt][mt + 1][j] += y[j];
          }
        }
      }
    }
}

// The pages of one group and segment, through the group's ring.
template <class C>
struct Ring {
  uint8_t* slots;
  uint64_t* full;
  uint64_t* empty;
  const int32_t* hrow;
  const int32_t* lrow;
  SeqInfo si;
  int head, blk_begin, n_my, wp;
  int win, pid;

  // Copy the group's k-th page of the segment (its `n`-th of the launch) in; the whole warp.
  __device__ bool issue(const Dev& d, int layer, int k, uint32_t n, int wc_count, int group,
                        int lane) {
    if (k >= win + 32) {
      win = k & ~31;
      const int j = win + lane;
      pid = j < n_my ? block_page(si, hrow, lrow, blk_begin + group + j * wp) : 0;
    }
    const int page = __shfl_sync(FULL, pid, k - win);
    const int st = n % C::STAGES;
    bool ok = true;
    if (wc_count > 1 && n >= C::STAGES)
      ok = __all_sync(FULL, mbar_wait(d, &empty[st], (n / C::STAGES - 1) & 1));
    if (!ok) return false;
    if (lane == 0) {
      fence_proxy_async_smem();
      mbar_arrive_expect_tx(&full[st], C::PAGE);
      const uint8_t* src = d.pool + tile_at(C::D, d.layers, d.kv_heads, page, layer, head, 0);
      bulk_g2s(slots + st * C::PAGE, src, C::PAGE, &full[st]);
    }
    return true;
  }
};

// Rows of a pair from the parts that cover it: part i of `parts` is in slot part(i), [col][D] and
// (m, l) per column.  Called by every thread of the last CTA to arrive.
template <class C, typename PartFn>
__device__ void merge_parts(const float* part_o, const float2* part_ml, int cols_slot, int parts,
                            PartFn part, int rows, const float* col_scale, float* s_w,
                            typename C::T* out, size_t out_row,
                            int q_heads, int tid, int n_threads) {
  using T = typename C::T;
  constexpr int D = C::D;
  // Weights of the parts, divided by the total: one thread per row.
  for (int r = tid; r < rows; r += n_threads) {
    float M = -INFINITY;
    for (int i = 0; i < parts; ++i) M = fmaxf(M, __ldcg(&part_ml[(size_t)part(i) * cols_slot + r]).x);
    float L = 0.f;
    for (int i = 0; i < parts; ++i) {
      const float2 ml = __ldcg(&part_ml[(size_t)part(i) * cols_slot + r]);
      const float w = weight2(ml.x, M, col_scale[r]);
      s_w[i * rows + r] = w;
      L += ml.y * w;
    }
    const float inv = 1.f / L;
    for (int i = 0; i < parts; ++i) s_w[i * rows + r] *= inv;
  }
  __syncthreads();
  for (int e = tid; e < rows * (D / 4); e += n_threads) {
    const int r = e / (D / 4), dd = e % (D / 4) * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < parts; ++i) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(
          part_o + ((size_t)part(i) * cols_slot + r) * D + dd));
      const float w = s_w[i * rows + r];
      acc.x += x.x * w;
      acc.y += x.y * w;
      acc.z += x.z * w;
      acc.w += x.w * w;
    }
    T* to = out + out_row + ((size_t)(r / G) * q_heads + r % G) * D + dd;
    to[0] = from_float<T>(acc.x * 16.f);
    to[1] = from_float<T>(acc.y * 16.f);
    to[2] = from_float<T>(acc.z * 16.f);
    to[3] = from_float<T>(acc.w * 16.f);
  }
}

template <class C>
__global__ void __launch_bounds__(C::MOST_THREADS, 1) attn_kv4_kernel(
    Dev d, int layer, const typename C::T* __restrict__ q, typename C::T* __restrict__ out,
    float qk_scale, int wc_count, int wp_count, int min_units, int max_parts, float* part_o,
    float2* part_ml, int* count, int early) {
  using T = typename C::T;
  constexpr int D = C::D;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_last, s_abort;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_threads = blockDim.x;
  const int group = warp / wc_count, wc = warp % wc_count;
  const Layout<C> lay(wc_count, wp_count, max_parts);
  const int tiles = wc_count * C::NT, cols = tiles * 8;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + lay.bars);
  float* col_scale = reinterpret_cast<float*>(smem + lay.scale);
  float* merge = reinterpret_cast<float*>(smem + lay.merge);
  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < wp_count * C::STAGES; ++i) {
      mbar_init(&bars[i], 1);
      mbar_init(&bars[wp_count * C::STAGES + i], wc_count);
    }
    fence_mbar_init();
  }
  __syncthreads();
  // Before the wait below an early launch reads only what the append wrote (work list, page
  // tables, pages); q, outputs, partial states and counters come after it.
  if (!early) pdl_wait();
  pdl_launch_dependents();
  bool waited = false;

  const int H = d.kv_heads;
  const UnitSplit us = unit_split(d, gridDim.x, min_units, max_parts);
  if ((int)blockIdx.x >= us.n_cta) return;
  const int cta = blockIdx.x;
  const int u_begin = us.start_of(cta), u_end = us.start_of(cta + 1);
  Ring<C> ring;
  ring.slots = smem + lay.ring + group * C::STAGES * C::PAGE;
  ring.full = bars + group * C::STAGES;
  ring.empty = bars + (wp_count + group) * C::STAGES;
  ring.wp = wp_count;
  uint32_t loads = 0;  // of the group, over all segments
  State<C> st;

  for (int u = u_begin; u < u_end;) {
    const UnitSeg seg = unit_segment(d, u, u_end);
    const SeqInfo& si = seg.si;
    const int nblk = seg.end - u;
    ring.si = si;
    ring.head = seg.head;
    ring.blk_begin = u - seg.pair_start;
    ring.hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
    ring.lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
    ring.n_my = nblk > group ? (nblk - group + wp_count - 1) / wp_count : 0;
    ring.win = -32;
    ring.pid = 0;
    int issued = 0;  // pages of this segment copied or in flight (loader warp)
    bool ok = true;
    if (wc == 0)
      for (; ok && issued < min(C::STAGES, ring.n_my); ++issued)
        ok = ring.issue(d, layer, issued, loads + issued, wc_count, group, lane);
    if (!waited) {
      pdl_wait();
      waited = true;
    }
    build_queries<C>(d, si, seg.head, cols, q, qk_scale, smem + lay.q, col_scale, tid, n_threads);
    __syncthreads();
    st.clear();
    const int last0 = si.n_hist + si.n_live - si.t;
    int done = 0;
    for (; ok && done < ring.n_my; ++done) {
      const uint32_t n = loads + done;
      const int stage = n % C::STAGES;
      ok = __all_sync(FULL, mbar_wait(d, &ring.full[stage], (n / C::STAGES) & 1));
      if (!ok) break;
      const BlockRange br = block_range(si, ring.blk_begin + group + done * wp_count);
      page_step<C>(ring.slots + stage * C::PAGE, smem + lay.q, col_scale, br, last0, wc * C::NT, st,
                   lane);
      __syncwarp();
      if (wc_count > 1 && lane == 0) mbar_arrive(&ring.empty[stage]);
      if (wc == 0 && issued < ring.n_my) {
        ok = ring.issue(d, layer, issued, loads + issued, wc_count, group, lane);
        if (ok) ++issued;
      }
    }
    if (!ok && lane == 0) s_abort = 1;
    __syncthreads();
    if (s_abort) {
      // A wait gave up: the loader drains the copies that it still has in flight (bounded), then
      // the whole CTA stops.
      if (wc == 0)
        for (int k = done; k < issued; ++k)
          mbar_wait(d, &ring.full[(loads + k) % C::STAGES], ((loads + k) / C::STAGES) & 1);
      return;
    }
    loads += ring.n_my;

    // Merge the groups, halving their number; complete the sums over the lanes of a row.
    for (int half = wp_count / 2; half > 0; half /= 2) {
      float* at = merge + ((size_t)(group % half) * wc_count + wc) * 32 * C::STATE + lane;
      if (group >= half && group < 2 * half) st.each([&](int i, float& x) { at[i * 32] = x; });
      __syncthreads();
      if (group < half) st.add(at, col_scale + wc * C::NT * 8 + 2 * (lane & 3));
      __syncthreads();
    }
    const bool whole = seg.whole();
    const int slot = 2 * cta + (u == u_begin ? 0 : 1);
    const int g = lane >> 2, t = lane & 3, rows = si.t * G;
    const size_t out_row = ((size_t)si.q_row0 * d.q_heads + seg.head * G) * D;
    if (group == 0) {
#pragma unroll
      for (int nt = 0; nt < C::NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float l = st.l[nt][j];
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(FULL, l, off);
          const int col = (wc * C::NT + nt) * 8 + 2 * t + j;
          if (col >= rows) continue;
          constexpr int PIECE = D / 8;
          if (whole) {
            const float inv = 16.f / l;
            T* to = out + out_row + ((size_t)(col / G) * d.q_heads + col % G) * D + g * PIECE;
#pragma unroll
            for (int i = 0; i < PIECE; i += 8) {
              float f[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) f[e] = st.o[nt][(i + e) / 2][j + 2 * (e & 1)] * inv;
              Eight<T>::store(to + i, f);
            }
          } else {
            float* to = part_o + ((size_t)slot * cols + col) * D + g * PIECE;
#pragma unroll
            for (int i = 0; i < PIECE; i += 4)
              *reinterpret_cast<float4*>(to + i) =
                  make_float4(st.o[nt][i / 2][j], st.o[nt][i / 2][j + 2],
                              st.o[nt][i / 2 + 1][j], st.o[nt][i / 2 + 1][j + 2]);
            if (g == 0) part_ml[(size_t)slot * cols + col] = make_float2(st.m[nt][j], l);
          }
        }
    }
    if (!whole) {
      const int cf = us.owner(seg.pair_start), cl = us.owner(seg.pair_end - 1);
      const int parts = cl - cf + 1;
      int* counter = &count[seg.seq * H + seg.head];
      __syncthreads();
      if (tid == 0) s_last = arrive_acq_rel(counter, parts);
      __syncthreads();
      if (s_last) {
        const int first_slot = us.slot_of(cf, cf, seg.pair_start);
        merge_parts<C>(part_o, part_ml, cols, parts,
                       [&](int i) { return i ? 2 * (cf + i) : first_slot; }, rows, col_scale,
                       reinterpret_cast<float*>(smem + lay.weight), out, out_row, d.q_heads, tid,
                       n_threads);
        if (tid == 0) *counter = 0;
      }
    }
    __syncthreads();
    u = seg.end;
  }
}

// Chunks have ceil(rows / 24) warps per page group.
constexpr int PF_NT = 3, PF_STAGES = 4, PF_PARTS = 32;
template <typename T, int D>
using PfCfg = Cfg<T, D, PF_NT, PF_STAGES>;

int pf_warps(int max_t) { return (max_t * G + 8 * PF_NT - 1) / (8 * PF_NT); }
int pf_groups(int wc) { return wc <= 3 ? 4 : 2; }

template <class C>
cudaError_t grid_of(int wc, int wp, int parts, int sms, int* grid) {
  const Layout<C> lay(wc, wp, parts);
  int per_sm = 0;
  const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(
      &per_sm, reinterpret_cast<const void*>(&attn_kv4_kernel<C>), 32 * wc * wp, lay.total);
  *grid = per_sm * sms;
  return e;
}

template <typename T, int D>
cudaError_t limits_of(Limits* lim) {
  constexpr int MOST = 226 * 1024;
  cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(&attn_kv4_kernel<PfCfg<T, D>>),
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, MOST);
  for (int wc = 1; wc <= KV4_PF_WARPS && e == cudaSuccess; ++wc)
    e = grid_of<PfCfg<T, D>>(wc, pf_groups(wc), PF_PARTS, lim->sms, &lim->kv4_prefill[wc]);
  return e;
}

template <typename T, int D>
cudaError_t launch_any(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                       int max_t, bool early, cudaStream_t s) {
  using C = PfCfg<T, D>;
  const int wc = pf_warps(max_t), wp = pf_groups(wc);
  const Layout<C> lay(wc, wp, PF_PARTS);
  // Each CTA of the split may leave two partial states.
  const int cols = wc * C::NT * 8;
  const int64_t slots = (int64_t)d.pf_slots * PF_MAX_TOKENS * G * 128 / (cols * D);
  const int grid = (int)std::min<int64_t>(
      lim.kv4_prefill[wc], std::min<int64_t>(slots, (int64_t)d.pf_slots * PF_MAX_TOKENS * G / cols) / 2);
  const float scale = 16.f * LOG2E / sqrtf((float)D);
  return launch_ex(&attn_kv4_kernel<C>, dim3(grid), dim3(32 * wc * wp), lay.total, s, true, d, layer,
                   static_cast<const T*>(q), static_cast<T*>(out), scale, wc, wp, wp, PF_PARTS,
                   d.pf_part_o, d.pf_part_ml, d.pf_count, (int)early);
}

}  // namespace

cudaError_t kv4_prefill_limits(const Dev& d, Limits* lim) {
  return d.esz == 2 ? kv4_prefill_tc_limits(lim) : limits_of<float, 64>(lim);
}

cudaError_t launch_attn_kv4(const Dev& d, const Limits& lim, LaunchOrder* order, int layer,
                            const void* new_k, const void* new_v, const void* q, void* out,
                            int n_seq, int total, int max_t, int64_t units, cudaStream_t s) {
  const bool fused = new_k != nullptr;
  if (max_t == 1) {
    const cudaError_t e = launch_decode_kv4(d, lim, layer, q, out, new_k, new_v, n_seq * d.kv_heads,
                                            units, order->early(layer, fused), s);
    if (e == cudaSuccess) order->launched(layer, fused);
    return e;
  }
  if (fused) {
    const cudaError_t e = launch_append_layers_kv4(d, total, layer, 1, new_k, new_v, false,
                                                   order->planned(), lim.sms, s);
    if (e != cudaSuccess) return e;
    order->layer_write(layer);
  }
  const bool early = order->early(layer, false);
  const cudaError_t e =
      d.esz == 2 ? launch_prefill_kv4_tc(d, lim, layer, q, out, n_seq * d.kv_heads, units, early, s)
                 : launch_any<float, 64>(d, lim, layer, q, out, max_t, early, s);
  if (e == cudaSuccess) order->launched(layer, false);
  return e;
}

}  // namespace kvc
