// Chunked-prefill attention over a cache held in 4 bits (KVC_KV4), binary32 calls.
//
// For each session of the last append, KV head and query row r (token tq, query head gq of the
// group): out = softmax(RoPE(q) . k / sqrt(D)) v over the resident keys up to the row's own
// position, k and v the numbers that the codes stand for.
//
// One page of 16 keys is one step of mma.sync m16n8k16 (binary16 in, binary32 accumulate) with the
// keys as M, eight query rows (a column tile) as N:
//   S^T [16 keys x 8 rows] = K [16 x D] . Q^T [D x 8],   O^T [D x 8 rows] += V^T [D x 16] . P^T.
// The A operands come out of the nibbles exact (kvc_kv4.h): only q and P are rounded.  They are split
// into two binary16 pieces each, so that their products keep about 22 bits, and no sum of the tensor
// cores is longer than a page: 11-bit operands and long sums (the bfloat16 kernels') would leave
// errors of 2^-11 where callers of a float cache expect those of float.
//   - q rows are divided by a power of two first (largest element in [1, 2)), so that neither
//     large nor small rows leave binary16; the factor returns with the softmax scale.
//   - P is exp2(s - m + 8): 22 octaves below the row's largest weight stay normal numbers.
//   - Masked keys get weight 0, and an invalid slot's V scale is set to 0: what a page held before
//     cannot reach a row.  A V group that stands for NaN reaches exactly the rows that see its key.
//
// A CTA is WP page groups of WC warps.  A group takes every WP-th page of the CTA's through its
// own ring of bulk copies (18 D bytes: K and V tiles of a head); its warps share each page, warp
// wc taking column tiles [wc * NT, (wc + 1) * NT).  The groups' states merge in shared memory.  Each
// (session, KV head) pair's pages are cut into slices, one CTA each, whose states merge in global
// memory, by the last CTA of a pair to arrive.  What bounds a small call is the chain of phases of a
// CTA (queries, pages, merges), not its 0.25 instructions a cycle: one slice a CTA keeps that short
// where an even cut of all units would leave most CTAs two pairs.  Three sessions of 1,100 positions (8
// heads, up to 23 tokens): 13 us a layer, 20 with that cut; the bytes are 0.3 us.
#include <algorithm>

#include "kvc_kv4.cuh"

namespace kvc {

namespace {

using namespace kv4;

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int G = 4;               // query heads per KV head
constexpr float LOG2E = 1.4426950408889634f;
constexpr float P_SHIFT = 8.f;     // log2 of the largest weight P

constexpr int D = 64;              // head dim of float caches
constexpr int NT = 3;              // column tiles (of 8 query rows) of a warp
constexpr int STAGES = 4;          // pages in a ring
constexpr int PIECES = 2;          // binary16 pieces of q and of P
constexpr int PAGE = 18 * D;       // bytes of a page of one head, K and V
constexpr int WORDS = D / 32;      // 32-bit words of K codes per lane and row
constexpr int MT = D / 16;         // row tiles of O^T
constexpr int STATE = NT * (4 * MT + 4);          // floats of a lane's (o, m, l)
constexpr int Q_TILE = PIECES * WORDS * 32 * 16;  // bytes of a column tile's query fragments
constexpr int PARTS = 32;          // CTAs that share a pair, at most (a warp merges a row's)

// Shared memory of a CTA, in bytes from the start.
struct Layout {
  int ring, q, scale, merge, weight, bars, total;
  __host__ __device__ Layout(int wc, int wp) {
    const int tiles = wc * NT;
    ring = 0;
    q = ring + wp * STAGES * PAGE;
    scale = q + tiles * Q_TILE;                       // [tiles * 8] softmax scales of the columns
    merge = scale + tiles * 8 * 4;                    // [wp / 2 groups][wc][32 lanes][STATE]
    weight = merge + (wp / 2) * wc * 32 * STATE * 4;  // [PARTS][tiles * 8]
    bars = weight + PARTS * tiles * 8 * 4;            // [wp][STAGES] full, then empty
    bars = (bars + 7) & ~7;
    total = bars + wp * STAGES * 2 * 8;
  }
};

// Weight of a state with running maximum x against the maximum m of both, 0 where there is no key.
// Maxima are of the raw products S, c is the row's softmax scale: S - max is rounded before c comes
// in, so that logits of any size leave exponents that are exact near 0 and never positive.
__device__ inline float weight2(float x, float m, float c) {
  return m == -INFINITY ? 0.f : exp2f((x - m) * c);
}

// Query rows of a pair as B operands, in shared memory: item (column, c) rotates dims
// [8c, 8c + 8) and their partners; the KC threads of a column find its largest element.
// Columns past the chunk's rows are zero.
__device__ void build_queries(const Dev& d, const SeqInfo& si, int head, int n_cols,
                              const float* q, float scale, uint8_t* frag, float* col_scale,
                              int tid, int n_threads) {
  constexpr int KC = D / 16;
  const int rows = si.t * G;
  for (int i0 = 0; i0 < n_cols * KC; i0 += n_threads) {
    const int i = i0 + tid, col = i / KC, c = i % KC;
    const bool real = i < n_cols * KC && col < rows;
    float x1[8] = {}, x2[8] = {}, ya[8], yb[8];
    if (real) {
      const float* row = q + ((size_t)(si.q_row0 + col / G) * d.q_heads + head * G + col % G) * D + c * 8;
      Eight<float> a, b;
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
      for (int piece = 0; piece < PIECES; ++piece) {
        uint32_t u[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const __half2 v = __floats2half2_rn(y[p], y[p + 4]);
          u[p] = h2_bits(v);
          y[p] -= __low2float(v);
          y[p + 4] -= __high2float(v);
        }
        *reinterpret_cast<uint4*>(frag + (size_t)tile * Q_TILE +
                                  ((piece * WORDS + w) * 32 + n * 4 + t) * 16) =
            make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
  }
}

// A warp's running state: rows (columns of the MMAs) 8 nt + 2t, 2t + 1; dims D/8 of them from
// g * D / 8 (o[nt][mt][0..3]: dims 2 mt, 2 mt, 2 mt + 1, 2 mt + 1 of rows 2t, 2t + 1, 2t, 2t + 1).
struct State {
  float o[NT][MT][4];
  float m[NT][2], l[NT][2];  // l: this lane's keys only
  __device__ void clear() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
    }
  }
  // To and from shared memory, one lane's floats 32 apart.
  template <typename F>
  __device__ void each(F f) {
    int i = 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        f(i++, m[nt][j]);
        f(i++, l[nt][j]);
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) f(i++, o[nt][mt][j]);
    }
  }
  // Add the state that another group's warp left at p (+ lane).  col_scale: of this lane's first column.
  __device__ void add(const float* p, const float* col_scale) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float* b = p + nt * (4 * MT + 4) * 32;
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
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[nt][mt][j] = o[nt][mt][j] * mine[j & 1] + b[(4 + 4 * mt + j) * 32] * theirs[j & 1];
    }
  }
};

// One page: scores, running softmax, P V.  [lo, hi): its valid slots; base: retained index of
// slot 0; last0 + tq: retained index of token tq's own row, the last that it sees.
__device__ inline void page_step(const uint8_t* page, const uint8_t* frag, const float* col_scale,
                                 const BlockRange& br, int last0, int tile0, State& st,
                                 int lane) {
  const int g = lane >> 2, t = lane & 3;
  const uint8_t* kt = page;
  const uint8_t* vt = page + 9 * D;
  // Every key of the page is valid and seen by every row of the chunk.
  const bool open = br.lo == 0 && br.hi == PS && br.base + PS - 1 <= last0;

  float s[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
  {
    uint32_t wa[WORDS], wb[WORDS];  // rows g and g + 8
    const uint2 a = *reinterpret_cast<const uint2*>(kt + g * 32 + t * 8);
    const uint2 b = *reinterpret_cast<const uint2*>(kt + (g + 8) * 32 + t * 8);
    wa[0] = a.x; wa[1] = a.y;
    wb[0] = b.x; wb[1] = b.y;
    const __half2 m72 = __float2half2_rn(-72.f);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const __half2 ma = __half2half2(*reinterpret_cast<const __half*>(kt + k_scale(D, g, w)));
      const __half2 mb = __half2half2(*reinterpret_cast<const __half*>(kt + k_scale(D, g + 8, w)));
      const __half2 na = __hmul2(ma, m72), nb = __hmul2(mb, m72);
      uint32_t pa[4], pb[4];
      pairs_of(wa[w], ma, na, pa);
      pairs_of(wb[w], mb, nb, pb);
      const uint32_t a[8] = {pa[0], pb[0], pa[1], pb[1], pa[2], pb[2], pa[3], pb[3]};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint8_t* qf = frag + (size_t)(tile0 + nt) * Q_TILE + (w * 32 + lane) * 16;
        const uint4 b = *reinterpret_cast<const uint4*>(qf);
        // The sum of each 16 dims by itself, then added rounded: the tensor cores cut off what
        // they add to an accumulator.
        const uint4 b2 = *reinterpret_cast<const uint4*>(qf + WORDS * 32 * 16);
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

  uint32_t pb[NT][PIECES][2];
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
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) st.o[nt][mt][j] *= alpha[j & 1];
    }
#pragma unroll
    for (int piece = 0; piece < PIECES; ++piece)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const __half2 v = __floats2half2_rn(p[2 * j], p[2 * j + 1]);
        pb[nt][piece][j] = transpose8(h2_bits(v));
        p[2 * j] -= __low2float(v);
        p[2 * j + 1] -= __high2float(v);
      }
  }

  // V^T: lane (g, t) takes piece g of rows 2t, 2t + 1 (lo) and 2t + 8, 2t + 9 (hi).
  uint32_t v[2][2];  // [lo, hi][row of the pair]
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* at = vt + i * (D * 4) + lane * (D / 8);
    const uint2 w = *reinterpret_cast<const uint2*>(at);
    v[i][0] = w.x;
    v[i][1] = w.y;
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
              for (int mt = 0; mt < MT; ++mt)
                st.o[nt][mt][j] = st.o[nt][mt][j + 2] = __uint_as_float(0x7FC00000u);
      }
    }
  }
  const __half2 m72 = __float2half2_rn(-72.f);
  const __half2 ml = bits_h2(sc[0]), mh = bits_h2(sc[1]);
  const __half2 nl = __hmul2(ml, m72), nh = __hmul2(mh, m72);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    // Dims 4 half + 0..3 of the piece: nibble p of both halves of a word, the pair's rows.
    const uint32_t sel = half ? 0x7632u : 0x5410u;
    const uint32_t lo = __byte_perm(v[0][0], v[0][1], sel);
    const uint32_t hi = __byte_perm(v[1][0], v[1][1], sel);
    uint32_t pl[4], ph[4];
    pairs_of(lo, ml, nl, pl);
    pairs_of(hi, mh, nh, ph);
    const uint32_t a[8] = {pl[0], pl[1], ph[0], ph[1], pl[2], pl[3], ph[2], ph[3]};
    const int mt = 2 * half;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // A page's sums by themselves, then added rounded: the tensor cores cut off what they add,
      // and the losses of many pages would all go the same way.
      float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int piece = PIECES - 1; piece >= 0; --piece) {
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

// The pages of one group, through the group's ring.
struct Ring {
  uint8_t* slots;
  uint64_t* full;
  uint64_t* empty;
  const int32_t* hrow;
  const int32_t* lrow;
  SeqInfo si;
  int head, blk_begin, n_my, wp;
  int win, pid;
  int first_new;  // block whose copy, and of those behind it, waits for the kernels in front

  // Copy the group's k-th page in; the whole warp.
  __device__ bool issue(const Dev& d, int layer, int k, int wc_count, int group, int lane) {
    if (k >= win + 32) {
      win = k & ~31;
      const int j = win + lane;
      pid = j < n_my ? block_page(si, hrow, lrow, blk_begin + group + j * wp) : 0;
    }
    if (blk_begin + group + k * wp >= first_new) pdl_wait();
    const int page = __shfl_sync(FULL, pid, k - win);
    const int st = k % STAGES;
    bool ok = true;
    if (wc_count > 1 && k >= STAGES)
      ok = __all_sync(FULL, mbar_wait(d, &empty[st], (k / STAGES - 1) & 1));
    if (!ok) return false;
    if (lane == 0) {
      fence_proxy_async_smem();
      mbar_arrive_expect_tx(&full[st], PAGE);
      const uint8_t* src = d.pool + tile_at(D, d.layers, d.kv_heads, page, layer, head, 0);
      bulk_g2s(slots + st * PAGE, src, PAGE, &full[st]);
    }
    return true;
  }
};

// Rows of a pair from the `parts` slots from `slot` on: [col][D] and (m, l) per column.  Called by
// every thread of the last CTA to arrive.
__device__ void merge_parts(const float* part_o, const float2* part_ml, int cols, int slot, int parts,
                            int rows, const float* col_scale, float* s_w, float* out, int q_heads,
                            int tid, int n_threads) {
  // Weights of the parts, divided by the total: a warp per row, a part per lane.  (Four rows' loads at a
  // time here, and sixteen of a thread below: a wait for each would be most of the merge.)
  const int lane = tid & 31, warp = tid >> 5, n_warps = n_threads >> 5;
  constexpr int ROWS = 4, BATCH = 8;
  for (int r0 = warp; r0 < rows; r0 += ROWS * n_warps) {
    float2 ml[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const int r = r0 + u * n_warps;
      ml[u] = lane < parts && r < rows ? __ldcg(&part_ml[(size_t)(slot + lane) * cols + r])
                                       : make_float2(-INFINITY, 0.f);
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const int r = r0 + u * n_warps;
      if (r >= rows) break;
      float M = ml[u].x;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor_sync(FULL, M, o));
      const float w = lane < parts ? weight2(ml[u].x, M, col_scale[r]) : 0.f;
      float L = ml[u].y * w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) L += __shfl_xor_sync(FULL, L, o);
      if (lane < parts) s_w[lane * rows + r] = 16.f * w / L;
    }
  }
  __syncthreads();
  const int n = rows * (D / 4);
  for (int e0 = tid; e0 < n; e0 += 2 * n_threads) {
    float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int i0 = 0; i0 < parts; i0 += BATCH) {
      float4 x[2][BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          x[u][i] = __ldcg(reinterpret_cast<const float4*>(
                               part_o + (size_t)(slot + min(i0 + i, parts - 1)) * cols * D) +
                           min(e0 + u * n_threads, n - 1));
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        if (i0 + i >= parts) break;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float w = s_w[(i0 + i) * rows + min(e0 + u * n_threads, n - 1) / (D / 4)];
          acc[u].x += x[u][i].x * w;
          acc[u].y += x[u][i].y * w;
          acc[u].z += x[u][i].z * w;
          acc[u].w += x[u][i].w * w;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int e = e0 + u * n_threads, r = e / (D / 4);
      if (e >= n) break;
      *reinterpret_cast<float4*>(out + ((size_t)(r / G) * q_heads + r % G) * D + e % (D / 4) * 4) = acc[u];
    }
  }
}

__global__ void __launch_bounds__(384, 1) prefill_kv4_f32_kernel(
    Dev d, int layer, const float* __restrict__ q, float* __restrict__ out, float qk_scale, int wc_count,
    int wp_count, int k_slices, float* part_o, float2* part_ml, int* count, Early early) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_last, s_abort;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_threads = blockDim.x;
  const int group = warp / wc_count, wc = warp % wc_count;
  const Layout lay(wc_count, wp_count);
  const int tiles = wc_count * NT, cols = tiles * 8;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + lay.bars);
  float* col_scale = reinterpret_cast<float*>(smem + lay.scale);
  float* merge = reinterpret_cast<float*>(smem + lay.merge);
  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < wp_count * STAGES; ++i) {
      mbar_init(&bars[i], 1);
      mbar_init(&bars[wp_count * STAGES + i], wc_count);
    }
    fence_mbar_init();
  }
  __syncthreads();
  // Before the wait below an early launch reads only what the append wrote (sessions, page tables,
  // pages); q, outputs, partial states and counters come after it.
  if (early == EARLY_NONE) pdl_wait();
  pdl_launch_dependents();

  const int H = d.kv_heads, pair = blockIdx.x / k_slices, slice = blockIdx.x % k_slices;
  const int seq = pair / H, head = pair % H;
  const SeqInfo si = d.seq[seq];
  const int parts = min(k_slices, si.n_blocks);
  if (d.g->n_units == 0 || slice >= parts) {  // the append failed; no page left for this CTA
    pdl_wait();
    return;
  }
  Ring ring;
  ring.slots = smem + lay.ring + group * STAGES * PAGE;
  ring.full = bars + group * STAGES;
  ring.empty = bars + (wp_count + group) * STAGES;
  ring.wp = wp_count;
  ring.si = si;
  ring.head = head;
  ring.blk_begin = (int)((int64_t)slice * si.n_blocks / parts);
  ring.hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
  ring.lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
  const int nblk = (int)((int64_t)(slice + 1) * si.n_blocks / parts) - ring.blk_begin;
  ring.n_my = nblk > group ? (nblk - group + wp_count - 1) / wp_count : 0;
  ring.win = -32;
  ring.pid = 0;
  ring.first_new = early == EARLY_OLD ? si.n_hist_pages + (si.live_head + si.n_live - si.t) / PS : si.n_blocks;
  int issued = 0;  // pages copied or in flight (loader warp)
  bool ok = true;
  if (wc == 0)
    for (; ok && issued < min(STAGES, ring.n_my); ++issued)
      ok = ring.issue(d, layer, issued, wc_count, group, lane);
  pdl_wait();
  build_queries(d, si, head, cols, q, qk_scale, smem + lay.q, col_scale, tid, n_threads);
  __syncthreads();
  State st;
  st.clear();
  const int last0 = si.n_hist + si.n_live - si.t;
  int done = 0;
  for (; ok && done < ring.n_my; ++done) {
    const int stage = done % STAGES;
    ok = __all_sync(FULL, mbar_wait(d, &ring.full[stage], (done / STAGES) & 1));
    if (!ok) break;
    const BlockRange br = block_range(si, ring.blk_begin + group + done * wp_count);
    page_step(ring.slots + stage * PAGE, smem + lay.q, col_scale, br, last0, wc * NT, st, lane);
    __syncwarp();
    if (wc_count > 1 && lane == 0) mbar_arrive(&ring.empty[stage]);
    if (wc == 0 && issued < ring.n_my) {
      ok = ring.issue(d, layer, issued, wc_count, group, lane);
      if (ok) ++issued;
    }
  }
  if (!ok && lane == 0) s_abort = 1;
  __syncthreads();
  if (s_abort) {
    // A wait gave up: the loader drains the copies that it still has in flight (bounded), then the
    // whole CTA stops.
    if (wc == 0)
      for (int k = done; k < issued; ++k) mbar_wait(d, &ring.full[k % STAGES], (k / STAGES) & 1);
    return;
  }

  // Merge the groups, halving their number; complete the sums over the lanes of a row.
  for (int half = wp_count / 2; half > 0; half /= 2) {
    float* at = merge + ((size_t)(group % half) * wc_count + wc) * 32 * STATE + lane;
    if (group >= half && group < 2 * half) st.each([&](int i, float& x) { at[i * 32] = x; });
    __syncthreads();
    if (group < half) st.add(at, col_scale + wc * NT * 8 + 2 * (lane & 3));
    __syncthreads();
  }
  const int g = lane >> 2, t = lane & 3, rows = si.t * G;
  const size_t out_row = ((size_t)si.q_row0 * d.q_heads + head * G) * D;
  if (group == 0) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float l = st.l[nt][j];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(FULL, l, off);
        const int col = (wc * NT + nt) * 8 + 2 * t + j;
        if (col >= rows) continue;
        const float f = parts == 1 ? 16.f / l : 1.f;
        float* to = parts == 1
                        ? out + out_row + ((size_t)(col / G) * d.q_heads + col % G) * D + g * (D / 8)
                        : part_o + ((size_t)blockIdx.x * cols + col) * D + g * (D / 8);
        float y[D / 8];
#pragma unroll
        for (int e = 0; e < D / 8; ++e) y[e] = st.o[nt][e / 2][j + 2 * (e & 1)] * f;
        Eight<float>::store(to, y);
        if (parts > 1 && g == 0) part_ml[(size_t)blockIdx.x * cols + col] = make_float2(st.m[nt][j], l);
      }
  }
  if (parts == 1) return;
  int* counter = &count[pair];
  __syncthreads();
  if (tid == 0) s_last = arrive_acq_rel(counter, parts);
  __syncthreads();
  if (!s_last) return;
  merge_parts(part_o, part_ml, cols, pair * k_slices, parts, rows, col_scale,
              reinterpret_cast<float*>(smem + lay.weight), out + out_row, d.q_heads, tid, n_threads);
  if (tid == 0) *counter = 0;
}

// Warps of a page group for chunks of up to max_t tokens, and page groups of a CTA: 12 warps at most.
int warps_of(int max_t) { return (max_t * G + 8 * NT - 1) / (8 * NT); }
int groups_of(int wc) { return wc <= 3 ? 4 : 2; }

}  // namespace

cudaError_t kv4_prefill_f32_limits(Limits* lim) {
  constexpr int MOST = 226 * 1024;
  const void* fn = reinterpret_cast<const void*>(&prefill_kv4_f32_kernel);
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST);
  for (int wc = 1; wc <= KV4_PF_WARPS && e == cudaSuccess; ++wc) {
    const int wp = groups_of(wc);
    int per_sm = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, fn, 32 * wc * wp, Layout(wc, wp).total);
    lim->kv4_prefill[wc] = per_sm * lim->sms;
  }
  return e;
}

cudaError_t launch_prefill_kv4_f32(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                                   int n_pairs, int max_t, int64_t units, Early early, cudaStream_t s) {
  const int wc = warps_of(max_t), wp = groups_of(wc), cols = wc * NT * 8, grid = lim.kv4_prefill[wc];
  // Slots of partial states, one to a CTA.
  const int64_t floats = (int64_t)d.pf_slots * PF_MAX_TOKENS * G * 128;
  const int64_t slots = std::min<int64_t>(floats / (cols * D), (int64_t)d.pf_slots * PF_MAX_TOKENS * G / cols);
  // Slices of a pair, by what they were measured to take: a CTA 4 us beside its groups' pages of 1.4 us
  // each, a merge 9 us and 0.7 us a slice (one session of 600 positions, 23 tokens: 31 us in one slice,
  // 21.6 in 4, 23 in 8, 33 in 19; of 8000 positions, 17 tokens: 196, 60, 38, 31.6 us).
  const int pages = (int)std::max<int64_t>(1, (units + n_pairs - 1) / n_pairs);
  int k = 1;
  float least = 1e30f;
  for (int x = 1; x <= std::min<int64_t>(std::min(PARTS, pages), std::max<int64_t>(1, slots / n_pairs)); ++x) {
    const int waves = (n_pairs * x + grid - 1) / grid, each = ((pages + x - 1) / x + wp - 1) / wp;
    const float t = waves * (4.f + 1.4f * each) + (x > 1 ? 9.f + 0.7f * x : 0.f);
    if (t < least) {
      least = t;
      k = x;
    }
  }
  const float scale = 16.f * LOG2E / sqrtf((float)D);
  return launch_ex(&prefill_kv4_f32_kernel, dim3(n_pairs * k), dim3(32 * wc * wp), Layout(wc, wp).total,
                   s, true, d, layer, static_cast<const float*>(q), static_cast<float*>(out), scale, wc,
                   wp, k, d.pf_part_o, d.pf_part_ml, d.pf_count, early);
}

}  // namespace kvc
