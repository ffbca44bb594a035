// Attention weights of single tokens (kvc_attn_weights), one token of each session of the call.
//
// The first kernel streams the keys once: scores of a (session, KV head, page) unit, 16 keys x 4 query
// heads, go to scratch ([page][KV head][slot][4], 256 bytes, a sixteenth of the unit's keys), and each
// CTA keeps the running (max, sum) of its part of a (session, KV head) pair.  The second merges the
// parts, forms 2^(s - lse) of the scores and adds them up over query heads, in one order: position by
// position, so that results repeat.  Units are split evenly over the CTAs (UnitSplit), pages of a
// segment in turn over its warps, each of which has a ring of its own.
//   bfloat16  mma.sync m16n8k16 with the keys as M: the eight columns are the four heads' q twice, in its
//             upper and lower bfloat16 piece, whose products are added in binary32: q keeps 16 bits or
//             more at the price of one
//   binary32  eight lanes a key, an eighth of the query rows in the registers of each
// Bound by the keys' bytes for many sessions: 64 sessions of 4,100 positions, 8 KV heads, 96 us a layer
// for 79 us at the copy bandwidth (5.6 TB/s); binary32, 4 KV heads, 57 us for 40.  One session, 7.9 us for 1.3
// (binary32 8.6), is two launches' latencies: their release, q or the parts, a ring's first tiles, then the
// scores' way back through L2.
#include <cmath>

#include "kvc_decode_common.cuh"
#include "kvc_rope.cuh"
#include "kvc_weights_plain.cuh"

namespace kvc {

namespace {

constexpr int TOKEN_WARPS = 8, TOKEN_THREADS = TOKEN_WARPS * 32;
constexpr int TOKEN_STAGES = 2;                    // 4 KiB each, a warp (16 warps an SM hide the latency of a unit's
                                                   // chain: 4 warps of 6 stages took 9.4 and 100 us, see above)
constexpr int UNIT_BYTES = 4096;                   // the keys of a unit, in either type
constexpr int TOKEN_SMEM = TOKEN_WARPS * TOKEN_STAGES * UNIT_BYTES + 1024;
constexpr int TOKEN_MIN_UNITS = 4;                 // of a CTA, at least
constexpr int TOKEN_NO_LIMIT = 1 << 16;

// Copy of a unit's keys into a stage (one lane).
template <typename T>
__device__ inline void load_unit(const Dev& d, int layer, int page, int head, uint8_t* dst, uint64_t* bar,
                                 const CUtensorMap* lo, const CUtensorMap* hi, uint64_t policy) {
  mbar_arrive_expect_tx(bar, UNIT_BYTES);
  if constexpr (sizeof(T) == 2) {
    const int row = (((page * d.layers + layer) * 2) * d.kv_heads + head) * PS;
    tma_load_2d_hint(dst, lo, 0, row, bar, policy);
    tma_load_2d_hint(dst + 2048, hi, 0, row, bar, policy);
  } else {
    bulk_g2s(dst, d.pool + pool_offset_elems(d, page, layer, 0, head, 0) * sizeof(T), UNIT_BYTES, bar);
  }
}

// q of `head`, rotated and scaled, as the B operand of the products: columns 0-3 the upper pieces of
// the four rows, columns 4-7 the lower ones; lane (g, t) has column g, dims 16 ks + 2t (+ 1) and + 8.
__device__ inline void q_pieces(const Dev& d, const SeqInfo& si, int head, const __nv_bfloat16* q,
                                float qk_scale, int lane, uint32_t (&qb)[8][2]) {
  constexpr int D = 128;
  const int g = lane >> 2, t = lane & 3;
  const uint32_t* row = reinterpret_cast<const uint32_t*>(
      q + ((size_t)si.q_row0 * d.q_heads + (size_t)head * G + (g & 3)) * D);
  const float2* cs = d.rope + (size_t)si.pos_first * (D / 2);
  auto piece = [&](float x, float y) {
    const uint32_t up = pack_bf16x2(x, y);
    return g < G ? up : pack_bf16x2(x - bf16lo(up), y - bf16hi(up));
  };
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t a = row[8 * ks + t + 4 * j], b = row[8 * (ks + 4) + t + 4 * j];
      const float2 c0 = cs[16 * ks + 2 * t + 8 * j], c1 = cs[16 * ks + 2 * t + 8 * j + 1];
      float a0, a1, b0, b1;
      rope_pair(bf16lo(a), bf16lo(b), c0, a0, b0);
      rope_pair(bf16hi(a), bf16hi(b), c1, a1, b1);
      qb[ks][j] = piece(a0 * qk_scale, a1 * qk_scale);
      qb[ks + 4][j] = piece(b0 * qk_scale, b1 * qk_scale);
    }
}

// A head's query rows and rotary row into L2 (either type: 1 KiB and 512 bytes).
template <typename T>
__device__ inline void prefetch_q_rows(const Dev& d, const SeqInfo& si, int head, const T* q, int lane) {
  const char* rows = reinterpret_cast<const char*>(
      q + ((size_t)si.q_row0 * d.q_heads + (size_t)head * G) * d.head_dim);
  const char* cs = reinterpret_cast<const char*>(d.rope + (size_t)si.pos_first * (d.head_dim / 2));
  if (lane < 8) prefetch_l2(rows + lane * 128);
  else if (lane < 8 + d.head_dim / 32) prefetch_l2(cs + (lane - 8) * 128);
}

// The running (max, sum) of two states.
__device__ inline void join(float& m, float& l, float mo, float lo) {
  const float mn = fmaxf(m, mo);
  l = l * exp2_safe(m, mn) + lo * exp2_safe(mo, mn);
  m = mn;
}

// The scores of a warp's units of a segment again in plain arithmetic (kvc_weights_plain.cuh), and their
// (max, sum) to ml: lane i has key i % 16 and the query heads 2 (i / 16) and + 1.
__device__ __noinline__ void score_again(const Dev& d, const SeqInfo& si, int layer, int head, int first,
                                         int count, const __nv_bfloat16* q, float qk_scale, float* scores,
                                         float2* ml, int lane) {
  const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
  const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
  const int key = lane % PS, g = lane / PS * 2;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  for (int k = 0; k < count; ++k) {
    const int blk = first + k * TOKEN_WARPS, page = block_page(si, hrow, lrow, blk);
    const BlockRange br = block_range(si, blk);
    if (key < br.lo || key >= br.hi) continue;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float s = plain_score<__nv_bfloat16, 128>(d, si, layer, head, 0, g + r, q, qk_scale, page, key);
      scores[((size_t)page * d.kv_heads + head) * (PS * G) + key * G + g + r] = s;
      join(m[r], l[r], s, s == s ? 1.f : s);
    }
  }
  __syncwarp();
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int o = 1; o < PS; o <<= 1)
      join(m[r], l[r], __shfl_xor_sync(FULL, m[r], o), __shfl_xor_sync(FULL, l[r], o));
  if (key == 0) {
    ml[g] = make_float2(m[0], l[0]);
    ml[g + 1] = make_float2(m[1], l[1]);
  }
}

// The units of a launch made for n_launch single tokens; none where the last append is of other chunks (the launch
// was captured, and d_q holds other rows).
__device__ inline UnitSplit token_split(const Dev& d, int grid, int n_launch) {
  UnitSplit us = unit_split(d, grid, TOKEN_MIN_UNITS, TOKEN_NO_LIMIT);
  if (d.g->total_tokens != n_launch || d.g->n_seq != n_launch) us.U = 0;
  return us;
}

// Two scores into a running (max, sum); -infinity adds nothing, a NaN makes the sum one (in front of all other
// keys as well, where the maximum is still -infinity).
__device__ inline void add_two(float& m, float& l, float x, float y) {
  const float mn = fmaxf(m, fmaxf(x, y)), ref = mn == -INFINITY ? 0.f : mn;
  l = l * exp2f(m - ref) + exp2f(x - ref) + exp2f(y - ref);
  m = mn;
}

template <typename T, int D>
__global__ void __launch_bounds__(TOKEN_THREADS) weights_token_kernel(
    Dev d, int layer, const __grid_constant__ CUtensorMap map_lo,
    const __grid_constant__ CUtensorMap map_hi, const T* __restrict__ q, float qk_scale,
    WeightsWork work, int n_launch, int early) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ uint64_t s_bars[TOKEN_WARPS * TOKEN_STAGES];
  __shared__ float2 s_ml[TOKEN_WARPS * G];
  __shared__ int s_abort;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = d.kv_heads;
  uint8_t* ring = tiles + warp * TOKEN_STAGES * UNIT_BYTES;
  uint64_t* bars = s_bars + warp * TOKEN_STAGES;
  if (lane == 0) {
    for (int i = 0; i < TOKEN_STAGES; ++i) mbar_init(&bars[i], 1);
    fence_mbar_init();
  }
  if (tid == 0) s_abort = 0;
  __syncthreads();
  if (!early) pdl_wait();  // (the first call after an append waits before it lets others start)
  pdl_launch_dependents();
  bool waited = false;
  const UnitSplit us = token_split(d, gridDim.x, n_launch);
  const int cta = blockIdx.x;
  if (us.U == 0 || cta >= us.n_cta) {
    if (us.U == 0 && cta == 0 && tid == 0) note_other_chunks(d);
    pdl_wait();
    return;
  }
  const int u_begin = us.start_of(cta), u_end = us.start_of(cta + 1);
  const uint64_t policy = evict_first_policy();
  uint32_t n = 0;  // units of this warp so far
  for (int u = u_begin; u < u_end;) {
    const UnitSeg seg = unit_segment(d, u, u_end);
    const SeqInfo& si = seg.si;
    const int head = seg.head, b0 = seg.blk_begin(), n_blk = seg.end - u;
    const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
    const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
    const int mine = n_blk > warp ? (n_blk - warp + TOKEN_WARPS - 1) / TOKEN_WARPS : 0;
    // Lane i has the page of this warp's unit i of a window of 32.
    auto page_of = [&](int k) { return k < mine ? block_page(si, hrow, lrow, b0 + warp + k * TOKEN_WARPS) : 0; };
    int pid = page_of(lane), pid_next = page_of(32 + lane);
    int window = 0;
    auto page_at = [&](int k) {
      return __shfl_sync(FULL, k - window < 32 ? pid : pid_next, k & 31);
    };
    for (int k = 0; k < min(mine, TOKEN_STAGES); ++k) {
      const int page = page_at(k);
      const uint32_t s = (n + k) % TOKEN_STAGES;
      if (lane == 0) load_unit<T>(d, layer, page, head, ring + s * UNIT_BYTES, &bars[s], &map_lo, &map_hi, policy);
    }
    if (!waited) {
      if (warp == 0) prefetch_q_rows(d, si, head, q, lane);
      pdl_wait();
      waited = true;
    }
    uint32_t qb[8][2];
    float qr[G][8];  // binary32: dims 4c .. and 4c + 32 .. of the rows, c = lane % 8
    if constexpr (sizeof(T) == 2) {
      q_pieces(d, si, head, q, qk_scale, lane, qb);
    } else {
      const int c = lane & 7;
      const float2* cs = d.rope + (size_t)si.pos_first * (D / 2) + 4 * c;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float* row = q + ((size_t)si.q_row0 * d.q_heads + head * G + g) * D + 4 * c;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          rope_pair(row[e], row[e + D / 2], cs[e], qr[g][e], qr[g][4 + e]);
          qr[g][e] *= qk_scale;
          qr[g][4 + e] *= qk_scale;
        }
      }
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    int failed_at = -1;
    for (int k = 0; k < mine; ++k) {
      const uint32_t s = (n + k) % TOKEN_STAGES;
      if (!__all_sync(FULL, mbar_wait(d, &bars[s], ((n + k) / TOKEN_STAGES) & 1))) {
        failed_at = k;
        break;
      }
      const int blk = b0 + warp + k * TOKEN_WARPS, page = page_at(k);
      const BlockRange br = block_range(si, blk);
      float* to = work.scores + ((size_t)page * H + head) * (PS * G);
      const uint8_t* kt = ring + s * UNIT_BYTES;
      if constexpr (sizeof(T) == 2) {
        const int g = lane >> 2, t = lane & 3;
        const int k_key = (lane & 7) + 8 * ((lane >> 3) & 1), k_col = 8 * (lane >> 4);
        const uint32_t kb = smem_u32(kt);
        float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          uint32_t a[4];
          ldsm_x4(a, kb + swz(k_key, 16 * ks + k_col));
          mma_16816(c, a, qb[ks][0], qb[ks][1]);
        }
        // Columns 2t, 2t + 1 of keys g and g + 8; the lower pieces' products are two lanes on.
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] += __shfl_xor_sync(FULL, c[i], 2);
        *reinterpret_cast<float2*>(to + (g + (t & 2) * 4) * G + 2 * (t & 1)) =
            t < 2 ? make_float2(c[0], c[1]) : make_float2(c[2], c[3]);
        const bool in0 = g >= br.lo && g < br.hi, in1 = g + 8 >= br.lo && g + 8 < br.hi;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float x = in0 ? c[r] : -INFINITY, y = in1 ? c[2 + r] : -INFINITY;
          add_two(m[r], l[r], x, y);
        }
      } else {
        // Key 4 i + j of lane group j = lane / 8; lane c of it ends up with row c % 4.
        const int j = lane >> 3, c = lane & 7;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 4 * i + j;
          const float4 ka = *reinterpret_cast<const float4*>(kt + key * 256 + c * 16);
          const float4 kb = *reinterpret_cast<const float4*>(kt + key * 256 + 128 + c * 16);
          float p[G];
#pragma unroll
          for (int g = 0; g < G; ++g) {
            p[g] = qr[g][0] * ka.x;
            p[g] = fmaf(qr[g][1], ka.y, p[g]);
            p[g] = fmaf(qr[g][2], ka.z, p[g]);
            p[g] = fmaf(qr[g][3], ka.w, p[g]);
            p[g] = fmaf(qr[g][4], kb.x, p[g]);
            p[g] = fmaf(qr[g][5], kb.y, p[g]);
            p[g] = fmaf(qr[g][6], kb.z, p[g]);
            p[g] = fmaf(qr[g][7], kb.w, p[g]);
          }
          // Sums over the eight lanes, each keeping half of its rows at a step.
          const bool up = c & 2, odd = c & 1;
          float x = up ? p[2] : p[0], y = up ? p[3] : p[1];
          x += __shfl_xor_sync(FULL, up ? p[0] : p[2], 2);
          y += __shfl_xor_sync(FULL, up ? p[1] : p[3], 2);
          float z = (odd ? y : x) + __shfl_xor_sync(FULL, odd ? x : y, 1);
          z += __shfl_xor_sync(FULL, z, 4);
          if (c < 4) to[key * G + c] = z;
          const float sc = key >= br.lo && key < br.hi ? z : -INFINITY;
          add_two(m[0], l[0], sc, -INFINITY);
        }
      }
      __syncwarp();
      if (k + TOKEN_STAGES < mine) {
        const int next = page_at(k + TOKEN_STAGES);
        if (lane == 0) {
          fence_proxy_async_smem();
          load_unit<T>(d, layer, next, head, ring + s * UNIT_BYTES, &bars[s], &map_lo, &map_hi, policy);
        }
      }
      if (k + 1 - window == 32) {
        pid = pid_next;
        window += 32;
        pid_next = page_of(window + 32 + lane);
      }
    }
    if (failed_at >= 0 && lane == 0) s_abort = 1;
    // This warp's state: lanes of the same rows together.
    bool again = false;
    if constexpr (sizeof(T) == 2) again = __any_sync(FULL, isnan(l[0] + l[1])) && failed_at < 0;
    if (again) {
      if constexpr (sizeof(T) == 2) {
        const Dev dev = d;  // (copies, so that only this branch has them in memory)
        const SeqInfo info = si;
        score_again(dev, info, layer, head, b0 + warp, mine, q, qk_scale, work.scores, s_ml + warp * G, lane);
      }
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
          join(m[r], l[r], __shfl_xor_sync(FULL, m[r], o), __shfl_xor_sync(FULL, l[r], o));
      if (lane < 2) {
        s_ml[warp * G + 2 * lane] = make_float2(m[0], l[0]);
        s_ml[warp * G + 2 * lane + 1] = make_float2(m[1], l[1]);
      }
    } else {
      for (int o = 8; o < 32; o <<= 1)
        join(m[0], l[0], __shfl_xor_sync(FULL, m[0], o), __shfl_xor_sync(FULL, l[0], o));
      if (lane < 4) s_ml[warp * G + lane] = make_float2(m[0], l[0]);
    }
    __syncthreads();
    if (s_abort) {
      // Copies still in flight land (bounded waits) before the CTA ends.
      if (failed_at >= 0)
        for (int k = failed_at; k < min(mine, failed_at + TOKEN_STAGES); ++k)
          mbar_wait(d, &bars[(n + k) % TOKEN_STAGES], ((n + k) / TOKEN_STAGES) & 1);
      return;
    }
    n += mine;
    if (tid < G) {
      float2 a = s_ml[tid];
      for (int w = 1; w < TOKEN_WARPS; ++w) join(a.x, a.y, s_ml[w * G + tid].x, s_ml[w * G + tid].y);
      if (seg.whole()) work.whole[((size_t)seg.seq * H + head) * G + tid] = a;
      else work.parts[(size_t)(2 * cta + (u == u_begin ? 0 : 1)) * G + tid] = a;
    }
    __syncthreads();
    u = seg.end;
  }
}

// Pages of one session, eight at a time: blockIdx.y is the session of the call.  (Everything that the
// append wrote is complete before the kernel in front lets this one start.)
__global__ void __launch_bounds__(TOKEN_THREADS) weights_token_add_kernel(Dev d, int grid,
                                                                          WeightsWork work,
                                                                          float* weights) {
  __shared__ __align__(16) float s_lse[64 * G];
  constexpr int AT_ONCE = TOKEN_THREADS / PS, HEADS = 8;  // pages; heads' scores on their way
  const int tid = threadIdx.x, H = d.kv_heads, seq = blockIdx.y;
  pdl_launch_dependents();
  const UnitSplit us = token_split(d, grid, gridDim.y);
  const SeqInfo si = d.seq[seq];
  const int nb = si.n_blocks, slot = tid % PS;
  if (us.U == 0 || (int)blockIdx.x * AT_ONCE >= nb) {
    pdl_wait();
    return;
  }
  const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
  const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
  int b = blockIdx.x * AT_ONCE + tid / PS, page = 0, pos = 0;
  bool in = false;
  auto find = [&] {  // this thread's slot of its page b
    in = false;
    if (b >= nb) return;
    const BlockRange br = block_range(si, b);
    in = slot >= br.lo && slot < br.hi;
    if (!in) return;
    page = block_page(si, hrow, lrow, b);
    pos = d.meta_pos[page * PS + slot];
  };
  find();
  const int lane = tid & 31;
  // A row of lse, eight lanes to its parts.
  int r = min(tid / 8, H * G - 1), start = si.unit_base + r / G * nb;
  int cf = us.owner(start), cl = us.owner(start + nb - 1), first = us.slot_of(cf, cf, start);
  pdl_wait();
  float4 x[HEADS];
  float before = 0.f;
  const float4* scores = reinterpret_cast<const float4*>(work.scores) + slot;
  auto fetch = [&](int h0) {
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
      if (in && h0 + h < H) x[h] = scores[((size_t)page * H + h0 + h) * PS];
  };
  float* at = weights + (size_t)si.sid * d.max_positions;
  fetch(0);
  if (in) before = at[pos];
  for (int r0 = 0;;) {
    float2 a = make_float2(-INFINITY, 0.f);
    if (cf == cl) {
      if (lane % 8 == 0) a = work.whole[(size_t)seq * H * G + r];
    } else {
      for (int c = cf + lane % 8; c <= cl; c += 32) {  // four loads in flight
        float2 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[i] = c + 8 * i <= cl ? work.parts[(size_t)(c + 8 * i == cf ? first : 2 * (c + 8 * i)) * G + r % G]
                                 : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) join(a.x, a.y, o[i].x, o[i].y);
      }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
      join(a.x, a.y, __shfl_xor_sync(FULL, a.x, o), __shfl_xor_sync(FULL, a.y, o));
    if (lane % 8 == 0) s_lse[r] = a.x + log2f(a.y);
    r0 += TOKEN_THREADS / 8;
    if (r0 >= H * G) break;
    r = min(r0 + tid / 8, H * G - 1);
    start = si.unit_base + r / G * nb;
    cf = us.owner(start);
    cl = us.owner(start + nb - 1);
    first = us.slot_of(cf, cf, start);
  }
  __syncthreads();
  for (;;) {
    float w = 0.f;
    for (int h0 = 0;;) {
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
        if (h0 + h < H) {
          const float4 lse = reinterpret_cast<const float4*>(s_lse)[h0 + h];
          w += (exp2f(x[h].x - lse.x) + exp2f(x[h].y - lse.y)) + (exp2f(x[h].z - lse.z) + exp2f(x[h].w - lse.w));
        }
      h0 += HEADS;
      if (h0 >= H) break;
      fetch(h0);
    }
    if (in) at[pos] = before + w;
    b += gridDim.x * AT_ONCE;
    if (b - tid / PS >= nb) break;
    find();
    fetch(0);
    if (in) before = at[pos];
  }
}

template <typename T, int D>
cudaError_t launch(const Dev& d, const Limits& lim, int layer, const void* q, float* weights,
                   const WeightsWork& work, int n_seq, bool early, cudaStream_t s, int64_t* launches) {
  CUtensorMap lo = {}, hi = {};
  if (sizeof(T) == 2 && !pool_tensor_maps(d, &lo, &hi)) return cudaErrorInvalidValue;
  const int grid = lim.sms * 2;
  cudaError_t e = launch_ex(&weights_token_kernel<T, D>, dim3(grid), dim3(TOKEN_THREADS), TOKEN_SMEM, s,
                            true, d, layer, lo, hi, static_cast<const T*>(q), LOG2E / sqrtf((float)D),
                            work, n_seq, (int)early);
  *launches += e == cudaSuccess;
  if (e != cudaSuccess) return e;
  const int per = max(1, min(64, 16 * lim.sms / n_seq));
  e = launch_ex(&weights_token_add_kernel, dim3(per, n_seq), dim3(TOKEN_THREADS), 0, s, true, d, grid,
                work, weights);
  *launches += e == cudaSuccess;
  return e;
}

template <typename T, int D>
cudaError_t attributes() {
  return cudaFuncSetAttribute(weights_token_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              TOKEN_SMEM);
}

}  // namespace

cudaError_t weights_token_attributes(const Dev& d) {
  return d.esz == 2 ? attributes<__nv_bfloat16, 128>() : attributes<float, 64>();
}

cudaError_t launch_weights_token(const Dev& d, const Limits& lim, int layer, const void* q,
                                 float* weights, const WeightsWork& work, int n_seq, bool early,
                                 cudaStream_t s, int64_t* launches) {
  return d.esz == 2 ? launch<__nv_bfloat16, 128>(d, lim, layer, q, weights, work, n_seq, early, s, launches)
                    : launch<float, 64>(d, lim, layer, q, weights, work, n_seq, early, s, launches);
}

}  // namespace kvc
