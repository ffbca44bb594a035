// Attention weights that the resident positions draw (kvc_attn_weights): for the queries of the last
// append, w_j += sum over tokens t and query heads h of p_thj = 2^(s_thj - lse_th), where s are the
// scores in units of log2 (scaled by log2(e) / sqrt(D)) and lse_th = log2 sum_j 2^s_thj over the keys
// that t sees.  Everything is in binary32.
//
// A weight needs its row's sum first, so the scores are formed twice: the first kernel forms lse, the
// second the sums over rows, for a key tile and KV head each; a third adds the heads up in their order,
// so that results repeat.
#include <algorithm>
#include <cmath>

#include "kvc_prompt_tile.cuh"
#include "kvc_weights.h"

namespace kvc {

namespace {

// lse of every row: a CTA takes 16 tokens of one session and KV head at a time.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) weights_lse_kernel(Dev d, int layer, const T* q, float scale,
                                                              WeightsWork work) {
  extern __shared__ __align__(16) float sm[];
  using TL = Tile<T, D>;
  float *s_q = sm, *s_k = sm + RT * TL::PITCH;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  pdl_wait();
  pdl_launch_dependents();
  if (d.g->n_units == 0) return;  // the append failed
  float* lse = work.lse;
  int item = blockIdx.x;
  for (int i = 0; i < d.g->n_seq; ++i) {
    const SeqInfo si = d.seq[i];
    const int items = (si.t + 15) / 16 * d.kv_heads;
    for (; item < items; item += gridDim.x) {
      const int head = item % d.kv_heads, t0 = item / d.kv_heads * 16;
      const int q_log = si.n_hist + si.n_live - si.t + t0 + ty;
      __syncthreads();
      TL::load_q(d, si, head, t0, q, scale, s_q);
      float m[4], l[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
      }
      for (int b0 = 0; b0 < si.n_blocks; b0 += 4) {
        __syncthreads();
        TL::load_kv(d, si, layer, 0, head, b0, s_k);
        __syncthreads();
        float s[4][4];
        TL::scores(s_q, s_k, ty, tx, s);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          int index;
          const bool seen = key_index(si, b0 + c, tx, &index) && index <= q_log;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (!seen) continue;
            const float mn = fmaxf(m[r], s[r][c]);
            l[r] = l[r] * exp2_safe(m[r], mn) + exp2f(s[r][c] - mn);
            m[r] = mn;
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
          const float mo = __shfl_xor_sync(FULL, m[r], o), lo = __shfl_xor_sync(FULL, l[r], o);
          const float mn = fmaxf(m[r], mo);
          l[r] = l[r] * exp2_safe(m[r], mn) + lo * exp2_safe(mo, mn);
          m[r] = mn;
        }
        if (tx == 0 && t0 + ty < si.t)
          lse[(size_t)(si.q_row0 + t0 + ty) * d.q_heads + head * G + r] = m[r] + log2f(l[r]);
      }
    }
    item -= items;
  }
}

// Sums over the rows of one KV head for each key: a CTA takes four pages of one session and head.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) weights_sum_kernel(Dev d, int layer, const T* q, float scale,
                                                              WeightsWork work) {
  extern __shared__ __align__(16) float sm[];
  using TL = Tile<T, D>;
  float *s_q = sm, *s_k = sm + RT * TL::PITCH;
  __shared__ float s_sum[16][KT + 1];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  pdl_wait();
  pdl_launch_dependents();
  if (d.g->n_units == 0) return;
  const float* lse = work.lse;
  float* sums = work.scores;
  int item = blockIdx.x;
  for (int i = 0; i < d.g->n_seq; ++i) {
    const SeqInfo si = d.seq[i];
    const int items = (si.n_blocks + 3) / 4 * d.kv_heads;
    const int q_log0 = si.n_hist + si.n_live - si.t;
    for (; item < items; item += gridDim.x) {
      const int head = item % d.kv_heads, b0 = item / d.kv_heads * 4;
      __syncthreads();
      TL::load_kv(d, si, layer, 0, head, b0, s_k);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      int index[4];
      bool in[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) in[c] = key_index(si, b0 + c, tx, &index[c]);
      // The first token that sees a key of the tile.
      const int t_first = max(0, block_range(si, b0).base - q_log0) / 16 * 16;
      for (int t0 = t_first; t0 < si.t; t0 += 16) {
        __syncthreads();
        TL::load_q(d, si, head, t0, q, scale, s_q);
        __syncthreads();
        float s[4][4];
        TL::scores(s_q, s_k, ty, tx, s);
        if (t0 + ty < si.t) {
          const float* row = lse + (size_t)(si.q_row0 + t0 + ty) * d.q_heads + head * G;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (in[c] && index[c] <= q_log0 + t0 + ty)
#pragma unroll
              for (int r = 0; r < 4; ++r) sum[c] += exp2f(s[r][c] - row[r]);
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) s_sum[ty][tx + 16 * c] = sum[c];
      __syncthreads();
      if (threadIdx.x < KT) {
        const int b = b0 + threadIdx.x / PS, s = threadIdx.x % PS;
        int at;
        if (key_index(si, b, s, &at)) {
          float w = 0.f;
          for (int r = 0; r < 16; ++r) w += s_sum[r][threadIdx.x];
          const int page = block_page(si, d.hist_pt + (size_t)si.sid * d.max_pages_per_session,
                                      d.live_pt + (size_t)si.sid * d.max_pages_per_session, b);
          sums[((size_t)head * d.n_pages + page) * PS + s] = w;
        }
      }
    }
    item -= items;
  }
}

// The planes' sums of each resident position, added to what it weighs: blockIdx.y is the session of the
// call.
__global__ void __launch_bounds__(THREADS) weights_add_kernel(Dev d, int planes, WeightsWork work,
                                                              float* weights) {
  pdl_wait();
  pdl_launch_dependents();
  if (d.g->n_units == 0) return;
  const SeqInfo si = d.seq[blockIdx.y];
  const size_t plane = (size_t)d.n_pages * PS;
  for (int at = blockIdx.x * THREADS + threadIdx.x; at < si.n_blocks * PS; at += gridDim.x * THREADS) {
    int index;
    if (!key_index(si, at / PS, at % PS, &index)) continue;
    const int page = block_page(si, d.hist_pt + (size_t)si.sid * d.max_pages_per_session,
                                d.live_pt + (size_t)si.sid * d.max_pages_per_session, at / PS);
    const int gs = page * PS + at % PS;
    float w = 0.f;
#pragma unroll 8
    for (int h = 0; h < planes; ++h) w += work.scores[h * plane + gs];
    weights[(size_t)si.sid * d.max_positions + d.meta_pos[gs]] += w;
  }
}

cudaError_t launch_add(const Dev& d, const Limits& lim, int planes, const WeightsWork& work, float* weights,
                       int n_seq, cudaStream_t s, int64_t* launches) {
  const dim3 grid(std::max(1, std::min(64, 8 * lim.sms / n_seq)), n_seq);
  const cudaError_t e = launch_ex(&weights_add_kernel, grid, dim3(THREADS), 0, s, true, d, planes, work,
                                  weights);
  *launches += e == cudaSuccess;
  return e;
}

template <typename T, int D>
cudaError_t attributes() {
  const int smem = Tile<T, D>::SMEM;
  const cudaError_t e = cudaFuncSetAttribute(weights_lse_kernel<T, D>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e != cudaSuccess ? e
                          : cudaFuncSetAttribute(weights_sum_kernel<T, D>,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
}

template <typename T, int D>
cudaError_t launch(const Dev& d, const Limits& lim, int layer, const void* q, const WeightsWork& work,
                   cudaStream_t s, int64_t* launches) {
  const float scale = LOG2E / sqrtf((float)D);
  const dim3 grid(lim.sms * 3);
  cudaError_t e = launch_ex(&weights_lse_kernel<T, D>, grid, dim3(THREADS), Tile<T, D>::SMEM, s, true, d,
                            layer, static_cast<const T*>(q), scale, work);
  *launches += e == cudaSuccess;
  if (e != cudaSuccess) return e;
  e = launch_ex(&weights_sum_kernel<T, D>, grid, dim3(THREADS), Tile<T, D>::SMEM, s, true, d, layer,
                static_cast<const T*>(q), scale, work);
  *launches += e == cudaSuccess;
  return e;
}

}  // namespace

namespace {

// The parts of a scratch area, from its start; their bytes.
size_t lay_out(uint8_t* base, int64_t n_pages, int q_heads, int max_tokens, int max_seq, WeightsWork* w) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    uint8_t* p = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  uint8_t* scores = take((size_t)n_pages * PS * q_heads * sizeof(float));
  uint8_t* lse = take((size_t)max_tokens * q_heads * sizeof(float));
  uint8_t* stats = take(((size_t)max_tokens * q_heads + WEIGHTS_STATS) * sizeof(float2));
  uint8_t* whole = take((size_t)max_seq * q_heads * sizeof(float2));
  uint8_t* parts = take((size_t)WEIGHTS_PARTS * G * sizeof(float2));
  if (w) {
    w->scores = reinterpret_cast<float*>(scores);
    w->lse = reinterpret_cast<float*>(lse);
    w->stats = reinterpret_cast<float2*>(stats);
    w->whole = reinterpret_cast<float2*>(whole);
    w->parts = reinterpret_cast<float2*>(parts);
  }
  return off;
}

}  // namespace

size_t weights_work_bytes(const kvc_config& c) {
  return lay_out(nullptr, c.n_pages, c.q_heads, c.max_tokens_per_call, c.max_seq_per_call, nullptr);
}

cudaError_t weights_attributes(const Dev& d) {
  const cudaError_t e = d.esz == 2 ? weights_tc_attributes() : attributes<float, 64>();
  return e != cudaSuccess ? e : weights_token_attributes(d);
}

cudaError_t launch_attn_weights(const Dev& d, const Limits& lim, int layer, const void* q,
                                float* weights, void* work, int n_seq, int total, int max_t,
                                int pages_max, int64_t pages_sum, LaunchOrder* order, cudaStream_t s, int64_t* launches) {
  WeightsWork w;
  lay_out(static_cast<uint8_t*>(work), d.n_pages, d.q_heads, d.max_tokens, d.max_seq, &w);
  // (Each kernel but an early one waits for the one before it before it lets the next one start.)
  const bool early = order->early(layer, false);
  order->launched(layer, false);
  if (max_t == 1) return launch_weights_token(d, lim, layer, q, weights, w, n_seq, early, s, launches);
  int shares = 1;
  cudaError_t e;
  if (d.esz == 2) {
    // Where the chunk's rows alone are too few items, the keys are cut into parts; where the keys are,
    // the tokens into shares.
    const int64_t rows = ((int64_t)total + 63 * n_seq) / 64 * d.kv_heads;
    const int64_t stats = (int64_t)d.max_tokens * d.q_heads + WEIGHTS_STATS;
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>(2 * lim.sms / rows, (pages_max + 7) / 8));
    parts = std::max<int64_t>(1, std::min(parts, stats / ((int64_t)total * d.q_heads)));
    const int64_t keys = (pages_sum / 16 + n_seq) * d.kv_heads;
    while (shares < WEIGHTS_SHARES && keys * shares < 4 * lim.sms && max_t / 32 > 4 * shares) shares *= 2;
    e = launch_weights_tc(d, lim, layer, q, w, (int)parts, shares, s, launches);
  } else {
    e = launch<float, 64>(d, lim, layer, q, w, s, launches);
  }
  return e != cudaSuccess ? e : launch_add(d, lim, d.kv_heads * shares, w, weights, n_seq, s, launches);
}

}  // namespace kvc
