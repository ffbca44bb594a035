// Attention over whole prompts (kvc_attn_prompt): for the queries of the last append, chunks of any
// length, out = softmax(RoPE(q, p) . k / sqrt(D)) v over every resident key at or before the query.
//
// One pass over the keys with a running maximum and sum a row, in binary32.
#include <cmath>

#include "kvc_prompt.h"
#include "kvc_prompt_tile.cuh"

namespace kvc {

namespace {

// A CTA takes 16 tokens of one session and KV head at a time: thread (ty, tx) has the scores of rows
// 4 ty + i and keys tx + 16 c, and of the output rows 4 ty + i the dims 4 tx + 64 c.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) prompt_kernel(Dev d, int layer, const T* q, T* out,
                                                         float scale) {
  extern __shared__ __align__(16) float sm[];
  using TL = Tile<T, D>;
  constexpr int NC = D / 64, PP = KT + 4;
  float *s_q = sm, *s_k = s_q + RT * TL::PITCH, *s_p = s_k + KT * TL::PITCH;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  pdl_wait();
  pdl_launch_dependents();
  if (d.g->n_units == 0) return;  // the append failed
  int item = blockIdx.x;
  for (int i = 0; i < d.g->n_seq; ++i) {
    const SeqInfo si = d.seq[i];
    const int items = (si.t + 15) / 16 * d.kv_heads;
    for (; item < items; item += gridDim.x) {
      const int head = item % d.kv_heads, t0 = item / d.kv_heads * 16;
      const int q_log0 = si.n_hist + si.n_live - si.t, q_log = q_log0 + t0 + ty;
      const int seen_last = q_log0 + min(t0 + 15, si.t - 1);  // by any row of the item
      __syncthreads();
      TL::load_q(d, si, head, t0, q, scale, s_q);
      float m[4], l[4];
      float4 o[4][NC];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[r][c] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      for (int b0 = 0; b0 < si.n_blocks && block_range(si, b0).base <= seen_last; b0 += 4) {
        __syncthreads();
        TL::load_kv(d, si, layer, 0, head, b0, s_k);
        __syncthreads();
        float s[4][4];
        TL::scores(s_q, s_k, ty, tx, s);
        __syncthreads();
        TL::load_kv(d, si, layer, 1, head, b0, s_k);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          int index;
          const bool seen = key_index(si, b0 + c, tx, &index) && index <= q_log;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!seen) s[r][c] = -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float mx = fmaxf(fmaxf(s[r][0], s[r][1]), fmaxf(s[r][2], s[r][3]));
#pragma unroll
          for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, off));
          const float mn = fmaxf(m[r], mx), al = exp2_safe(m[r], mn);
          m[r] = mn;
          float rs = 0.f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float p = exp2_safe(s[r][c], mn);
            rs += p;
            s_p[(4 * ty + r) * PP + tx + 16 * c] = p;
          }
          l[r] = l[r] * al + rs;
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            o[r][c].x *= al;
            o[r][c].y *= al;
            o[r][c].z *= al;
            o[r][c].w *= al;
          }
        }
        __syncthreads();
        for (int k = 0; k < KT; ++k) {
          // A key that the token does not see counts as absent, whatever its value holds.
          int index;
          if (!key_index(si, b0 + k / PS, k % PS, &index) || index > q_log) continue;
          float4 v[NC];
#pragma unroll
          for (int c = 0; c < NC; ++c)
            v[c] = *reinterpret_cast<const float4*>(s_k + k * TL::PITCH + 4 * tx + 64 * c);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = s_p[(4 * ty + r) * PP + k];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              o[r][c].x = fmaf(p, v[c].x, o[r][c].x);
              o[r][c].y = fmaf(p, v[c].y, o[r][c].y);
              o[r][c].z = fmaf(p, v[c].z, o[r][c].z);
              o[r][c].w = fmaf(p, v[c].w, o[r][c].w);
            }
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) l[r] += __shfl_xor_sync(FULL, l[r], off);
        if (t0 + ty >= si.t) continue;
        const float inv = 1.f / l[r];
        T* row = out + ((size_t)(si.q_row0 + t0 + ty) * d.q_heads + head * G + r) * D + 4 * tx;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          row[64 * c] = from_float<T>(o[r][c].x * inv);
          row[64 * c + 1] = from_float<T>(o[r][c].y * inv);
          row[64 * c + 2] = from_float<T>(o[r][c].z * inv);
          row[64 * c + 3] = from_float<T>(o[r][c].w * inv);
        }
      }
    }
    item -= items;
  }
}

template <typename T, int D>
constexpr int prompt_smem() {
  return Tile<T, D>::SMEM + RT * (KT + 4) * 4;
}

template <typename T, int D>
cudaError_t launch(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                   cudaStream_t s) {
  return launch_ex(&prompt_kernel<T, D>, dim3(lim.sms * 2), dim3(THREADS), prompt_smem<T, D>(), s, true,
                   d, layer, static_cast<const T*>(q), static_cast<T*>(out), LOG2E / sqrtf((float)D));
}

template <typename T, int D>
cudaError_t attributes() {
  return cudaFuncSetAttribute(prompt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              prompt_smem<T, D>());
}

}  // namespace

cudaError_t prompt_attributes(const Dev& d) {
  const cudaError_t e = d.esz == 2 ? prompt_tc_attributes() : attributes<float, 64>();
  return e != cudaSuccess ? e : weights_attributes(d);
}

cudaError_t launch_attn_prompt(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                               int n_seq, int max_t, int pages_max, int64_t pages_sum,
                               LaunchOrder* order, cudaStream_t s, int64_t* launches) {
  // (The kernel waits for the one before it before it lets the next one start.)
  const cudaError_t e = d.esz == 2 ? launch_prompt_tc(d, lim, layer, q, out, s)
                                   : launch<float, 64>(d, lim, layer, q, out, s);
  *launches += e == cudaSuccess;
  order->launched(layer, false);
  return e;
}

}  // namespace kvc
