// Score tiles on CUDA cores, for the calls on whole prompts: 64 query rows (16 tokens of one KV head's
// four query heads) by 64 keys (four pages), in binary32.
#pragma once

#include "kvc_launch.cuh"
#include "kvc_rope.cuh"

namespace kvc {

namespace {

constexpr int G = 4;
constexpr int RT = 64, KT = 64;  // query rows and keys of a tile
constexpr int THREADS = 256;     // 16 x 16: four rows (a token's heads) and four keys each
constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr float LOG2E = 1.4426950408889634f;

template <typename T, int D>
struct Tile {
  static constexpr int PITCH = D + 4;
  static constexpr int SMEM = (RT + KT) * PITCH * 4;

  // Query rows of tokens [t0, t0 + 16), rotated and scaled; rows past the chunk are zero.
  __device__ static void load_q(const Dev& d, const SeqInfo& si, int head, int t0, const T* q,
                                float scale, float* s_q) {
    using CK = Chunk16<T>;
    constexpr int VEC = CK::N, HALF = D / 2, KC = HALF / VEC;
    for (int i = threadIdx.x; i < RT * KC; i += THREADS) {
      const int r = i / KC, c = i % KC, t = t0 + r / G;
      float ya[VEC], yb[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) ya[e] = yb[e] = 0.f;
      if (t < si.t) {
        const T* row = q + ((size_t)(si.q_row0 + t) * d.q_heads + head * G + r % G) * D + c * VEC;
        float xa[VEC], xb[VEC];
        CK::unpack(*reinterpret_cast<const uint4*>(row), xa);
        CK::unpack(*reinterpret_cast<const uint4*>(row + HALF), xb);
        const float2* cs = d.rope + (size_t)(si.pos_first + t) * HALF + c * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          rope_pair(xa[e], xb[e], cs[e], ya[e], yb[e]);
          ya[e] *= scale;
          yb[e] *= scale;
        }
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        s_q[r * PITCH + c * VEC + e] = ya[e];
        s_q[r * PITCH + HALF + c * VEC + e] = yb[e];
      }
    }
  }
  // Keys (kv = 0) or values (1) of pages b0 .. b0 + 3; slots that hold none are zero.
  __device__ static void load_kv(const Dev& d, const SeqInfo& si, int layer, int kv, int head, int b0,
                                 float* s_k) {
    using CK = Chunk16<T>;
    constexpr int VEC = CK::N, KC = D / VEC;
    const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
    const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
    for (int i = threadIdx.x; i < KT * KC; i += THREADS) {
      const int key = i / KC, c = i % KC, b = b0 + key / PS;
      float x[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[e] = 0.f;
      if (b < si.n_blocks) {
        const BlockRange br = block_range(si, b);
        const int s = key % PS;
        if (s >= br.lo && s < br.hi) {
          const int page = block_page(si, hrow, lrow, b);
          CK::unpack(*reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(d.pool) +
                                                     pool_offset_elems(d, page, layer, kv, head, s) + c * VEC), x);
        }
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) s_k[key * PITCH + c * VEC + e] = x[e];
    }
  }
  // Scores of rows 4 ty + i and keys tx + 16 c.
  __device__ static void scores(const float* s_q, const float* s_k, int ty, int tx, float (&s)[4][4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[i][c] = 0.f;
#pragma unroll 4
    for (int j = 0; j < D; j += 4) {
      float4 x[4], k[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(s_q + (4 * ty + i) * PITCH + j);
#pragma unroll
      for (int c = 0; c < 4; ++c) k[c] = *reinterpret_cast<const float4*>(s_k + (tx + 16 * c) * PITCH + j);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[i][c] = fmaf(x[i].x, k[c].x, s[i][c]);
          s[i][c] = fmaf(x[i].y, k[c].y, s[i][c]);
          s[i][c] = fmaf(x[i].z, k[c].z, s[i][c]);
          s[i][c] = fmaf(x[i].w, k[c].w, s[i][c]);
        }
    }
  }
};

// Whether key tx of page b is resident, and its index in retained order.
__device__ inline bool key_index(const SeqInfo& si, int b, int tx, int* index) {
  if (b >= si.n_blocks) return false;
  const BlockRange br = block_range(si, b);
  *index = br.base + tx;
  return tx >= br.lo && tx < br.hi;
}

}  // namespace

}  // namespace kvc
