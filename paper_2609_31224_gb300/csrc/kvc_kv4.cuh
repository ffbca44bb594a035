// Device code shared by the kernels on 4-bit rows (kvc_kv4.h): a group's scale and codes, the
// rotation of a key that is held in 4 bits, and a row's chunk back from its bytes.
#pragma once

#include <cuda_fp16.h>

#include "kvc_kv4.h"
#include "kvc_launch.cuh"
#include "kvc_rope.cuh"

namespace kvc {

namespace kv4 {

// Bits of |x|: they order as the numbers do, infinities above them and NaN on top.
__device__ inline uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The scale of a group whose largest |x| has these bits.
__device__ inline float scale_of(uint32_t most) {
  if (most >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  // most / 7 by the two words of 1 / 7 (the nearest binary32 number and what is left): rounded as the
  // quotient is, for every most.
  constexpr float SEVENTH = (float)(1. / CODE_MAX), REST = (float)(1. / CODE_MAX - (double)SEVENTH);
  const float s = __fmaf_rn(__uint_as_float(most), SEVENTH, __uint_as_float(most) * REST);
  // Multiples of 2^e: the seventh significant bit of s, 2^-20 at the finest.
  const int e = max((int)(__float_as_uint(s) >> 23) - 127 - (SCALE_BITS - 1), SCALE_FINEST_EXP);
  const float step = __uint_as_float((uint32_t)(127 + e) << 23);
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  return fminf(rintf(s * inv) * step, SCALE_MAX);
}
__device__ inline __half stored_scale(float s) { return __float2half_rn(s * 0.0625f); }

// Largest |x| of three, NaN if one is.
__device__ inline float most_of(float a, float b, float c) {
  float y;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
template <int N>
__device__ inline uint32_t most_of(const float (&x)[N]) {
  float y = 0.f;
#pragma unroll
  for (int i = 0; i + 1 < N; i += 2) y = most_of(y, x[i], x[i + 1]);
  if constexpr (N % 2 == 1) y = most_of(y, x[N - 1], 0.f);
  return __float_as_uint(y);
}

// What a group's elements are divided by (its scale, 1 where that is 0 or NaN), and the reciprocal in
// two words: inv within a unit in the last place, rest = 1 / by - inv from the remainder 1 - inv by,
// which one fma gives exactly.  x inv + x rest is then the quotient but for 2^-44 of it, and its rounding
// to binary32 is that of x / by wherever the nearest integer depends on it: `by` has 7 significant bits,
// so the quotient of a number next to (k + 1/2) by is at least 2^-33 away from what rounds to k + 1/2.
struct Divisor {
  float by, inv, rest;
  __device__ explicit Divisor(float s) {
    by = s > 0.f ? s : 1.f;
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(by));
    rest = __fmaf_rn(-inv, by, 1.f) * inv;
  }
  // Whether a code of the group whose largest |x| has these bits can pass CODE_MAX (its scale is the
  // finest, the largest or none).
  __device__ bool passes(uint32_t most) const { return most > __float_as_uint(7.4f * by); }
};
// Elements of a group whose codes may pass CODE_MAX, at what CODE_MAX stands for (NaN at 0).
template <int N>
__device__ inline void hold_codes(float (&x)[N], float by) {
  const float lim = CODE_MAX * by;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = isnan(x[i]) ? 0.f : fminf(fmaxf(x[i], -lim), lim);
}

// Nibbles of N <= 8 elements (rounded to nearest, ties to even, of the quotient; none passes
// CODE_MAX).  1.5 2^23 + 8 puts code + 8 in the low bits of the sum; the bits above them add up to a
// constant that the word starts without.
template <int N>
__device__ inline uint32_t codes_of(const float (&x)[N], float inv, float rest) {
  constexpr uint32_t MAGIC = 0x4B400000u;  // 1.5 2^23
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) w -= MAGIC << (4 * i);
  if constexpr (N % 2 == 1) {
    w += __float_as_uint(__fmaf_rn(x[N - 1], inv, x[N - 1] * rest) + (12582912.f + 8.f)) << (4 * (N - 1));
  }
  const float2 inv2 = make_float2(inv, inv), rest2 = make_float2(rest, rest);
  const float2 up = make_float2(12582912.f + 8.f, 12582912.f + 8.f);
#pragma unroll
  for (int i = 0; i + 1 < N; i += 2) {
    const float2 y = make_float2(x[i], x[i + 1]);
    const float2 z = __fadd2_rn(__ffma2_rn(y, inv2, __fmul2_rn(y, rest2)), up);
    w += __float_as_uint(z.x) << (4 * i);
    w += __float_as_uint(z.y) << (4 * i + 4);
  }
  return w;
}

// Rotate-half of one pair, every product and sum rounded (rope_pair fuses one of each): codes
// next to a rounding boundary depend on the last bit.
__device__ inline void turn_pair(float x1, float x2, float2 c, float& y1, float& y2) {
  y1 = __fsub_rn(__fmul_rn(x1, c.x), __fmul_rn(x2, c.y));
  y2 = __fadd_rn(__fmul_rn(x2, c.x), __fmul_rn(x1, c.y));
}

// 8 elements of T as binary32 and back.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 w;
  __device__ void load(const __nv_bfloat16* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ void get(float (&f)[8]) const { Chunk16<__nv_bfloat16>::unpack(w, f); }
  __device__ static void store(__nv_bfloat16* p, const float (&f)[8]) {
    *reinterpret_cast<uint4*>(p) = Chunk16<__nv_bfloat16>::pack(f);
  }
};
template <>
struct Eight<float> {
  uint4 a, b;
  __device__ void load(const float* p) {
    a = __ldcs(reinterpret_cast<const uint4*>(p));
    b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
  }
  __device__ void get(float (&f)[8]) const {
    f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y);
    f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
    f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y);
    f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
  }
  __device__ static void store(float* p, const float (&f)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *(reinterpret_cast<float4*>(p) + 1) = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// Values of 8 nibbles of a group whose stored scale is m.
__device__ inline void values_of(uint32_t w, __half m, float (&f)[8]) {
  const float s = __half2float(m) * 16.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)((int)(w >> (4 * i) & 15u) - 8) * s;
}

// -- tensor cores ------------------------------------------------------------------------------
__device__ inline uint32_t h2_bits(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
__device__ inline __half2 bits_h2(uint32_t u) { return *reinterpret_cast<const __half2*>(&u); }

__device__ inline void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                               uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// d = a b + c.
__device__ inline void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                               uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]),
        "f"(c[3]));
}

// Transpose of an 8 x 8 matrix of binary16 numbers held as accumulators are (lane (g, t): row g,
// columns 2t and 2t + 1).
__device__ inline uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// (x & a) | b in one instruction.
__device__ inline uint32_t and_or(uint32_t x, uint32_t a, uint32_t b) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(x), "r"(a), "r"(b));
  return y;
}

// The pairs of a word as binary16 numbers (n - 8) m, exact: pair p is nibbles p and p + 4, m a scale
// for each of the two, neg72m = -72 m.  Bits 4..7 of a half are (64 + n) m - 72 m in one step; bits
// 0..3 are (1024 + n) - 1032, then times m: as many instructions as a shift would take, but the
// pipes of shifts and of products then have about the same to do.
__device__ inline void pairs_of(uint32_t w, __half2 m, __half2 neg72m, uint32_t (&v)[4]) {
  const __half2 k1032 = __float2half2_rn(-1032.f);
  const uint32_t x = w >> 8;
  v[0] = h2_bits(__hmul2(__hadd2(bits_h2(and_or(w, 0x000F000Fu, 0x64006400u)), k1032), m));
  v[1] = h2_bits(__hfma2(bits_h2(and_or(w, 0x00F000F0u, 0x54005400u)), m, neg72m));
  v[2] = h2_bits(__hmul2(__hadd2(bits_h2(and_or(x, 0x000F000Fu, 0x64006400u)), k1032), m));
  v[3] = h2_bits(__hfma2(bits_h2(and_or(x, 0x00F000F0u, 0x54005400u)), m, neg72m));
}

// Words of shared memory (32-bit address).
__device__ inline void lds(uint32_t at, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
               : "r"(at));
}
__device__ inline void lds(uint32_t at, uint32_t (&w)[2]) {
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
}
__device__ inline void lds(uint32_t at, uint32_t (&w)[1]) {
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at));
}
__device__ inline void lds(uint32_t at, uint32_t& w) {
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at));
}

// bulk_g2s with an L2 policy.
__device__ inline void bulk_g2s_hint(void* dst_smem, const void* src_gmem, uint32_t bytes,
                                     uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], "
      "%2, [%3], %4;" ::"r"(smem_u32(dst_smem)),
      "l"(src_gmem), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}

}  // namespace kv4

}  // namespace kvc
