// Rows held in 4 bits (KVC_KV4): the write (rotation and quantisation in one pass), the move of
// survivors of an eviction, and the read-back of rows of either kind of cache in the element type.
#include "kvc_kv4.cuh"

namespace kvc {

namespace {

using namespace kv4;

constexpr int THREADS = 256;
constexpr unsigned FULL = 0xFFFFFFFFu;

// K rotated at its position and V, quantised into the page slots of the plan kernel.  Input
// [L][total][Hkv][D]; blockIdx.y is the input layer, cache layer layer0 + blockIdx.y.
// A thread takes 8 dims of the first half of a K row with their rotate-half partners, and the
// same dims of the V row.  Its 4 x 8 elements lie in four groups, which it shares with three other
// threads: each of the four finds the scale and the reciprocal of one group and hands them out.
// `early`: the caller's rows were complete before the kernel in front could start.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) append_kv4_kernel(Dev d, int total, int layer0,
                                                             const T* k, const T* v, int early) {
  constexpr int KC = D / 16, HALF = D / 2, NG = D / GROUP;
  static_assert(GROUP == 32 && KC % 4 == 0, "four threads of eight dims share a scale");
  const int H = d.kv_heads;
  const int64_t idx = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  const int c = (int)(idx % KC);
  const int64_t row = idx / KC;
  const int g = (int)(row / H), h = (int)(row % H);
  const bool in = g < total;
  if (!early) pdl_wait();
  pdl_launch_dependents();
  Eight<T> ka = {}, kb = {}, va = {}, vb = {};
  if (in) {
    const size_t off = (((size_t)blockIdx.y * total + g) * H + h) * D + c * 8;
    ka.load(k + off);
    kb.load(k + off + HALF);
    va.load(v + off);
    vb.load(v + off + HALF);
  }
  pdl_wait();
  // (Nothing to do where the plan kernel failed: error recorded.  All threads stay for the
  // shuffles.)
  const bool live = in && g < d.g->total_tokens;
  const int gs = live ? d.tok_slot[g] : 0, pos = live ? d.tok_pos[g] : 0;
  float x1[8], x2[8], ya[8], yb[8], wa[8], wb[8];
  ka.get(x1);
  kb.get(x2);
  va.get(wa);
  vb.get(wb);
  const float4* t4 = reinterpret_cast<const float4*>(d.rope + (size_t)pos * HALF + c * 8);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float4 cs = t4[e / 2];
    turn_pair(x1[e], x2[e], make_float2(cs.x, cs.y), ya[e], yb[e]);
    turn_pair(x1[e + 1], x2[e + 1], make_float2(cs.z, cs.w), ya[e + 1], yb[e + 1]);
  }
  // Largest |x| of group i to the quad's thread i.
  const int own = c % 4, lane = threadIdx.x & 31;
  const uint32_t most[4] = {most_of(ya), most_of(yb), most_of(wa), most_of(wb)};
  uint32_t mx;
  {
    const bool b1 = own & 2, b0 = own & 1;
    const uint32_t p = max(b1 ? most[2] : most[0], __shfl_xor_sync(FULL, b1 ? most[0] : most[2], 2));
    const uint32_t r = max(b1 ? most[3] : most[1], __shfl_xor_sync(FULL, b1 ? most[1] : most[3], 2));
    mx = max(b0 ? r : p, __shfl_xor_sync(FULL, b0 ? p : r, 1));
  }
  const float s = scale_of(mx);
  const Divisor div(s);
  const bool passes = __any_sync(FULL, div.passes(mx));
  float inv[4], rest[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    inv[i] = __shfl_sync(FULL, div.inv, lane & ~3 | i);
    rest[i] = __shfl_sync(FULL, div.rest, lane & ~3 | i);
  }
  if (passes) {
    hold_codes(ya, __shfl_sync(FULL, div.by, lane & ~3));
    hold_codes(yb, __shfl_sync(FULL, div.by, lane & ~3 | 1));
    hold_codes(wa, __shfl_sync(FULL, div.by, lane & ~3 | 2));
    hold_codes(wb, __shfl_sync(FULL, div.by, lane & ~3 | 3));
  }
  if (!live) return;
  const int page = gs / PS, slot = gs % PS, layer = layer0 + blockIdx.y;
  uint8_t* kt = d.pool + tile_at(D, d.layers, H, page, layer, h, 0);
  uint8_t* vt = kt + tile_bytes(D);
  *reinterpret_cast<uint32_t*>(kt + k_codes(D, slot, 8 * c)) = codes_of(ya, inv[0], rest[0]);
  *reinterpret_cast<uint32_t*>(kt + k_codes(D, slot, HALF + 8 * c)) = codes_of(yb, inv[1], rest[1]);
  *reinterpret_cast<uint32_t*>(vt + v_codes(D, slot, 8 * c)) = codes_of(wa, inv[2], rest[2]);
  *reinterpret_cast<uint32_t*>(vt + v_codes(D, slot, HALF + 8 * c)) = codes_of(wb, inv[3], rest[3]);
  const int group = c / 4 + (own & 1) * (NG / 2);
  const int at = own & 2 ? tile_bytes(D) + v_scale(D, slot, group) : k_scale(D, slot, group);
  *reinterpret_cast<__half*>(kt + at) = stored_scale(s);
}

// Survivors of an eviction (the move list of evict_plan_kernel), every layer, K and V, and head.
// Eight threads move a row: piece p of D / 16 bytes each, the first D / 32 a scale too.
template <int D>
__global__ void __launch_bounds__(THREADS) evict_copy_kv4_kernel(Dev d) {
  pdl_wait();
  pdl_launch_dependents();
  const int n_moves = d.g->n_moves, rows = d.layers * d.kv_heads * 2;
  const int64_t total = (int64_t)n_moves * rows * 8;
  for (int64_t u = (int64_t)blockIdx.x * THREADS + threadIdx.x; u < total;
       u += (int64_t)gridDim.x * THREADS) {
    const int p = (int)(u % 8);
    const int r = (int)(u / 8 % rows), m = (int)(u / 8 / rows);
    const int kv = r % 2, h = r / 2 % d.kv_heads, layer = r / 2 / d.kv_heads;
    const int2 mv = d.moves[m];
    const int ss = mv.x % PS, ds = mv.y % PS;
    const uint8_t* src = d.pool + tile_at(D, d.layers, d.kv_heads, mv.x / PS, layer, h, kv);
    uint8_t* dst = d.pool + tile_at(D, d.layers, d.kv_heads, mv.y / PS, layer, h, kv);
    const int so = kv ? v_piece(D, ss, p) : k_piece(D, ss, p);
    const int to = kv ? v_piece(D, ds, p) : k_piece(D, ds, p);
    if constexpr (D == 128)
      *reinterpret_cast<uint2*>(dst + to) = *reinterpret_cast<const uint2*>(src + so);
    else
      *reinterpret_cast<uint32_t*>(dst + to) = *reinterpret_cast<const uint32_t*>(src + so);
    if (p < D / GROUP) {
      const int sc = kv ? v_scale(D, ss, p) : k_scale(D, ss, p);
      const int tc = kv ? v_scale(D, ds, p) : k_scale(D, ds, p);
      *reinterpret_cast<uint16_t*>(dst + tc) = *reinterpret_cast<const uint16_t*>(src + sc);
    }
  }
}

// 8 elements from dim dd of a stored row, as they are given back.
template <typename T, int D, bool KV4>
__device__ inline void copy_eight(const Dev& d, int gs, int layer, int kv, int h, int dd, T* to) {
  const int page = gs / PS, slot = gs % PS;
  if constexpr (KV4) {
    const uint8_t* tile = d.pool + tile_at(D, d.layers, d.kv_heads, page, layer, h, kv);
    const uint32_t w =
        *reinterpret_cast<const uint32_t*>(tile + (kv ? v_codes(D, slot, dd) : k_codes(D, slot, dd)));
    const __half m = *reinterpret_cast<const __half*>(
        tile + (kv ? v_scale(D, slot, dd / GROUP) : k_scale(D, slot, dd / GROUP)));
    float f[8];
    values_of(w, m, f);
    Eight<T>::store(to, f);
  } else {
    const uint4* src = reinterpret_cast<const uint4*>(
        reinterpret_cast<const T*>(d.pool) + pool_offset_elems(d, page, layer, kv, h, slot) + dd);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(to)[i] = src[i];
  }
}

// One warp's share of a row: all heads of K and of V, `row` their place in the outputs.
template <typename T, int D, bool KV4>
__device__ inline void read_row(const Dev& d, int gs, int layer, size_t row, T* k_out, T* v_out,
                                int lane) {
  const int chunks = d.kv_heads * (D / 8);
  for (int i = lane; i < 2 * chunks; i += 32) {
    const int kv = i >= chunks, j = kv ? i - chunks : i;
    T* to = (kv ? v_out : k_out) + (row * chunks + j) * 8;
    if (gs >= 0) {
      copy_eight<T, D, KV4>(d, gs, layer, kv, j / (D / 8), j % (D / 8) * 8, to);
    } else {
      const float zero[8] = {};
      Eight<T>::store(to, zero);
    }
  }
}

// Rows of the listed sessions (kvc_read_kv): output row r of layer blockIdx.y belongs to the
// session i with cu[i] <= r < cu[i + 1] and is its retained position first[i] + r - cu[i]; zeros
// where it holds no such position.
template <typename T, int D, bool KV4, int N>
__global__ void __launch_bounds__(THREADS) read_kv_kernel(Dev d, ReadArgsT<N> a, int layer0,
                                                          T* k_out, T* v_out,
                                                          int64_t* resident_out) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  if (resident_out != nullptr && blockIdx.x == 0 && blockIdx.y == 0)
    for (int i = threadIdx.x; i < a.n_seq; i += THREADS) {
      const SessState& st = d.sess[a.sessions[i]];
      resident_out[i] = (int64_t)st.n_hist + st.n_live;
    }
  const int64_t n_warps = (int64_t)gridDim.x * (THREADS / 32);
  for (int64_t r = ((int64_t)blockIdx.x * THREADS + threadIdx.x) / 32; r < a.total; r += n_warps) {
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.cu[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    const int sid = a.sessions[lo];
    const SessState& st = d.sess[sid];
    const int64_t i = a.first[lo] + (r - a.cu[lo]);
    const size_t pt = (size_t)sid * d.max_pages_per_session;
    int gs = -1;
    if (i < st.n_hist) {
      gs = d.hist_pt[pt + i / PS] * PS + (int)(i % PS);
    } else if (i < (int64_t)st.n_hist + st.n_live) {
      const int j = st.live_head + (int)(i - st.n_hist);
      gs = d.live_pt[pt + j / PS] * PS + j % PS;
    }
    read_row<T, D, KV4>(d, gs, layer0 + blockIdx.y, (size_t)blockIdx.y * a.total + r, k_out, v_out,
                        lane);
  }
}

// The transcript's rows (part 1 has left their slots in the move list): [L][cap][Hkv][D].
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) transcript_copy_kv4_kernel(Dev d, int cap, T* k_out,
                                                                      T* v_out) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = d.g->n_moves, lane = threadIdx.x & 31;
  const int64_t total = (int64_t)n * d.layers, n_warps = (int64_t)gridDim.x * (THREADS / 32);
  for (int64_t u = ((int64_t)blockIdx.x * THREADS + threadIdx.x) / 32; u < total; u += n_warps) {
    const int layer = (int)(u / n), i = (int)(u % n);
    read_row<T, D, true>(d, d.moves[i].x, layer, (size_t)layer * cap + i, k_out, v_out, lane);
  }
}

template <typename T, int D, bool KV4, int N>
cudaError_t launch_read(const Dev& d, const ReadArgsT<N>& a, int layer0, int n_layers, void* k_out,
                        void* v_out, int64_t* resident_out, int sms, cudaStream_t s) {
  // As many warps as rows, up to a few CTAs per SM; one CTA for the counts alone.
  const int rows = (a.total + THREADS / 32 - 1) / (THREADS / 32);
  const dim3 grid(max(1, min(rows, sms * 8)), a.total > 0 ? n_layers : 1);
  return launch_ex(&read_kv_kernel<T, D, KV4, N>, grid, dim3(THREADS), 0, s, true, d, a, layer0,
                   static_cast<T*>(k_out), static_cast<T*>(v_out), resident_out);
}

template <int N>
cudaError_t launch_read_of(const Dev& d, bool kv4, const ReadArgsT<N>& a, int layer0, int n_layers,
                           void* k_out, void* v_out, int64_t* res, int sms, cudaStream_t s) {
  using B = __nv_bfloat16;
  if (d.esz == 2)
    return kv4 ? launch_read<B, 128, true, N>(d, a, layer0, n_layers, k_out, v_out, res, sms, s)
               : launch_read<B, 128, false, N>(d, a, layer0, n_layers, k_out, v_out, res, sms, s);
  return kv4 ? launch_read<float, 64, true, N>(d, a, layer0, n_layers, k_out, v_out, res, sms, s)
             : launch_read<float, 64, false, N>(d, a, layer0, n_layers, k_out, v_out, res, sms, s);
}

}  // namespace

cudaError_t launch_append_layers_kv4(const Dev& d, int total, int layer0, int n_layers,
                                     const void* k, const void* v, bool after_plan,
                                     cudaStream_t s) {
  const int64_t threads = (int64_t)total * d.kv_heads * (d.head_dim / 16);
  const dim3 grid((unsigned)((threads + THREADS - 1) / THREADS), n_layers);
  if (d.esz == 2)
    return launch_ex(&append_kv4_kernel<__nv_bfloat16, 128>, grid, dim3(THREADS), 0, s, true, d,
                     total, layer0, static_cast<const __nv_bfloat16*>(k),
                     static_cast<const __nv_bfloat16*>(v), (int)after_plan);
  return launch_ex(&append_kv4_kernel<float, 64>, grid, dim3(THREADS), 0, s, true, d, total, layer0,
                   static_cast<const float*>(k), static_cast<const float*>(v), (int)after_plan);
}

cudaError_t launch_evict_copy_kv4(const Dev& d, int sms, cudaStream_t s) {
  return launch_ex(d.head_dim == 128 ? &evict_copy_kv4_kernel<128> : &evict_copy_kv4_kernel<64>,
                   dim3(sms * 4), dim3(THREADS), 0, s, true, d);
}

cudaError_t launch_transcript_copy_kv4(const Dev& d, int cap, void* k_out, void* v_out, int sms,
                                       cudaStream_t s) {
  if (d.esz == 2)
    return launch_ex(&transcript_copy_kv4_kernel<__nv_bfloat16, 128>, dim3(sms * 4), dim3(THREADS),
                     0, s, true, d, cap, static_cast<__nv_bfloat16*>(k_out),
                     static_cast<__nv_bfloat16*>(v_out));
  return launch_ex(&transcript_copy_kv4_kernel<float, 64>, dim3(sms * 4), dim3(THREADS), 0, s, true,
                   d, cap, static_cast<float*>(k_out), static_cast<float*>(v_out));
}

cudaError_t launch_read_kv(const Dev& d, bool kv4, const ReadArgs& a, int layer0, int n_layers,
                           void* k_out, void* v_out, int64_t* resident_out, int sms,
                           cudaStream_t s) {
  if (a.n_seq > FEW)
    return launch_read_of(d, kv4, a, layer0, n_layers, k_out, v_out, resident_out, sms, s);
  ReadArgsT<FEW> few;
  few.n_seq = a.n_seq;
  few.total = a.total;
  for (int i = 0; i < a.n_seq; ++i) {
    few.sessions[i] = a.sessions[i];
    few.first[i] = a.first[i];
  }
  for (int i = 0; i <= a.n_seq; ++i) few.cu[i] = a.cu[i];
  return launch_read_of(d, kv4, few, layer0, n_layers, k_out, v_out, resident_out, sms, s);
}

}  // namespace kvc
