// Rows held in 4 bits (KVC_KV4): the write (rotation and quantisation in one pass), the move of
// survivors of an eviction, and the read-back of rows of either kind of cache in the element type.
//
// All move bytes.  A layer of 5,500 bfloat16 positions (8 heads) is 30 MB, 4.4 us at the copy rate, and
// its write takes 9.5 us behind another one: 12 instructions an element (rotation, largest |x|, two
// products, a sum and a shifted add a code) in one wave of CTAs whose loads are one block of rows ahead
// (17 us with a division a code; 11 us a head a thread, 18 instructions).  Its read-back, 16 layers in a
// launch, takes 74 us for 460 MB (6.2 TB/s).  A token or two take what a launch takes, 2.6 us.
// A whole chunk's write is one launch for all layers: 60 us for 64 sessions of 17 tokens in 32 layers
// with its plan (10 us of it), where 183 MB take 27; 122 us for 5,490 rows in 16 layers (68).  The same
// read-back of rows in the element type: 130 us for 720 MB (5.5 TB/s).
//
// An eviction's copy moves 8 bytes (D = 64: 4) a thread, which finds its row by divisions: 49 us for 4,768
// survivors in 8 layers, whose 88 MB would take 13; 334 us for 33,900 (92).  The transcript's rows take
// 6.4 us behind the 5.5 of finding them, 565 of 8 layers (3.5 us of bytes).
#include "kvc_kv4.cuh"

namespace kvc {

namespace {

using namespace kv4;

constexpr int THREADS = 256;
constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int APPEND_CTAS = 2;  // CTAs of the write per SM: what its 105 registers let run at once

// K rotated at its position and V, quantised into the page slots of the plan kernel.  Input
// [L][total][Hkv][D]; blockIdx.y is the input layer, cache layer layer0 + blockIdx.y.  The first
// half of the CTAs takes K, the other V (in turn they would leave every second SM the rotations), each
// several blocks of rows: the next block's rows and slots are on their way while one is worked on.
// A thread takes 8 dims of the first half of a row and their rotate-half partners, of two heads of a
// token, which share slot and rotation.  Its 4 x 8 elements lie in four groups, which it shares with three
// other threads: each of the four finds the scale and the reciprocal of one and hands them out.
// Before the kernel in front is complete, `early` launches read the caller's rows (complete before
// that kernel could start), `planned` ones the slots (the plan kernel was complete by then).
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) append_kv4_kernel(Dev d, int total, int layer0,
                                                             const T* k, const T* v, bool early,
                                                             bool planned) {
  constexpr int KC = D / 16, HALF = D / 2, NG = D / GROUP;
  static_assert(GROUP == 32 && KC % 4 == 0, "four threads of eight dims share a scale");
  const int H = d.kv_heads, HP = (H + 1) / 2;
  const int n_cta = gridDim.x >> 1, kv = (int)blockIdx.x >= n_cta, layer = layer0 + blockIdx.y;
  const T* from = (kv ? v : k) + (size_t)blockIdx.y * total * H * D;
  // (A call has 2^20 tokens at most: rows count in 32 bits.)  A row's token and head are
  // carried along, not divided out.
  const int step = n_cta * (THREADS / KC), n = total * HP;
  const int c = threadIdx.x % KC, lane = threadIdx.x & 31, step_g = step / HP, step_h = step % HP;
  struct Block {
    Eight<T> x[2][2];  // [head][half]
    int g, h, gs, pos;
    bool live;
  };
  int n_tok = 0;
  auto ask_rows = [&](Block& x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x.x[i][0] = {};
      x.x[i][1] = {};
      if (x.g >= total || x.h + i * HP >= H) continue;
      const T* p = from + ((size_t)x.g * H + x.h + i * HP) * D + c * 8;
      x.x[i][0].load(p);
      x.x[i][1].load(p + HALF);
    }
  };
  auto ask_slots = [&](Block& x) {
    // (Nothing to do where the plan kernel failed: error recorded.  All threads stay for the
    // shuffles.)
    x.live = x.g < n_tok;
    x.gs = x.live ? d.tok_slot[x.g] : 0;
    x.pos = x.live && !kv ? d.tok_pos[x.g] : 0;
  };
  int first = ((int)blockIdx.x - kv * n_cta) * (THREADS / KC);
  Block cur, next;
  cur.g = (first + (int)threadIdx.x / KC) / HP;
  cur.h = (first + (int)threadIdx.x / KC) % HP;
  if (early) {
    ask_rows(cur);
    pdl_launch_dependents();
  }
  if (planned) {
    n_tok = min(total, d.g->total_tokens);
    ask_slots(cur);
  }
  pdl_wait();
  if (!planned) {
    n_tok = min(total, d.g->total_tokens);
    ask_slots(cur);
  }
  if (!early) {
    pdl_launch_dependents();
    ask_rows(cur);
  }
  for (; first < n; first += step, cur = next) {
    float x[2][2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      cur.x[i][0].get(x[i][0]);
      cur.x[i][1].get(x[i][1]);
    }
    next.g = cur.g + step_g;
    next.h = cur.h + step_h;
    if (next.h >= HP) {
      next.h -= HP;
      ++next.g;
    }
    if (kv == 0) {
      const float4* t4 = reinterpret_cast<const float4*>(d.rope + (size_t)cur.pos * HALF + c * 8);
      float4 cs[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) cs[e] = t4[e];
      ask_rows(next);
      ask_slots(next);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 t = e % 2 ? make_float2(cs[e / 2].z, cs[e / 2].w) : make_float2(cs[e / 2].x, cs[e / 2].y);
          float y0, y1;
          turn_pair(x[i][0][e], x[i][1][e], t, y0, y1);
          x[i][0][e] = y0;
          x[i][1][e] = y1;
        }
    } else {
      ask_rows(next);
      ask_slots(next);
    }
    // Largest |x| of group i (head i / 2, half i % 2) to thread i of the four.
    const int own = lane & 3;
    uint32_t mx;
    {
      const uint32_t m[4] = {most_of(x[0][0]), most_of(x[0][1]), most_of(x[1][0]), most_of(x[1][1])};
      const bool b1 = own & 2, b0 = own & 1;
      const uint32_t p = max(b1 ? m[2] : m[0], __shfl_xor_sync(FULL, b1 ? m[0] : m[2], 2));
      const uint32_t r = max(b1 ? m[3] : m[1], __shfl_xor_sync(FULL, b1 ? m[1] : m[3], 2));
      mx = max(b0 ? r : p, __shfl_xor_sync(FULL, b0 ? p : r, 1));
    }
    const float s = scale_of(mx);
    const Divisor div(s);
    if (__any_sync(FULL, div.passes(mx))) {
#pragma unroll
      for (int i = 0; i < 4; ++i) hold_codes(x[i / 2][i % 2], __shfl_sync(FULL, div.by, lane & ~3 | i));
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = codes_of(x[i / 2][i % 2], __shfl_sync(FULL, div.inv, lane & ~3 | i),
                      __shfl_sync(FULL, div.rest, lane & ~3 | i));
    if (!cur.live) continue;
    const int page = cur.gs / PS, slot = cur.gs % PS;
    uint8_t* tile = d.pool + tile_at(D, d.layers, H, page, layer, cur.h, kv);
    const int at[2] = {kv ? v_codes(D, slot, 8 * c) : k_codes(D, slot, 8 * c),
                       kv ? v_codes(D, slot, HALF + 8 * c) : k_codes(D, slot, HALF + 8 * c)};
    const int to_second = HP * 2 * (int)tile_bytes(D);
    const bool second = cur.h + HP < H;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < 2 || second)
        *reinterpret_cast<uint32_t*>(tile + (i / 2) * to_second + at[i % 2]) = w[i];
    if (own < 2 || second) {
      const int group = c / 4 + (own & 1) * (NG / 2);
      *reinterpret_cast<__half*>(tile + (own >> 1) * to_second +
                                 (kv ? v_scale(D, slot, group) : k_scale(D, slot, group))) = stored_scale(s);
    }
  }
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

// 8 elements as they are given back, from their word and scale.  bfloat16: 128 + code + 8 is its pattern
// 0x4300 | nibble, so the code comes exactly and the product with the scale (7 bits, exact too) is
// rounded once.
template <typename T>
__device__ inline void give_eight(uint32_t w, __half m, T* to) {
  if constexpr (sizeof(T) == 2) {
    const __nv_bfloat162 s = __float2bfloat162_rn(__half2float(m) * 16.f), k136 = __float2bfloat162_rn(136.f);
    uint32_t v[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {  // dims p and p + 4
      const uint32_t u = and_or(w >> (4 * p), 0x000F000Fu, 0x43004300u);
      const __nv_bfloat162 y = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), k136), s);
      v[p] = *reinterpret_cast<const uint32_t*>(&y);
    }
    *reinterpret_cast<uint4*>(to) =
        make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410),
                   __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
  } else {
    float f[8];
    values_of(w, m, f);
    Eight<T>::store(to, f);
  }
}

// One warp's share of a row: all heads of K and of V, `row` their place in the outputs.  A lane keeps
// its 8 dims and takes every STEP-th head, four of them on their way at a time.
template <typename T, int D, bool KV4>
__device__ inline void read_row(const Dev& d, int gs, int layer, size_t row, T* k_out, T* v_out,
                                int lane) {
  constexpr int CHUNKS = D / 8, STEP = 32 / CHUNKS, BATCH = 4;
  const int H = d.kv_heads, dd = lane % CHUNKS * 8, h0 = lane / CHUNKS;
  k_out += row * H * D + dd;
  v_out += row * H * D + dd;
  if (gs < 0) {
    const float zero[8] = {};
    for (int h = h0; h < H; h += STEP) {
      Eight<T>::store(k_out + h * D, zero);
      Eight<T>::store(v_out + h * D, zero);
    }
    return;
  }
  const int page = gs / PS, slot = gs % PS;
  if constexpr (KV4) {
    const uint8_t* tile = d.pool + tile_at(D, d.layers, H, page, layer, 0, 0);
    const int TB = (int)tile_bytes(D);
    const int kc = k_codes(D, slot, dd), ks = k_scale(D, slot, dd / GROUP);
    const int vc = TB + v_codes(D, slot, dd), vs = TB + v_scale(D, slot, dd / GROUP);
    for (int h = h0; h < H; h += BATCH * STEP) {
      uint32_t w[BATCH][2];
      __half m[BATCH][2];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const uint8_t* at = tile + (size_t)min(h + u * STEP, H - 1) * 2 * TB;
        w[u][0] = *reinterpret_cast<const uint32_t*>(at + kc);
        w[u][1] = *reinterpret_cast<const uint32_t*>(at + vc);
        m[u][0] = *reinterpret_cast<const __half*>(at + ks);
        m[u][1] = *reinterpret_cast<const __half*>(at + vs);
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        if (h + u * STEP >= H) break;
        give_eight(w[u][0], m[u][0], k_out + (h + u * STEP) * D);
        give_eight(w[u][1], m[u][1], v_out + (h + u * STEP) * D);
      }
    }
  } else {
    for (int h = h0; h < H; h += STEP) {
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint4* src = reinterpret_cast<const uint4*>(
            reinterpret_cast<const T*>(d.pool) + pool_offset_elems(d, page, layer, kv, h, slot) + dd);
        uint4* to = reinterpret_cast<uint4*>((kv ? v_out : k_out) + h * D);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) to[i] = src[i];
      }
    }
  }
}

// Rows of the listed sessions (kvc_read_kv): output row r of a layer belongs to the session i with
// cu[i] <= r < cu[i + 1] and is its retained position first[i] + r - cu[i]; zeros where it holds no
// such position.  A warp finds a row's slot once and gives it back for `per` layers, blockIdx.y per on.
template <typename T, int D, bool KV4, int N>
__global__ void __launch_bounds__(THREADS) read_kv_kernel(Dev d, ReadArgsT<N> a, int layer0,
                                                          int n_layers, int per, T* k_out, T* v_out,
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
    const int end = min(n_layers, ((int)blockIdx.y + 1) * per);
    for (int l = blockIdx.y * per; l < end; ++l)
      read_row<T, D, KV4>(d, gs, layer0 + l, (size_t)l * a.total + r, k_out, v_out, lane);
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
  // A warp to a row, in up to a few CTAs per SM, and to as many layers as leave two rounds of them; one
  // CTA for the counts alone.
  const int rows = (a.total + THREADS / 32 - 1) / (THREADS / 32);
  const int per = (int)max((int64_t)1, min((int64_t)n_layers, (int64_t)rows * n_layers / (sms * 16)));
  const dim3 grid(max(1, min(rows, sms * 8)), a.total > 0 ? (n_layers + per - 1) / per : 1);
  return launch_ex(&read_kv_kernel<T, D, KV4, N>, grid, dim3(THREADS), 0, s, true, d, a, layer0,
                   n_layers, per, static_cast<T*>(k_out), static_cast<T*>(v_out), resident_out);
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
                                     const void* k, const void* v, bool early, bool planned, int sms,
                                     cudaStream_t s) {
  const int rows = THREADS / (d.head_dim / 16);  // of a block
  const int blocks = (total * ((d.kv_heads + 1) / 2) + rows - 1) / rows;
  // Two blocks of rows a CTA or more where there are enough of them.
  const int per_layer = max(1, sms * APPEND_CTAS / 2 / n_layers);
  const dim3 grid(2 * (unsigned)min(blocks, per_layer), n_layers);
  if (d.esz == 2)
    return launch_ex(&append_kv4_kernel<__nv_bfloat16, 128>, grid, dim3(THREADS), 0, s, true, d,
                     total, layer0, static_cast<const __nv_bfloat16*>(k),
                     static_cast<const __nv_bfloat16*>(v), early, planned);
  return launch_ex(&append_kv4_kernel<float, 64>, grid, dim3(THREADS), 0, s, true, d, total, layer0,
                   static_cast<const float*>(k), static_cast<const float*>(v), early, planned);
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
