// Eviction by weight (kvc_evict_weighted): of each listed session's candidates (types in `kinds`,
// positions in [sink, pos_next - recent)) the lightest go, the oldest of equal ones first, until
// `keep` positions are left or no candidate is.
//
// Unlike the rule of Sec. 3.3 this may drop any retained position, the compacted ones of earlier
// evictions too.  The survivors are packed in place.  Count the slots of a session's page sequence
// (compacted pages, then the live pages that the call consumes whole) one after the other: survivor i
// goes to slot i, which never lies behind the slot it comes from, so rows moved in ascending order
// overwrite only slots that were read before.  The live prefix up to the last position that goes is
// consumed; the rest of the live region keeps its slots, and with them its tail's offset in a page,
// which the host knows.  The consumed pages become compacted ones; at most one page a session is new
// (where survivors reach into the page that the rest of the live region starts in).
//
//   weigh_select_kernel  a CTA per session: keys that order as the weights do, the key of the last
//                        one to go by four 8-bit radix passes; the last CTA allocates
//   weigh_apply_kernel   a CTA per session: moves, tags, page lists, state, mask
//   weigh_copy_kernel    a CTA per session and (layer, K or V, head): the rows, ascending
//
// kvc_evict takes this way too, with the rule of its policy in place of the weights, for sessions that were
// thinned out by weight: what it may drop then lies among the compacted positions as well.
//
// Bound by the rows that move, each read and written once.  4,099 positions of 32 layers thinned out to
// 2,048: select 13-19 us, apply 9-13, copy 92 (537 MB, 5.8 TB/s); 16 sessions of 16 layers to 700 each:
// copy 235 us.  Select and apply are one CTA's latencies a session: radix passes of 8 bits over keys in
// shared memory (four passes; a sort would move the positions too, which need not be in order).
#include <climits>
#include <type_traits>

#include "kvc_kv4.h"
#include "kvc_meta_common.cuh"

namespace kvc {

namespace {

constexpr uint32_t NO_KEY = 0xFFFFFFFFu;  // of a position that may not go
constexpr int CACHED_KEYS = 11 * 1024;    // keys of a session held in shared memory, at most
constexpr int BINS = 256;

// Sortable bits of a weight: ascending as numbers, -0 as 0, NaN as -infinity.
__device__ inline uint32_t weight_key(float w) {
  w = isnan(w) ? -INFINITY : w + 0.f;
  const uint32_t u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Slot in the pool of retained position j (rows of the session's page lists).
__device__ inline int retained_slot(const SessState& st, const int32_t* hrow, const int32_t* lrow,
                                    int j) {
  if (j < st.n_hist) return hrow[j / PS] * PS + j % PS;
  const int s = st.live_head + j - st.n_hist;
  return lrow[s / PS] * PS + s % PS;
}

// Whether position j (key k) goes.
__device__ inline bool goes(const WeighPlan& p, uint32_t k, int j) {
  return k < p.key || (k == p.key && j <= p.tie_last);
}

// First entry of session q's list: the sessions before it have as many entries as positions.
__device__ inline int64_t list_base(const Dev& d, const int32_t* sessions, int q, int* s_warp) {
  int n = 0;
  if ((int)threadIdx.x < q) {
    const SessState& st = d.sess[sessions[threadIdx.x]];
    n = st.n_hist + st.n_live;
  }
  int total;
  block_exclusive_scan(n, &total, s_warp);
  return total;  // (all positions of a pool are fewer than 2^31)
}

// Whether kvc_evict may drop a position: by the rule of Sec. 3.3 and its position-granular variant, or by the
// sink + recent variant.
__device__ inline bool rule_takes(const Dev& d, const SessState& st, int type, int unit, int pos) {
  if (d.policy == KVC_POLICY_SINK_RECENT) return pos >= d.sink && pos < st.pos_next - d.recent;
  return unit >= 0 && unit <= st.unit_cur - d.window && (type == KVC_ACOUSTIC || type == KVC_ASR_DELIM);
}

// RULE: by the context's policy instead of weights, kinds and counts to keep; of the candidates, in position
// order, the first ones go: as many as the budget wants, and the rest of the last one's unit (KVC_POLICY_UNIT).
template <int N, bool RULE>
__global__ void __launch_bounds__(META_THREADS) weigh_select_kernel(Dev d, WeighDev w,
                                                                    WeighArgsT<N> a,
                                                                    const float* weights,
                                                                    int64_t* used_out) {
  extern __shared__ uint32_t s_keys[];
  __shared__ int s_warp[33];
  __shared__ int s_hist[BINS];
  __shared__ int s_found[4];
  __shared__ int s_last;
  const int tid = threadIdx.x, q = blockIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  const int sid = a.sessions[q];
  const SessState st = d.sess[sid];
  const int32_t* hrow = d.hist_pt + (size_t)sid * d.max_pages_per_session;
  const int32_t* lrow = d.live_pt + (size_t)sid * d.max_pages_per_session;
  const int n = st.n_hist + st.n_live;
  const int64_t base = list_base(d, a.sessions, q, s_warp);
  uint2* list = w.list + base;
  const float* heavy = weights + (size_t)sid * d.max_positions;
  auto key_at = [&](int j) { return j < CACHED_KEYS ? s_keys[j] : list[j].x; };

  int n_cand = 0;
  for (int j = tid; j < n; j += META_THREADS) {
    const int gs = retained_slot(st, hrow, lrow, j);
    const int type = d.meta_type[gs], pos = d.meta_pos[gs];
    const bool cand = RULE ? rule_takes(d, st, type, d.meta_unit[gs], pos)
                           : type < 32 && (a.kinds >> type & 1) && pos >= a.sink && pos < st.pos_next - a.recent;
    const uint32_t k = !cand ? NO_KEY : RULE ? 0u : weight_key(heavy[pos]);
    list[j] = make_uint2(k, (uint32_t)gs);
    if (j < CACHED_KEYS) s_keys[j] = k;
    n_cand += cand;
  }
  int cands;
  block_exclusive_scan(n_cand, &cands, s_warp);
  int64_t over = n - a.keep[q];
  if (RULE) over = d.policy == KVC_POLICY_SINK_RECENT ? n : d.budget < 0 ? 0 : n - d.budget;
  int drop = (int)min(max((int64_t)0, over), (int64_t)cands);

  // Index of the rank-th position of a key.
  auto nth = [&](uint32_t key, int rank) {
    int seen = 0;
    for (int j0 = 0; j0 < n; j0 += META_THREADS) {
      const int j = j0 + tid;
      const int is = j < n && key_at(j) == key;
      int total;
      const int before = seen + block_exclusive_scan(is, &total, s_warp);
      if (is && before == rank - 1) s_found[3] = j;
      seen += total;
      if (seen >= rank) break;
    }
    __syncthreads();
    return s_found[3];
  };
  WeighPlan p = {};
  p.key = 0;
  p.tie_last = -1;
  if (drop > 0 && drop == cands) {
    p.key = NO_KEY;  // all that may
  } else if (RULE && drop > 0) {
    p.tie_last = nth(0, drop);
    if (d.policy == KVC_POLICY_UNIT) {
      const int unit = d.meta_unit[list[p.tie_last].y];
      int rest = 0, last = p.tie_last;
      for (int j = p.tie_last + 1 + tid; j < n; j += META_THREADS)
        if (key_at(j) == 0 && d.meta_unit[list[j].y] == unit) {
          ++rest;
          last = j;
        }
      int more;
      block_exclusive_scan(rest, &more, s_warp);
      drop += more;
      p.tie_last = block_max(last, s_warp);
    }
  } else if (drop > 0) {
    // The drop-th smallest key, digit by digit: `rank` of it among the keys that share the digits
    // found so far.
    uint32_t prefix = 0;
    int rank = drop, equal = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < BINS) s_hist[tid] = 0;
      __syncthreads();
      for (int j = tid; j < n; j += META_THREADS) {
        const uint32_t k = key_at(j);
        if (k != NO_KEY && (shift == 24 || k >> (shift + 8) == prefix))
          atomicAdd(&s_hist[k >> shift & 255], 1);
      }
      __syncthreads();
      const int mine = tid < BINS ? s_hist[tid] : 0;
      int total;
      const int before = block_exclusive_scan(mine, &total, s_warp);
      if (tid < BINS && before < rank && rank <= before + mine) {
        s_found[0] = tid;
        s_found[1] = before;
        s_found[2] = mine;
      }
      __syncthreads();
      prefix = prefix << 8 | (uint32_t)s_found[0];
      rank -= s_found[1];
      equal = s_found[2];
      __syncthreads();
    }
    p.key = prefix;
    // Of the keys equal to it the first `rank` go.
    p.tie_last = n;
    if (rank < equal) p.tie_last = nth(prefix, rank);
  }
  p.drop = drop;
  // The first and the last position that go.
  int first = INT_MAX, last = -1;
  if (drop > 0)
    for (int j = tid; j < n; j += META_THREADS)
      if (goes(p, key_at(j), j)) {
        first = min(first, j);
        last = max(last, j);
      }
  last = block_max(last, s_warp);
  first = -block_max(first == INT_MAX ? -INT_MAX : -first, s_warp);
  if (tid == 0) {
    p.list_at = base;
    p.first = drop > 0 ? first : n;
    p.end = max(0, last + 1 - st.n_hist);
    p.stay = drop > 0 ? st.n_hist + p.end - drop : st.n_hist;
    const int whole = (st.live_head + p.end) / PS;  // live pages consumed whole
    p.pages = (p.stay + PS - 1) / PS;
    p.taken = max(0, min(whole, p.pages - st.n_hist_pages));
    p.extra = p.pages > st.n_hist_pages + whole ? 1 : 0;
    p.freed = max(0, st.n_hist_pages + whole - p.pages);
    w.plan[q] = p;
  }
  __syncthreads();
  if (tid == 0) s_last = arrive_acq_rel(w.count, a.n_seq);
  __syncthreads();
  if (!s_last) return;

  // The last CTA: new pages, for all sessions or for none.
  int extra = 0, freed = 0, bad = 0;
  if (tid < a.n_seq) {
    const WeighPlan& o = w.plan[tid];
    extra = __ldcg(&o.extra);
    freed = __ldcg(&o.freed);
    bad = __ldcg(&o.pages) > d.max_pages_per_session && __ldcg(&o.drop) > 0;
  }
  bad = __syncthreads_or(bad);
  int total_extra, total_freed;
  const int off = block_exclusive_scan(extra, &total_extra, s_warp);
  block_exclusive_scan(freed, &total_freed, s_warp);
  int err = bad ? KVC_DERR_PAGE_TABLE : 0;
  if (!err && (total_extra > d.max_alloc || !block_alloc_lowest(d, total_extra, s_warp)))
    err = KVC_DERR_POOL;
  __syncthreads();
  if (tid < a.n_seq) {
    w.plan[tid].ok = err == 0;
    if (extra && !err) w.plan[tid].extra_page = d.alloc_list[off];
  }
  if (tid == 0) {
    if (err) set_error(d, err);
    else d.g->pages_used += total_extra - total_freed;
    *used_out = d.g->pages_used;
    *w.count = 0;
  }
}

constexpr int PER = 4;  // positions of a thread in a step of the packing

template <int N>
__global__ void __launch_bounds__(META_THREADS) weigh_apply_kernel(Dev d, WeighDev w,
                                                                   WeighArgsT<N> a,
                                                                   int64_t* resident_out,
                                                                   uint8_t* kept) {
  __shared__ int s_warp[33];
  const int tid = threadIdx.x, q = blockIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  const WeighPlan p = w.plan[q];
  const int sid = a.sessions[q];
  const SessState st = d.sess[sid];
  int32_t* hrow = d.hist_pt + (size_t)sid * d.max_pages_per_session;
  int32_t* lrow = d.live_pt + (size_t)sid * d.max_pages_per_session;
  if (!p.ok) {  // no session of the call changes
    if (tid == 0) w.plan[q].moves = 0;
    return;
  }
  uint2* list = w.list + p.list_at;
  const int n = st.n_hist + st.n_live, nhp = st.n_hist_pages;
  const int decided = p.drop > 0 ? st.n_hist + p.end : 0;
  uint8_t* mask = kept ? kept + (size_t)q * d.max_positions : nullptr;
  if (mask) {
    for (int i = tid; i < st.pos_next; i += META_THREADS) mask[i] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += META_THREADS)
      if (!goes(p, list[j].x, j)) mask[d.meta_pos[list[j].y]] = 1;
    __syncthreads();  // (the list and the tags change below)
  }
  // Where packing starts: everything before lies in its slot already, in a page that is taken over.
  const int whole = (st.live_head + p.end) / PS;              // live pages consumed whole
  const bool shifted = nhp * PS + st.live_head != st.n_hist;  // slots between the two regions
  const int start = min(min(p.first, (nhp + whole) * PS),
                        shifted && p.end > 0 ? min(st.n_hist, decided) : decided);
  int done = start;  // survivors placed
  for (int j0 = start; j0 < decided; j0 += PER * META_THREADS) {
    const int j = j0 + PER * tid;
    uint2 e[PER];
    bool stays[PER];
    int cnt = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      stays[u] = false;
      if (j + u < decided) {
        e[u] = list[j + u];
        stays[u] = !goes(p, e[u].x, j + u);
      }
      cnt += stays[u];
    }
    int pos[PER], unit[PER], type[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (stays[u]) {
        pos[u] = d.meta_pos[e[u].y];
        unit[u] = d.meta_unit[e[u].y];
        type[u] = d.meta_type[e[u].y];
      }
    int total;
    int i = done + block_exclusive_scan(cnt, &total, s_warp);  // (all of the step is read behind it)
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (stays[u]) {
        const int b = i / PS;
        const int page = b < nhp ? hrow[b] : b < nhp + p.taken ? lrow[b - nhp] : p.extra_page;
        const int to = page * PS + i % PS;
        d.meta_pos[to] = pos[u];
        d.meta_unit[to] = unit[u];
        d.meta_type[to] = (uint8_t)type[u];
        list[i - start] = make_uint2(e[u].y, (uint32_t)to);  // a move, for the rows
        ++i;
      }
    done += total;
    __syncthreads();
  }
  if (p.drop > 0) {
    // Page lists: consumed pages taken over or freed, the new one, compacted pages left over.
    for (int b = p.pages + tid; b < nhp; b += META_THREADS) free_page(d, hrow[b]);
    for (int b = tid; b < whole; b += META_THREADS) {
      if (b < p.taken) hrow[nhp + b] = lrow[b];
      else free_page(d, lrow[b]);
    }
    if (tid == 0 && p.extra) hrow[p.pages - 1] = p.extra_page;
    __syncthreads();
    const int remain = st.n_live_pages - whole;
    if (whole > 0)
      for (int b0 = 0; b0 < remain; b0 += META_THREADS) {
        const int b = b0 + tid;
        const int v = b < remain ? lrow[b + whole] : 0;
        __syncthreads();
        if (b < remain) lrow[b] = v;
        __syncthreads();
      }
    if (tid == 0) {
      SessState s1 = st;
      s1.n_hist = p.stay;
      s1.n_hist_pages = p.pages;
      s1.live_head = st.live_head + p.end - whole * PS;
      s1.n_live = st.n_live - p.end;
      s1.n_live_pages = remain;
      s1.n_evicted = st.n_evicted + p.drop;
      d.sess[sid] = s1;
    }
  }
  if (tid == 0) {
    w.plan[q].moves = done - start;
    if (resident_out) resident_out[q] = (int64_t)(n - p.drop);
  }
}

// Rows of one session, layer, K or V, and head, moved in ascending order: a step's rows are all read
// before the first of them is written, the next step's are on their way meanwhile.  (They lie behind
// the slots that this step writes.)
constexpr int COPY_THREADS = 256;

// 16 bytes a thread of rows of 256 bytes.
__global__ void __launch_bounds__(COPY_THREADS) weigh_copy_kernel(Dev d, WeighDev w) {
  constexpr int LANES = 16, ROWS = COPY_THREADS / LANES, U = 4, STEP = ROWS * U;
  pdl_wait();
  pdl_launch_dependents();
  const WeighPlan& p = w.plan[blockIdx.y];
  const int n = p.moves;
  if (n == 0) return;
  const uint2* list = w.list + p.list_at;
  // Stream (layer, K or V, head) starts there in a page; rows of a stream are side by side.
  const size_t row = (size_t)d.head_dim * d.esz, page = (size_t)d.layers * 2 * d.kv_heads * PS * row;
  uint8_t* at = d.pool + (size_t)blockIdx.x * PS * row + (threadIdx.x % LANES) * 16;
  const int r = threadIdx.x / LANES;
  auto place = [&](uint32_t gs) { return at + (gs / PS) * page + (gs % PS) * row; };
  uint4 x[U], y[U];
  uint32_t to[U], to_next[U];
  auto fetch = [&](int m0, uint4 (&v)[U], uint32_t (&t)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int m = m0 + u * ROWS + r;
      t[u] = NO_KEY;
      if (m < n) {
        const uint2 mv = list[m];
        t[u] = mv.y;
        v[u] = *reinterpret_cast<const uint4*>(place(mv.x));
      }
    }
  };
  fetch(0, x, to);
  for (int m0 = 0; m0 < n; m0 += STEP) {
    if (m0 + STEP < n) fetch(m0 + STEP, y, to_next);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (m0 + u * ROWS + r < n) *reinterpret_cast<uint4*>(place(to[u])) = x[u];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = y[u];
      to[u] = to_next[u];
    }
  }
}

// The same for rows in 4 bits: eight threads a row, a piece of D / 16 bytes each, the first D / 32 of
// them a scale too.
template <int D>
__global__ void __launch_bounds__(COPY_THREADS) weigh_copy_kv4_kernel(Dev d, WeighDev w) {
  using namespace kv4;
  constexpr int LANES = 8, ROWS_AT_ONCE = COPY_THREADS / LANES;
  using Piece = typename std::conditional<D == 128, uint2, uint32_t>::type;
  pdl_wait();
  pdl_launch_dependents();
  const WeighPlan& p = w.plan[blockIdx.y];
  const int n = p.moves;
  if (n == 0) return;
  const uint2* list = w.list + p.list_at;
  const int kv = blockIdx.x % 2, h = blockIdx.x / 2 % d.kv_heads, layer = blockIdx.x / 2 / d.kv_heads;
  const int i = threadIdx.x % LANES, r = threadIdx.x / LANES;
  for (int m0 = 0; m0 < n; m0 += ROWS_AT_ONCE) {
    const int m = m0 + r;
    Piece v = {};
    uint16_t s = 0;
    uint2 mv = {};
    if (m < n) {
      mv = list[m];
      const uint8_t* src = d.pool + tile_at(D, d.layers, d.kv_heads, mv.x / PS, layer, h, kv);
      const int slot = mv.x % PS;
      v = *reinterpret_cast<const Piece*>(src + (kv ? v_piece(D, slot, i) : k_piece(D, slot, i)));
      if (i < D / GROUP)
        s = *reinterpret_cast<const uint16_t*>(src + (kv ? v_scale(D, slot, i) : k_scale(D, slot, i)));
    }
    __syncthreads();
    if (m < n) {
      uint8_t* dst = d.pool + tile_at(D, d.layers, d.kv_heads, mv.y / PS, layer, h, kv);
      const int slot = mv.y % PS;
      *reinterpret_cast<Piece*>(dst + (kv ? v_piece(D, slot, i) : k_piece(D, slot, i))) = v;
      if (i < D / GROUP)
        *reinterpret_cast<uint16_t*>(dst + (kv ? v_scale(D, slot, i) : k_scale(D, slot, i))) = s;
    }
    __syncthreads();
  }
}

template <int N, bool RULE>
cudaError_t launch_plan(const Dev& d, const WeighDev& w, const WeighArgs& all, const float* weights,
                        int64_t* resident_out, uint8_t* kept, int64_t* used_out, cudaStream_t s, int64_t* launches) {
  WeighArgsT<N> a;
  a.n_seq = all.n_seq;
  a.kinds = all.kinds;
  a.sink = all.sink;
  a.recent = all.recent;
  for (int i = 0; i < a.n_seq; ++i) {
    a.sessions[i] = all.sessions[i];
    a.keep[i] = all.keep[i];
  }
  cudaError_t e = launch_ex(&weigh_select_kernel<N, RULE>, dim3(a.n_seq), dim3(META_THREADS),
                            CACHED_KEYS * 4, s, true, d, w, a, weights, used_out);
  if (e != cudaSuccess) return e;
  ++*launches;
  e = launch_ex(&weigh_apply_kernel<N>, dim3(a.n_seq), dim3(META_THREADS), 0, s, true, d, w, a,
                resident_out, kept);
  *launches += e == cudaSuccess;
  return e;
}

}  // namespace

cudaError_t launch_evict_weighted(const Dev& d, const WeighDev& w, bool kv4, const WeighArgs& a,
                                  const float* weights, int64_t* resident_out, uint8_t* kept,
                                  int64_t* used_out, cudaStream_t s, int64_t* launches) {
  auto plan = a.n_seq <= FEW ? (weights ? launch_plan<FEW, false> : launch_plan<FEW, true>)
                             : (weights ? launch_plan<MAX_SEQ, false> : launch_plan<MAX_SEQ, true>);
  cudaError_t e = plan(d, w, a, weights, resident_out, kept, used_out, s, launches);
  if (e != cudaSuccess) return e;
  const dim3 grid(d.layers * 2 * d.kv_heads, a.n_seq);
  if (!kv4)
    e = launch_ex(&weigh_copy_kernel, grid, dim3(COPY_THREADS), 0, s, true, d, w);
  else if (d.esz == 2)
    e = launch_ex(&weigh_copy_kv4_kernel<128>, grid, dim3(COPY_THREADS), 0, s, true, d, w);
  else
    e = launch_ex(&weigh_copy_kv4_kernel<64>, grid, dim3(COPY_THREADS), 0, s, true, d, w);
  *launches += e == cudaSuccess;
  return e;
}

}  // namespace kvc
