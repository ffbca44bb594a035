// Host-side launchers of the kvc kernels (defined in the .cu files) and the
// argument blocks they pass by value.
#pragma once

#include "kvc_decode_slices.h"
#include "kvc_internal.cuh"
#include "kvc_order.h"

namespace kvc {

// What a launch records that finds no units (one thread): it was captured, and replayed behind chunks that it does
// not take.  Behind a failed append, whose error is recorded, nothing.
__device__ inline void note_other_chunks(const Dev& d) {
  if (d.g->total_tokens > 0) set_error(d, KVC_DERR_CHUNK);
}

// ---------------------------------------------------------------------------
// Launchers (defined in the .cu files).
// ---------------------------------------------------------------------------
// Session lists of a call, by value.  Calls of up to FEW sessions pass the small block: the
// driver copies a launch's arguments, and 4 KB of them cost more than the rest of a launch.
constexpr int FEW = 32;
template <int N>
struct AppendArgsT {
  int32_t n_seq;
  int32_t total;
  int32_t max_t;  // longest chunk
  int32_t sessions[N];
  int32_t cu[N + 1];
};
using AppendArgs = AppendArgsT<MAX_SEQ>;

template <int N>
struct SeqArgsT {
  int32_t n_seq;
  int32_t sessions[N];
};
using SeqArgs = SeqArgsT<MAX_SEQ>;

// Rows to read back: rows [cu[i], cu[i + 1]) of the outputs are session i's retained positions from
// first[i] on.
template <int N>
struct ReadArgsT {
  int32_t n_seq;
  int32_t total;
  int32_t sessions[N];
  int32_t first[N];
  int32_t cu[N + 1];
};
using ReadArgs = ReadArgsT<MAX_SEQ>;

// Sessions to evict by weight, and what is left of each.
template <int N>
struct WeighArgsT {
  int32_t n_seq;
  int32_t kinds, sink, recent;
  int32_t sessions[N];
  int32_t keep[N];
};
using WeighArgs = WeighArgsT<MAX_SEQ>;

// What an eviction by weight does to one session of the call (kvc_evict_weighted.cu).
struct WeighPlan {
  int64_t list_at;     // its entries in the list
  uint32_t key;        // positions of smaller keys go, and of equal ones
  int32_t tie_last;    // those up to this retained index
  int32_t drop;        // positions that go
  int32_t first;       // retained index of the first of them
  int32_t end;         // live positions consumed
  int32_t stay;        // compacted positions afterwards
  int32_t pages;       // and their pages
  int32_t taken;       // of them live pages taken over
  int32_t extra;       // 1: the last one is new
  int32_t extra_page;
  int32_t freed;       // consumed or compacted pages that are free again
  int32_t moves;       // rows that move
  int32_t ok;          // 0: the call failed, nothing changes
  int32_t pad;
};
static_assert(sizeof(WeighPlan) == 64, "WeighPlan size");

// Its part of the metadata workspace.
struct WeighDev {
  WeighPlan* plan;     // [max_seq]
  uint2* list;         // [positions of max_seq sessions] (key, slot), then moves (from, to)
  int32_t* count;      // arrival counter
};

// What the device runs at once, for each kernel whose launch shape follows from it.  kvc_create
// looks it up for the current CUDA context; the first time for a context, element type and way of
// holding the rows that also sets the attributes of the kernels over them, which belong to the CUDA
// context too (about 2 ms in a process's first kvc_create, 0.5 to 1 ms for another kind).  What it
// does not look up is 0.
constexpr int PF_MAX_SLICES = 8;  // CTAs of a bfloat16 prefill cluster, at most
constexpr int KV4_PF_WARPS = 6;   // warps that share a page in the prefill over 4-bit rows, at most
struct Limits {
  int sms;                         // SMs
  int dec_stream_k;                // CTAs of the stream-K decode's grid
  int dec_wide, dec_narrow;        // CTAs of the 16-warp and 4-warp pair split in one wave
  int pf_stream_k;                 // CTAs of the stream-K prefill (bfloat16)
  int pf_clusters[PF_MAX_SLICES + 1];  // [k] clusters of k CTAs of the prefill's pair split
  int f32_cluster[2][2];           // largest cluster of the binary32 prefill: [rows][spread]
  int kv4_decode;                  // CTAs of the stream-K decode over 4-bit rows
  int kv4_prefill[KV4_PF_WARPS + 1];  // [w] CTAs of the prefill with w warps to a page
  int kv4_clusters[PF_MAX_SLICES + 1];  // [k] clusters of k CTAs of the bfloat16 prefill over them
};
cudaError_t query_limits(const Dev& d, bool kv4, Limits* lim);  // kv4: rows in 4 bits
// Id of the current CUDA context (never reused: a context that replaces a destroyed one at the
// same address has another).
cudaError_t current_context_id(unsigned long long* id);

cudaError_t launch_init(const Dev& d, double rope_base, cudaStream_t s);
// single: every session of the call gets exactly one token (one session: plan and K/V write in
// one launch).
// kv4: the rows are held in 4 bits.  Adds its launches to *launches, as the others that take it do.
cudaError_t launch_append(const Dev& d, bool kv4, const AppendArgs& a, const uint8_t* types,
                          const void* k, const void* v, bool single, int sms, cudaStream_t s,
                          int64_t* launches);
// after_plan: launched right behind the plan kernel of the same append.
cudaError_t launch_append_layers(const Dev& d, int total, int layer0, int n_layers, const void* k,
                                 const void* v, bool after_plan, cudaStream_t s);
cudaError_t launch_evict(const Dev& d, bool kv4, const SeqArgs& a, int64_t* resident_out,
                         int64_t* used_out, int sms, cudaStream_t s);
// (No weights: by the context's policy.)
cudaError_t launch_evict_weighted(const Dev& d, const WeighDev& wd, bool kv4, const WeighArgs& a,
                                  const float* weights, int64_t* resident_out, uint8_t* kept,
                                  int64_t* used_out, cudaStream_t s, int64_t* launches);
cudaError_t launch_release(const Dev& d, const SeqArgs& a, int64_t* used_out, cudaStream_t s);
cudaError_t launch_transcript(const Dev& d, bool kv4, int session, int cap, int32_t* pos_out,
                              void* k_out, void* v_out, int32_t* count, cudaStream_t s);
cudaError_t launch_read_kv(const Dev& d, bool kv4, const ReadArgs& a, int layer0, int n_layers,
                           void* k_out, void* v_out, int64_t* resident_out, int sms,
                           cudaStream_t s);
// The parts of those calls that touch 4-bit rows (kvc_kv4_rows.cu), and the attention over them.
// early: k and v were complete before the kernel in front could start; planned: the plan was.
cudaError_t launch_append_layers_kv4(const Dev& d, int total, int layer0, int n_layers,
                                     const void* k, const void* v, bool early, bool planned, int sms,
                                     cudaStream_t s);
cudaError_t launch_evict_copy_kv4(const Dev& d, int sms, cudaStream_t s);
cudaError_t launch_transcript_copy_kv4(const Dev& d, int cap, void* k_out, void* v_out, int sms,
                                       cudaStream_t s);
// new_k / new_v (optional): the layer's rows of the append, written first.  Chunks of up to max_t
// tokens; units: estimate of the call's (session, KV head, page) units, for the choice of the shape
// only.  Asks `order` when it may read early, and reports its launches to it.
cudaError_t launch_attn_kv4(const Dev& d, const Limits& lim, LaunchOrder* order, int layer,
                            const void* new_k, const void* new_v, const void* q, void* out,
                            int n_seq, int total, int max_t, int64_t units, cudaStream_t s,
                            int64_t* launches);
// Single tokens (kvc_kv4_decode.cu); with new_k / new_v their rows are written by the launch itself.
cudaError_t launch_decode_kv4(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                              const void* new_k, const void* new_v, int n_pairs, int64_t units,
                              bool early, cudaStream_t s);
cudaError_t kv4_decode_limits(const Dev& d, Limits* lim);  // both set their kernels' attributes
cudaError_t kv4_prefill_limits(const Dev& d, Limits* lim);
// Chunks of bfloat16 calls (kvc_kv4_prefill_tc.cu).
cudaError_t launch_prefill_kv4_tc(const Dev& d, const Limits& lim, int layer, const void* q,
                                  void* out, int n_pairs, int64_t units, Early early,
                                  cudaStream_t s, int64_t* launches);
cudaError_t launch_prefill_kv4_f32(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                                   int n_pairs, int max_t, int64_t units, Early early, cudaStream_t s);
cudaError_t kv4_prefill_tc_limits(Limits* lim);
cudaError_t kv4_prefill_f32_limits(Limits* lim);
// Attention launches may start while the kernel before them in the stream finishes.  early:
// they may also read what the append wrote before that (an attention launch of the same
// append came before, so the append is complete).
// new_k / new_v (optional): the fused per-layer write of the new tokens' K/V.
// epoch: tag of this launch's partial states (nonzero, never reused while tags
// of it may remain in the slots); 0 selects the fenced arrival instead.
// pages: estimate of the longest session's pages, for the choice of the split only.
cudaError_t launch_attn_decode(const Dev& d, const Limits& lim, int layer, const void* q,
                               void* out, int n_seq, int pages, bool early, cudaStream_t s,
                               uint32_t epoch, const void* new_k = nullptr,
                               const void* new_v = nullptr);
// Stream-K decode kernel (kvc_attn_decode.cu): its grid (resident CTAs, capped by
// the partial slots; sets its attributes) and its launch.
int decode_stream_k_grid(const Dev& d);
cudaError_t launch_attn_decode_streamk(const Dev& d, int layer, const CUtensorMap& map_lo,
                                       const CUtensorMap& map_hi, const void* q, void* out,
                                       float scale, int grid, int min_units, const void* new_k,
                                       const void* new_v, bool early, cudaStream_t s);
// Pair-split decode kernel (kvc_attn_decode_split.cu).  wide: the 16-warp shape
// (one CTA per SM; tensor-core pages for bfloat16), else the 4-warp shape.  k_most: CTAs per
// pair; fit: how the 4-warp shape counts those that work.
// Resident CTAs in one wave (sets its attributes).
int decode_split_slots(int esz, bool wide, int sms);
bool decode_split_uses_tma(int esz, bool wide);      // needs the pool's tensor maps
cudaError_t launch_attn_decode_split(const Dev& d, bool wide, int layer, const CUtensorMap& map_lo,
                                     const CUtensorMap& map_hi, const void* q, void* out,
                                     float scale, int k_most, const NarrowFit& fit,
                                     uint32_t epoch, const void* new_k, const void* new_v,
                                     int n_pairs, bool early, cudaStream_t s);
// new_k / new_v (optional, bfloat16 only): the chunk's rows of this layer, written
// into the pool by the launch itself (the per-layer order).
// pages_max, pages_sum: estimates of the sessions' resident pages (largest, sum over the
// call), for the choice of the split only.
cudaError_t launch_attn_prefill(const Dev& d, const Limits& lim, int layer, const void* q,
                                void* out, int n_seq, int max_t, int pages_max,
                                int64_t pages_sum, bool early, cudaStream_t s,
                                const void* new_k = nullptr, const void* new_v = nullptr);
// k = 0: stream-K over `grid` CTAs; k >= 1: pair split, grid = pairs * k CTAs.
cudaError_t launch_attn_prefill_tc(const Dev& d, int layer, const CUtensorMap& lo,
                                   const CUtensorMap& hi, const void* q, void* out, int grid,
                                   int k, int max_t, bool early, cudaStream_t s, const void* new_k,
                                   const void* new_v);
// Sets its attributes; CTAs of the stream-K split and clusters of the pair split at once.
cudaError_t prefill_tc_limits(Limits* lim);
// binary32; pages_max as in launch_attn_prefill.
cudaError_t prefill_f32_limits(Limits* lim);
cudaError_t launch_attn_prefill_f32(const Dev& d, const Limits& lim, int layer, const void* q,
                                    void* out, int n_seq, int max_t, int pages_max, bool early,
                                    cudaStream_t s);
// Two 2-D views of the bfloat16 pool as rows of 128 elements (columns 0-63 and
// 64-127), 16-row boxes, 128-byte swizzle; cached per pool.  False if the driver
// entry point is missing or the encoding fails.
bool pool_tensor_maps(const Dev& d, CUtensorMap* lo, CUtensorMap* hi);
// A 4-D view whose boxes are the 4 KiB of a (page, layer, K or V, head) in one copy: 8-row groups of 1 KiB,
// 128-byte swizzle, columns 0-63 and 64-127 of a group side by side.  Coordinates (0, 0, 0, row / 8).
bool pool_tile_map(const Dev& d, CUtensorMap* tiles);
// Whole prompts (kvc_prompt.cu): chunks of any length, rows in the element type.  pages_max: an estimate of
// the longest session's pages, for the split alone.  tiles: of prompt_tokens tokens, all sessions'.
inline int prompt_tokens(const Dev& d) { return d.esz == 2 ? 64 : 32; }
cudaError_t launch_attn_prompt(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int tiles,
                               int pages_max, LaunchOrder* order, cudaStream_t s, int64_t* launches);
// Attributes of the kernels of both, in the current CUDA context.
cudaError_t prompt_attributes(const Dev& d);
cudaError_t weights_attributes(const Dev& d);
// Attention weights of the last append's queries, added to weights (kvc_weights.cu).  work: bytes as
// weights_work_bytes says.  pages_max, pages_sum: estimates of the sessions' pages, for the split alone.
size_t weights_work_bytes(const kvc_config& c);
cudaError_t launch_attn_weights(const Dev& d, const Limits& lim, int layer, const void* q,
                                float* weights, void* work, int n_seq, int total, int max_t,
                                int pages_max, int64_t pages_sum, LaunchOrder* order, cudaStream_t s,
                                int64_t* launches);
int noalloc_max_pairs();
cudaError_t launch_attn_decode_noalloc(const Dev& d, int layer, const void* q, void* out,
                                       int n_seq, cudaStream_t s);

}  // namespace kvc
