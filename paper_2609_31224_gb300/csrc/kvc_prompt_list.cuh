// What every kernel of whole prompts uses: the list of a call's items, and what a token sees.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

namespace {

constexpr unsigned ALL_LANES = 0xFFFFFFFFu;

// Blocks that the tokens up to `tok` of the chunk see.
__device__ inline int blocks_seen(const SeqInfo& si, int tok) {
  return si.n_hist_pages + (si.live_head + si.n_live - si.t + tok) / PS + 1;
}

// Slots [lo, hi) of block b that hold a position with index <= q_log.
__device__ inline uint32_t slots_seen(const SeqInfo& si, int b, int n_blocks, int q_log) {
  if (b >= n_blocks) return 0;
  const BlockRange br = block_range(si, b);
  const int hi = min(br.hi, q_log - br.base + 1);
  return hi <= br.lo ? 0u : ((1u << hi) - 1u) & ~((1u << br.lo) - 1u);
}

// Work lists: a session has count(session) items.  s_group holds the first item of each group of 16
// sessions, and the number of all behind the last.
constexpr int GROUP_SEQ = 16;
constexpr int GROUPS = MAX_SEQ / GROUP_SEQ;
static_assert(GROUPS <= 32, "a lane a group");

template <typename CountFn>
__device__ inline void list_items(int n_seq, int lane, int* s_group, CountFn count) {  // one warp
  int n = 0;
  for (int i = lane * GROUP_SEQ; i < min(n_seq, (lane + 1) * GROUP_SEQ); ++i) n += count(i);
  int upto = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(ALL_LANES, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane < GROUPS) s_group[lane] = upto - n;
  if (lane == 31) s_group[GROUPS] = upto;
}

// Session of item `at`, and which of the session's items it is (one warp).
template <typename CountFn>
__device__ inline int find_item(int n_seq, int lane, const int* s_group, int at, CountFn count, int* which) {
  const unsigned before = __ballot_sync(ALL_LANES, lane < GROUPS && s_group[min(lane, GROUPS)] <= at);
  const int group = 31 - __clz(before);
  const int i = group * GROUP_SEQ + lane, n = lane < GROUP_SEQ && i < n_seq ? count(i) : 0;
  int upto = n;
#pragma unroll
  for (int o = 1; o < GROUP_SEQ; o <<= 1) {
    const int y = __shfl_up_sync(ALL_LANES, upto, o);
    if (lane >= o) upto += y;
  }
  const int rest = at - s_group[group];
  const int mine = __ffs(__ballot_sync(ALL_LANES, lane < GROUP_SEQ && rest < upto)) - 1;
  *which = rest - __shfl_sync(ALL_LANES, upto - n, mine);
  return group * GROUP_SEQ + mine;
}

// Counters of a launch: its items so far, and its CTAs that are through.  The last of them leaves both as
// it found them.
__device__ inline int take_item(const Dev& d) { return atomicAdd(&d.pf_count[0], 1); }
__device__ inline void leave_counters(const Dev& d) {  // one thread of each CTA
  if (atomicAdd(&d.dec_count[0], 1) == (int)gridDim.x - 1) {
    d.pf_count[0] = 0;
    d.dec_count[0] = 0;
  }
}

}  // namespace

}  // namespace kvc
