// Attention over whole prompts (kvc_attn_prompt): the kernels' attributes and launches by element type
// (kvc_prompt_tc.cu: bfloat16, kvc_prompt_f32.cu: binary32).
#include <algorithm>

#include "kvc_prompt.h"

namespace kvc {

cudaError_t prompt_attributes(const Dev& d) {
  const cudaError_t e = d.esz == 2 ? prompt_tc_attributes() : prompt_f32_attributes();
  return e != cudaSuccess ? e : weights_attributes(d);
}

cudaError_t launch_attn_prompt(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int tiles,
                               int pages_max, LaunchOrder* order, cudaStream_t s, int64_t* launches) {
  // Items of 64 tokens (binary32: 32) of a KV head; where they are too few for the SMs, their keys are cut
  // into parts, an item a CTA in all (or three for two CTAs), which a second kernel joins.  Parts of four steps of 128 keys
  // (64) or more, few binary32 ones of two.  A chunk of 64 tokens, 8 KV heads (4), us a layer, against one
  // part, behind
  //   4,096 positions    bfloat16 77 -> 34, binary32 407 -> 49 (parts of two steps 37, 58)
  //   16,000 positions            263 -> 49,        1,560 -> 118 (two items a CTA 67, 127)
  //   600 positions               25 (of two steps 22), 73 -> 31 (of four steps 47)
  //   4,096, 8 sessions           82 -> 59,           412 -> 218
  // (16 sessions, 128 items in two parts each: 86 -> 108 and 412.)
  const bool tc = d.esz == 2;
  const int64_t items = (int64_t)tiles * d.kv_heads, steps = pages_max / (tc ? 8 : 4);
  const int64_t most = tc ? steps / 4 : std::max(steps / 4, std::min<int64_t>(steps / 2, 8));
  int64_t parts = lim.sms / items;
  if (parts == 1 && 2 * lim.sms / items > 2) parts = 3;
  parts = std::max<int64_t>(1, std::min({parts, most, part_items(d) / items}));
  const cudaError_t e = tc ? launch_prompt_tc(d, lim, layer, q, out, (int)parts, items, s, launches)
                           : launch_prompt_f32(d, lim, layer, q, out, (int)parts, items, s, launches);
  // (All kernels wait for the one before them before they let the next one start.)
  if (e == cudaSuccess) order->launched(layer, false);
  return e;
}

}  // namespace kvc
