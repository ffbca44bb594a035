// Attention over a cache held in 4 bits (KVC_KV4): which kernel takes a call.  Chunks of one token go to
// the decode kernel, which writes the layer's new rows itself; longer ones to the prefill of the
// element type, behind a launch that writes them.
#include "kvc_launch.cuh"

namespace kvc {

cudaError_t kv4_prefill_limits(const Dev& d, Limits* lim) {
  return d.esz == 2 ? kv4_prefill_tc_limits(lim) : kv4_prefill_f32_limits(lim);
}

cudaError_t launch_attn_kv4(const Dev& d, const Limits& lim, LaunchOrder* order, int layer,
                            const void* new_k, const void* new_v, const void* q, void* out,
                            int n_seq, int total, int max_t, int64_t units, cudaStream_t s,
                            int64_t* launches) {
  const bool fused = new_k != nullptr;
  if (max_t == 1) {
    const cudaError_t e = launch_decode_kv4(d, lim, layer, q, out, new_k, new_v, n_seq * d.kv_heads,
                                            units, order->early(layer, fused), s);
    if (e != cudaSuccess) return e;
    ++*launches;
    order->launched(layer, fused);
    return cudaSuccess;
  }
  if (fused) {
    const cudaError_t e = launch_append_layers_kv4(d, total, layer, 1, new_k, new_v, false,
                                                   order->planned(), lim.sms, s);
    if (e != cudaSuccess) return e;
    ++*launches;
    order->layer_write(layer);
  }
  const Early early = order->early_pages(layer);
  cudaError_t e;
  if (d.esz == 2) {
    e = launch_prefill_kv4_tc(d, lim, layer, q, out, n_seq * d.kv_heads, units, early, s, launches);
  } else {
    e = launch_prefill_kv4_f32(d, lim, layer, q, out, n_seq * d.kv_heads, max_t, units, early, s);
    if (e == cudaSuccess) ++*launches;
  }
  if (e == cudaSuccess) order->launched_pages(layer, early);
  return e;
}

}  // namespace kvc
