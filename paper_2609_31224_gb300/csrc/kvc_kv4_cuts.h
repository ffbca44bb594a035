// How a decode call over 4-bit rows is cut over the SMs.  Plain C++, so that it is tested on the CPU.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace kvc {
namespace kv4 {

constexpr int DECODE_MAX_PARTS = 64;  // CTAs that share a (session, KV head) pair, at most

// How a call is cut, by what a launch takes in us: a fixed chain, then times in units of a page's
// work (binary32 pages, half as long, take 0.7 of it): the pages of a warp one after the other, each
// the longer the more warps share an SM, and 2 for the merge of a pair's slices.  Measured (us,
// 8 KV heads; Mk, Nk: k slices of 8 and 4 warps, S: stream-K; the first is the one chosen):
//   pages      1 session                4                     14                     38, 64
//    to 7   N1 3.0  M1 3.2  S 7.9   M1 3.0  N1 3.1        M1 3.7  N1 3.8        M1 4.5 N1 3.8, N1 4.9 S 12.4
//      25   M1 3.9  N8 4.5  S 8.8   M1 4.0  N1 4.6        M1 4.8  N1 5.4        M1 6.7 N1 6.8, N1 9.0 S 15.8
//      94   M11 5.1 M14 4.9 S 9.5   M4 6.4  M8 6.2        M1 9.3  N5 9.3        M1 13.5, N1 23.8 S 27.4
//     288   M17 5.7 N16 6.2 S 11.0  M8 8.8  N17 9.2       N5 18.3 M2 20.6       M1 33.7, S 60.1 M1 63.0
// One slice each and no merge wins up to about 40 pages; then as many slices as give a warp a page or
// two; stream-K where pairs outnumber the SMs' room and their last CTAs would leave most SMs empty.
// A launch counts as if it stood alone: one layer's CTAs leave no room for the next one's.
// n_pairs (session, KV head) pairs with `units` pages in all.
struct DecodeCut {
  bool wide;   // 8 warps a CTA (else 4)
  int slices;  // of each pair; 0: stream-K, 4 warps
};
inline DecodeCut decode_cut(int sms, int n_pairs, int64_t units, int esz) {
  const float page = esz == 2 ? 1.f : 0.7f;
  const int pages = (int)((units + n_pairs - 1) / n_pairs);
  DecodeCut best = {false, 0};
  float least = 3.4f + page * (8.4f + 0.0534f * units / sms);
  for (int wide = 0; wide < 2; ++wide) {
    const int warps = wide ? 8 : 4;
    const int most = std::max(1, std::min(std::min(DECODE_MAX_PARTS, pages), sms * (16 / warps) / n_pairs));
    for (int k = 1; k <= most; ++k) {
      const int64_t ctas = (int64_t)n_pairs * k;
      const bool alone = ctas <= sms;
      const float each = !alone ? 0.85f : wide ? 0.56f : 0.43f;
      const int64_t room = sms * (16 / warps), waves = (ctas + room - 1) / room;
      const int64_t steps = waves * ((pages + k * warps - 1) / (k * warps));
      const float t = 3.4f + page * (steps * each + (k > 1 ? 2.f + 0.03f * k : 0.f) +
                                     (alone ? ctas / (float)sms : 1.5f));
      if (t < least) {
        least = t;
        best = {wide != 0, k};
      }
    }
  }
  return best;
}

}  // namespace kv4
}  // namespace kvc
