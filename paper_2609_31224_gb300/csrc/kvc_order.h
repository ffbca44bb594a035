// Order of the attention launches of one append (host side, no CUDA): which layers' K/V of
// the append are in the pool, and whether an attention launch may read pages before the
// kernels in front of it in the stream are complete ("early").
//
// Every attention launch lets the next one start before it has finished, so a chain of early
// launches may overlap.  The first launch after an append, or after a layer write, waits for
// it before it lets anything else start, but for those that know EARLY_OLD: behind a complete
// plan they let others start at once, read the older pages, and wait before the first page that
// holds a row of the append.  What they let start knows no more than they did.  A fused launch writes its layer's rows itself and
// reads them from the caller's buffers, so launches on other layers may overlap it, and so may
// a fused launch on the same layer; a plain launch on that layer reads the rows from the pool
// and has to wait, after which no fused write is pending any more.
#pragma once

#include <stdint.h>

namespace kvc {

// What a launch may read before the kernels in front of it are complete: nothing, the pages
// without a row of the last append, or all pages.
enum Early { EARLY_NONE, EARLY_OLD, EARLY_ALL };

class LaunchOrder {
 public:
  // An append: of all layers' K/V, or of none (layers follow one by one).
  void append(bool with_kv, int layers) {
    planned_ = false;
    written_ = !with_kv ? 0 : layers >= 64 ? ~0ull : (1ull << layers) - 1;
    settle();
  }
  // A separate write of one layer's K/V.  It waits for everything in front of it before it lets the
  // launch behind it start: the plan and all older rows are complete by then.  Its own rows are not,
  // until that launch has waited.
  void layer_write(int layer) {
    written_ |= 1ull << layer;
    planned_ = true;
    settle();
  }
  // Whether the append's plan is complete before any launch behind can start: a launch since has
  // waited for it before it let others start.
  bool planned() const { return planned_; }
  bool layer_written(int layer) const { return (written_ >> layer) & 1; }

  bool early(int layer, bool fused) const {
    return waited_ && (fused || !((pending_ >> layer) & 1));
  }
  // The attention launch that early(layer, fused) was asked for is in the stream.
  void launched(int layer, bool fused) {
    if (!early(layer, fused)) pending_ = 0;
    if (fused) {
      pending_ |= 1ull << layer;
      written_ |= 1ull << layer;
    }
    waited_ = planned_ = true;
  }

  // Plain launches that know EARLY_OLD: behind a complete plan, but not yet behind the write of the
  // append's rows, they read early all pages but those.  Such a launch lets others start before it
  // has waited itself, so that it changes nothing here: none of them may take the rows for complete.
  Early early_pages(int layer) const {
    return early(layer, false) ? EARLY_ALL : planned_ ? EARLY_OLD : EARLY_NONE;
  }
  void launched_pages(int layer, Early e) {
    if (e != EARLY_OLD) launched(layer, false);
  }

 private:
  void settle() {
    pending_ = 0;
    waited_ = false;
  }
  uint64_t written_ = 0;  // layers whose K/V of the append are in the pool, or will be
  uint64_t pending_ = 0;  // layers with a fused write that no launch has waited for
  bool planned_ = false;  // a launch or a layer write has waited for the append's plan
  bool waited_ = false;   // an attention launch has waited for the append (or layer write)
};

}  // namespace kvc
