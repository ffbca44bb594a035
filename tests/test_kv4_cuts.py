"""How decode calls over 4-bit rows are cut, without a GPU: within what the kernels take for every
number of pairs and pages, and one call of each kind as it is meant."""
import subprocess

from kv4_cuts import decode_cut, program

RANGE = r"""
#include "kvc_kv4_cuts.h"
#include <cstdio>
using namespace kvc::kv4;

int main() {
  for (int sms : {152, 148, 7})
    for (int esz : {2, 4})
      for (int pairs = 1; pairs <= 512 * 64; pairs += pairs < 700 ? 1 : 997)
        for (int pages = 1; pages <= 1 << 20; pages += pages < 600 ? 1 : 99991) {
          const DecodeCut c = decode_cut(sms, pairs, (int64_t)pairs * pages, esz);
          const long ctas = (long)pairs * c.slices;
          // A part for each slice of a pair, a partial state for each CTA (4,096 slots), all of them at
          // once: 16 warps an SM.  More slices than pages would leave CTAs without work.
          const bool ok = c.slices == 0 ? !c.wide
                                        : c.slices == 1 || (c.slices <= DECODE_MAX_PARTS && c.slices <= pages &&
                                                            ctas <= 4096 && ctas * (c.wide ? 8 : 4) <= sms * 16);
          if (!ok) {
            std::printf("%d SMs, %d bytes, %d pairs, %d pages: %d %d\n", sms, esz, pairs, pages, c.wide, c.slices);
            return 1;
          }
        }
  return 0;
}
"""


def test_every_cut_is_one_that_the_kernels_take(tmp_path):
    r = subprocess.run([program(tmp_path, RANGE)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_calls_of_each_kind(tmp_path):
    for esz in (2, 4):
        assert decode_cut(tmp_path, 152, 8, 8 * 4, esz)[1] == 1            # short sessions: no merge
        assert decode_cut(tmp_path, 152, 8, 8 * 288, esz)[1] > 8           # one long one: many slices
        assert decode_cut(tmp_path, 152, 512, 512 * 288, esz) == (False, 0)  # a full batch: stream-K
