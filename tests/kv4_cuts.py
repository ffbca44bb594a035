"""The rule by which a decode call over 4-bit rows is cut (csrc/kvc_kv4_cuts.h), asked from a test."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "kvc_kv4_cuts.h"
#include <cstdio>
#include <cstdlib>

int main(int argc, char** argv) {
  const kvc::kv4::DecodeCut c =
      kvc::kv4::decode_cut(std::atoi(argv[1]), std::atoi(argv[2]), std::atoll(argv[3]), std::atoi(argv[4]));
  std::printf("%d %d\n", (int)c.wide, c.slices);
}
"""


def program(folder, text):
    src, exe = folder / "cuts.cpp", folder / "cuts"
    src.write_text(text)
    inc = os.path.join(ROOT, "paper_2609_31224_gb300", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", inc, str(src), "-o", str(exe)], check=True)
    return str(exe)


def decode_cut(folder, sms, pairs, units, esz):
    """(8 warps a CTA, slices of each pair; 0: stream-K)."""
    r = subprocess.run([program(folder, PROGRAM)] + [str(x) for x in (sms, pairs, units, esz)],
                       capture_output=True, text=True, check=True)
    wide, slices = map(int, r.stdout.split())
    return bool(wide), slices
