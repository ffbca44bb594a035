"""What kvc_create looks up (csrc/kvc_decode_dispatch.cu, query_limits): each kind of cache its own
kernels' limits, once per CUDA context, and no error of the others' kernels.  Compiled with stand-ins
for the kernels' files and the CUDA runtime, so that it runs without a GPU."""
import os
import shutil
import subprocess

import pytest

from paper_2609_31224_gb300 import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "kvc_decode_dispatch.cu"
#include <cstdio>

static unsigned long long g_id = 1;
static int own_calls, kv4_calls, own_error, kv4_error;

namespace kvc {
cudaError_t own(int n) {
  own_calls += n;
  return own_error ? cudaErrorInvalidValue : cudaSuccess;
}
cudaError_t held(int n) {
  kv4_calls += n;
  return kv4_error ? cudaErrorInvalidValue : cudaSuccess;
}
cudaError_t current_context_id(unsigned long long* id) {
  *id = g_id;
  return cudaSuccess;
}
int decode_stream_k_grid(const Dev&) { own(1); return 456; }
int decode_split_slots(int, bool, int) { own(1); return 152; }
bool decode_split_uses_tma(int, bool) { return false; }
bool pool_tensor_maps(const Dev&, CUtensorMap*, CUtensorMap*) { return false; }
cudaError_t prefill_tc_limits(Limits* lim) { lim->pf_stream_k = 152; return own(1); }
cudaError_t prefill_f32_limits(Limits* lim) { lim->f32_cluster[0][0] = 8; return own(1); }
cudaError_t kv4_decode_limits(const Dev&, Limits* lim) { lim->kv4_decode = 608; return held(1); }
cudaError_t kv4_prefill_limits(const Dev& d, Limits* lim) {
  (d.esz == 2 ? lim->kv4_clusters : lim->kv4_prefill)[1] = 152;
  return held(1);
}
cudaError_t launch_attn_decode_split(const Dev&, bool, int, const CUtensorMap&, const CUtensorMap&,
                                     const void*, void*, float, int, const NarrowFit&, uint32_t,
                                     const void*, const void*, int, bool, cudaStream_t) {
  return cudaSuccess;
}
cudaError_t launch_attn_decode_streamk(const Dev&, int, const CUtensorMap&, const CUtensorMap&,
                                       const void*, void*, float, int, int, const void*, const void*,
                                       bool, cudaStream_t) {
  return cudaSuccess;
}
}  // namespace kvc

int main() {
  kvc::Limits lim;
  for (int esz : {2, 4}) {
    kvc::Dev d = {};
    d.esz = esz;
    // A cache in its own type, while nothing of the 4-bit kernels can be looked up.
    own_calls = kv4_calls = own_error = 0;
    kv4_error = 1;
    if (kvc::query_limits(d, false, &lim) != cudaSuccess) return 1;
    if (kv4_calls != 0 || own_calls != 4 || lim.sms != 152 || lim.dec_stream_k != 456) return 2;
    // A cache in 4 bits: not what was found for the other kind, and none of its kernels.
    if (kvc::query_limits(d, true, &lim) == cudaSuccess) return 3;
    own_calls = kv4_calls = kv4_error = 0;
    own_error = 1;
    if (kvc::query_limits(d, true, &lim) != cudaSuccess) return 4;
    if (own_calls != 0 || kv4_calls != 2 || lim.sms != 152 || lim.kv4_decode != 608) return 5;
    if ((esz == 2 ? lim.kv4_clusters : lim.kv4_prefill)[1] != 152) return 6;
    // Both are known now; another CUDA context starts over.
    kv4_error = 1;
    if (kvc::query_limits(d, false, &lim) != cudaSuccess || lim.dec_stream_k != 456) return 7;
    if (kvc::query_limits(d, true, &lim) != cudaSuccess || lim.kv4_decode != 608) return 8;
    if (own_calls != 0 || kv4_calls != 2) return 9;
    ++g_id;
    if (kvc::query_limits(d, false, &lim) == cudaSuccess || kvc::query_limits(d, true, &lim) == cudaSuccess)
      return 10;
  }
  return 0;
}
"""
# The runtime calls that it makes, and what the objects that nvcc makes refer to.
RUNTIME = r"""
extern "C" int cudaGetDevice(int* dev) {
  *dev = 0;
  return 0;
}
extern "C" int cudaDeviceGetAttribute(int* value, int, int) {
  *value = 152;
  return 0;
}
extern "C" void** __cudaRegisterFatBinary(void*) { return nullptr; }
extern "C" void __cudaRegisterFatBinaryEnd(void**) {}
extern "C" void __cudaUnregisterFatBinary(void**) {}
extern "C" char __cudaInitModule(void**) { return 0; }
"""


@pytest.mark.skipif(shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"),
                    reason="needs nvcc")
def test_each_kind_of_cache_looks_up_its_own_kernels(tmp_path):
    src, run, exe = tmp_path / "limits.cu", tmp_path / "runtime.cpp", tmp_path / "limits"
    src.write_text(PROGRAM)
    run.write_text(RUNTIME)
    inc = os.path.join(ROOT, "paper_2609_31224_gb300", "csrc")
    r = subprocess.run([B.nvcc(), *B.ARCH, "-std=c++17", "-I", inc, "-cudart", "none", str(src),
                        str(run), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([str(exe)]).returncode == 0
