"""kvc_launches against the kernel nodes of the same calls captured into a graph."""
import contextlib
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2609_31224_gb300 import KVCache, KvcError  # noqa: E402

pytestmark = pytest.mark.gpu

TD = {"bf16": torch.bfloat16, "f32": torch.float32}
DIM = {"bf16": 128, "f32": 64}
RELAXED, KERNEL = 2, 0


def ok(rc):
    assert rc == 0, rc


class Nodes:
    """Kernel nodes of what is launched on a stream inside `captured`."""

    def __init__(self):
        self.cu, self.count = ctypes.CDLL("libcuda.so.1"), 0

    @contextlib.contextmanager
    def captured(self, stream):
        cu, graph = self.cu, ctypes.c_void_p()
        ok(cu.cuStreamBeginCapture_v2(ctypes.c_void_p(stream.cuda_stream), RELAXED))
        yield
        ok(cu.cuStreamEndCapture(ctypes.c_void_p(stream.cuda_stream), ctypes.byref(graph)))
        n = ctypes.c_size_t()
        ok(cu.cuGraphGetNodes(graph, None, ctypes.byref(n)))
        nodes = (ctypes.c_void_p * n.value)()
        ok(cu.cuGraphGetNodes(graph, nodes, ctypes.byref(n)))
        self.count = 0
        for node in nodes:
            kind = ctypes.c_int()
            ok(cu.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)))
            self.count += kind.value == KERNEL
        ok(cu.cuGraphDestroy(graph))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_bits", [None, 4])
@pytest.mark.parametrize("n", [1, 3, 40])
def test_launches_are_the_kernels_of_a_call(dtype, kv_bits, n):
    """40 sessions of 8 heads: 320 pairs, for which the bfloat16 prefill over 4-bit rows takes two
    launches (whole waves of CTAs, then the rest in slices)."""
    d, layers, heads, most = DIM[dtype], 2, 8, 1600
    cache = KVCache(n_sessions=n, layers=layers, q_heads=4 * heads, kv_heads=heads, head_dim=d,
                    budget=-1, window=1, dtype=dtype, n_pages=n * (most // 16 + 1),
                    max_pages_per_session=most // 16 + 1, max_positions=most, max_seq_per_call=n,
                    max_tokens_per_call=n * most, kv_bits=kv_bits)
    every, stream, nodes = list(range(n)), torch.cuda.Stream(), Nodes()
    x = torch.zeros(layers, 17 * n, heads, d, device="cuda", dtype=TD[dtype])
    q = torch.zeros(17 * n, 4 * heads, d, device="cuda", dtype=TD[dtype])
    types = torch.full((17 * n,), 2, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros(layers, 17 * n, heads, d, device="cuda", dtype=TD[dtype]) for _ in range(2)]
    pos, count = torch.zeros(32, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    k, out, s = x.data_ptr(), torch.zeros_like(q), stream.cuda_stream
    seen = {}

    def launched(what, fn):
        before = cache.launches()
        with nodes.captured(stream):
            fn()
        seen[what] = cache.launches() - before
        assert seen[what] == nodes.count > 0, (what, seen[what], nodes.count)

    for tokens, attend, fused in ((1, "attn_decode_raw", "attn_decode_kv_raw"),
                                  (17, "attn_prefill_raw", "attn_prefill_kv_raw")):
        cu = np.arange(n + 1) * tokens
        launched(f"append {tokens}", lambda: cache.append_chunk(every, cu, types, x, x, stream=s))
        launched(f"attention {tokens}",
                 lambda: getattr(cache, attend)(1, q.data_ptr(), out.data_ptr(), s))
        launched(f"positions {tokens}", lambda: cache.append_chunk(every, cu, types, None, None, stream=s))
        launched(f"layer {tokens}", lambda: cache.append_kv_layer_raw(0, k, k, s))
        launched(f"fused {tokens}",
                 lambda: getattr(cache, fused)(1, k, k, q.data_ptr(), out.data_ptr(), s))
        if tokens == 1 and kv_bits is None:
            # (Its first call in a CUDA context may not be captured.)
            ok(cache.lib.kvc_attn_decode_noalloc(cache.ctx, 0, q.data_ptr(), out.data_ptr(), s))
            stream.synchronize()
            launched("noalloc", lambda: ok(cache.lib.kvc_attn_decode_noalloc(
                cache.ctx, 0, q.data_ptr(), out.data_ptr(), s)))
    launched("read", lambda: cache.read_kv([0], [0], [0, 17], k=outs[0][:, :17].contiguous(),
                                           v=outs[1][:, :17].contiguous(), stream=s))
    launched("transcript", lambda: ok(cache.lib.kvc_export_transcript(
        cache.ctx, 0, 17, pos.data_ptr(), outs[0].data_ptr(), outs[1].data_ptr(), count.data_ptr(), s)))
    launched("evict", lambda: cache.evict(every, stream=s))
    launched("release", lambda: cache.release(every, stream=s))
    two = dtype == "bf16" and kv_bits == 4 and n == 40
    assert seen["attention 17"] == 1 + two and seen["attention 1"] == seen["fused 1"] == 1, seen
    before = cache.launches()
    with pytest.raises(KvcError):
        cache.append_chunk([n], [0, 1], types, None, None)
    assert cache.launches() == before       # (what was refused launched nothing)


@pytest.mark.parametrize("kv_bits,per_layer", [(None, False), (4, False), (4, True)])
def test_the_driver_counts_what_was_launched(kv_bits, per_layer):
    """A unit of 40 sessions of 8 heads in one layer: the append (plan and rows, or the plan), the chunk's
    attention, which takes two launches over 4-bit rows, and the layer's rows in front of it."""
    from synth import gpu as synth_gpu
    from synth import script as S
    from synth.driver import Driver
    synth_gpu.build()
    w = S.SINGLE_BF16.with_(layers=1, q_heads=32, kv_heads=8, n_sessions=40, units=24, offset_max=0,
                            budget=4096)
    drv = Driver(w, S.workload_scripts(w), kv_bits=kv_bits)
    drv.fast_forward(18)                    # some 400 positions a session: four stages of 128 keys
    step = drv.prepare_step()
    chunk = next(c for c in step.calls if c.kind == "prefill")
    want = {(None, False): 2 + 1, (4, False): 2 + 2, (4, True): 1 + 1 + 2}[kv_bits, per_layer]
    assert len(chunk.sessions) == 40
    assert drv.run_call(chunk, per_layer=per_layer) == want
    torch.cuda.synchronize()
