"""New outputs of the binding's native path are torch's own in every respect: what watches or changes allocations sees them as it does on the Python path."""
import ctypes

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2506_04985_amd import binding as fptq
from test_gpu_binding import both, same  # noqa: F401

pytestmark = pytest.mark.gpu


def calls():
    """(call, outputs it allocates)"""
    M, N, K = 24, 48, 320
    g = torch.Generator(device="cuda").manual_seed(0)
    x, r = (torch.randn((M, K), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    w, s = torch.randint(-8, 8, (N, K), dtype=torch.int8, device="cuda", generator=g), torch.rand((N,), device="cuda", generator=g)
    ws = torch.rand((5, N), device="cuda", generator=g)
    wq, (xq, t) = fptq.fptq_pack_weights(w), fptq.fptq_quantize_act_dynamic(x)
    codes, scale, _ = fptq.fptq_norm_quantize8(x, r)
    return [(lambda: fptq.fptq_norm_quantize8(x, r), 3), (lambda: fptq.fptq_gated_quantize8(x, r), 2), (lambda: fptq.fptq_w4a8_linear(codes, scale, wq, M, N, K, 64, ws), 1),
            (lambda: fptq.fptq_quantize_act_dynamic(x), 2), (lambda: fptq.fptq_residual_norm_quantize(x, r, 0.4), 3), (lambda: fptq.fptq_w4a4_linear(xq, wq, M, N, K, 0.4, s, t), 1)]


class Allocations(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.made = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if func is torch.ops.aten.empty.memory_format or func is torch.ops.aten.empty_like.default:
            self.made.append(out)
        return out


def test_a_dispatch_mode_sees_them(both):  # noqa: F811
    for call, outputs in calls():
        def watched():
            with Allocations() as seen:
                got = call()
            got = [v for v in (got if isinstance(got, tuple) else (got,)) if v is not None]
            assert len(seen.made) == outputs == len(got)
            assert sorted(v.data_ptr() for v in got) == sorted(v.data_ptr() for v in seen.made)
            return tuple(got)
        same(*both(watched))


def test_the_profiler_sees_them(both):  # noqa: F811
    for call, outputs in calls():
        def watched():
            with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as profile:
                call()
            return sum(e.count for e in profile.key_averages() if e.key == "aten::empty" or e.key == "aten::empty_strided")
        native, python = both(watched)
        assert native == python == outputs


def test_deterministic_runs_fill_them(both):  # noqa: F811
    """One launch of the library's and one fill an output."""
    hip = ctypes.CDLL(next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64.so" in line))
    for call, outputs in calls():
        def nodes():
            call()
            torch.cuda.synchronize()
            graph, count = torch.cuda.CUDAGraph(keep_graph=True), ctypes.c_size_t(0)
            with torch.cuda.graph(graph):
                call()
            assert hip.hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(count)) == 0
            return count.value
        assert both(nodes) == (1, 1)
        torch.use_deterministic_algorithms(True)
        try:
            assert both(nodes) == (1 + outputs, 1 + outputs)
        finally:
            torch.use_deterministic_algorithms(False)
