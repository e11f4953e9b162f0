"""The binding of the 8-bit calls: native path and Python path alike, what both refuse, other streams and threads."""
import threading

import pytest
import torch

from paper_2506_04985_amd import binding as fptq
from test_gpu_binding import both, same  # noqa: F401

pytestmark = pytest.mark.gpu


def data(M=20, N=48, K=300, group=64):
    g = torch.Generator(device="cuda").manual_seed(M)
    x, r = (torch.randn((M, K), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    gain = torch.rand((K,), device="cuda", generator=g).to(torch.bfloat16)
    w = fptq.fptq_pack_weights(torch.randint(-8, 8, (N, K), dtype=torch.int8, device="cuda", generator=g))
    return x, r, gain, w, torch.rand((-(-K // group), N), device="cuda", generator=g)


@pytest.mark.parametrize("M,N,K", [(1, 48, 300), (20, 48, 300), (130, 64, 9000)])
def test_every_call_gives_the_same(both, M, N, K):  # noqa: F811
    x, r, gain, w, ws = data(M, N, K)
    codes, scale, z = fptq.fptq_norm_quantize8(x, r, gain, eps=1e-5)
    wide = torch.cat([x, r], 1)
    mine = lambda: (torch.empty_like(codes), torch.empty_like(scale), torch.empty_like(x))
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for f in (lambda: fptq.fptq_norm_quantize8(x, r, gain, eps=1e-5), lambda: fptq.fptq_norm_quantize8(x), lambda: fptq.fptq_norm_quantize8(x, None, gain, fptq.SCALE_NONE),
              lambda: fptq.fptq_norm_quantize8(x, r, want_residual=False), lambda: fptq.fptq_norm_quantize8(x, r, gain, 1, 1e-5, *mine()),
              lambda: fptq.fptq_gated_quantize8(x, r), lambda: fptq.fptq_gated_quantize8(*wide.split(K, 1)), lambda: fptq.fptq_gated_quantize8(x, r, *mine()[:2]),
              lambda: fptq.fptq_w4a8_linear(codes, scale, w, M, N, K, 64, ws), lambda: fptq.fptq_w4a8_linear(codes, scale, w, M, N, K, 64, ws, out_dtype=torch.float32),
              lambda: fptq.fptq_w4a8_linear(codes, scale, w, M, N, K, 64, ws, scratch=scratch),
              lambda: fptq.fptq_w4a8_linear(codes, scale, w, M, N, K, 64, ws, torch.empty((M, N), device="cuda"), torch.float32)):
        same(*both(f))


def test_what_is_refused(both):  # noqa: F811
    M, N, K = 20, 48, 300
    x, r, gain, w, ws = data(M, N, K)
    codes, scale, _ = fptq.fptq_norm_quantize8(x, r, gain)
    lin = lambda *a, **k: fptq.fptq_w4a8_linear(*a, **k)
    norm, gated = fptq.fptq_norm_quantize8, fptq.fptq_gated_quantize8
    for f, error in ((lambda: norm(x.float()), TypeError), (lambda: norm(x.cpu()), TypeError), (lambda: norm(x.t()), TypeError), (lambda: norm(x[0]), fptq.FptqError),
                     (lambda: norm(x, r[:, :-1].contiguous()), fptq.FptqError), (lambda: norm(x, r.float()), TypeError), (lambda: norm(x, None, gain[:-1].contiguous()), fptq.FptqError),
                     (lambda: norm(x, scale_mode=2), fptq.FptqError), (lambda: norm(x, eps=-1.0), fptq.FptqError), (lambda: norm(x, residual_out=r), fptq.FptqError),
                     (lambda: norm(x, r, residual_out=r[:-1]), fptq.FptqError), (lambda: norm(x, out=codes[:-1]), fptq.FptqError),
                     (lambda: norm(x, out=codes.view(torch.uint8)), TypeError), (lambda: norm(x, token_scale_out=scale[:-1]), fptq.FptqError),
                     (lambda: norm(torch.empty((0, 8), dtype=torch.bfloat16, device="cuda")), fptq.FptqError),
                     (lambda: gated(x, r[:-1]), fptq.FptqError), (lambda: gated(x, r.float()), TypeError), (lambda: gated(x.t(), r.t()), TypeError), (lambda: gated(x[0], r[0]), TypeError),
                     (lambda: gated(x, x[:1].expand(M, K)), fptq.FptqError),
                     (lambda: lin(codes, scale, w, M, N, K, 48, ws), fptq.FptqError), (lambda: lin(codes, scale, w, M, N, K, 0, ws), fptq.FptqError),
                     (lambda: lin(codes, scale, w, M, N, K, (1 << 64) + 128, ws), fptq.FptqError),
                     (lambda: lin(codes, scale, w, M, N, K, 32, ws), fptq.FptqError), (lambda: lin(codes, scale, w, M + 1, N, K, 64, ws), fptq.FptqError),
                     (lambda: lin(codes, scale, w, M, N + 1, K, 64, ws), fptq.FptqError), (lambda: lin(codes, scale[:-1], w, M, N, K, 64, ws), fptq.FptqError),
                     (lambda: lin(codes.view(torch.uint8), scale, w, M, N, K, 64, ws), TypeError), (lambda: lin(codes, scale.double(), w, M, N, K, 64, ws), TypeError),
                     (lambda: lin(codes, scale, w, M, N, K, 64, ws.to(torch.bfloat16)), TypeError), (lambda: lin(codes, scale, w, M, N, K, 64, ws, out_dtype=torch.float16), TypeError),
                     (lambda: lin(codes, scale, w, M, N, K, 64, ws, x[:, :1].contiguous()), fptq.FptqError), (lambda: lin(codes, scale, w, M, N, K, 64, ws, torch.empty((M, N), device="cuda")), TypeError),
                     (lambda: lin(codes, scale, w, M, N, K, 64, ws, scratch=scale), TypeError), (lambda: lin(codes, scale, w, 0, N, K, 64, ws), fptq.FptqError)):
        def refused():
            with pytest.raises(error):
                f()
        both(refused)
    torch.cuda.synchronize()


def test_another_stream_and_threads():
    """Calls on streams of their own, from threads of their own, with their own scratch: each as alone."""
    M, N, K = 100, 256, 14336
    x, r, gain, w, ws = data(M, N, K, 128)
    assert fptq.fptq_w4a8_linear_scratch_bytes(M, N, K, 128) > 0

    def chain(x):
        codes, scale, z = fptq.fptq_norm_quantize8(x, r, gain, eps=1e-5)
        c2, s2 = fptq.fptq_gated_quantize8(x, z)
        return fptq.fptq_w4a8_linear(codes, scale, w, M, N, K, 128, ws), fptq.fptq_w4a8_linear(c2, s2, w, M, N, K, 128, ws)
    inputs = [x.roll(i, 0) for i in range(4)]
    want = [chain(v) for v in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            for _ in range(20):
                got = chain(inputs[i])
            side.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                wrong.append(i)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
