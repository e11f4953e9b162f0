"""What the calls of 8-bit activations refuse: before any launch, so no GPU is needed."""
import ctypes

import pytest

from paper_2506_04985_amd import binding as fptq

P = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 1)
TWO = ctypes.c_void_p((1 << 20) + 2)
EIGHT = ctypes.c_void_p((1 << 20) + 8)
NULL, SHAPE, SIZE, MODE, VALUE, ALIGN = -1, -2, -3, -4, -6, -7


def refused(name, arguments, order, code, **changed):
    L = fptq.lib()
    assert not set(changed) - set(order)
    assert getattr(L, name)(*[changed.get(k, arguments[k]) for k in order]) == code, (name, changed)
    assert name.encode() in L.fptq_last_error()


NORM = dict(x=P, residual=P, gain=P, M=4, K=300, mode=1, eps=1e-5, out=P, nbytes=4 * 384, scale=P, z=P, stream=None)
GATED = dict(gate=P, up=P, M=4, K=300, gs=600, us=600, out=P, nbytes=4 * 384, scale=P, stream=None)
LINEAR = dict(x=P, s=P, w=P, M=4, N=5, K=300, group=64, ws=P, y=P, type=0, scratch=None, sbytes=0, stream=None)


@pytest.mark.parametrize("code,changed", [
    (NULL, dict(x=None)), (NULL, dict(out=None)), (NULL, dict(scale=None)), (SHAPE, dict(M=0)), (SHAPE, dict(K=0)), (SHAPE, dict(M=-1)), (SHAPE, dict(M=1 << 40)),
    (SIZE, dict(nbytes=4 * 384 - 1)), (SIZE, dict(nbytes=0)), (MODE, dict(mode=2)), (MODE, dict(mode=-1)), (MODE, dict(residual=None)),
    (VALUE, dict(eps=-1e-9)), (VALUE, dict(eps=float("nan"))), (VALUE, dict(eps=float("inf"))),
    (ALIGN, dict(x=ODD)), (ALIGN, dict(residual=ODD)), (ALIGN, dict(gain=ODD)), (ALIGN, dict(z=ODD)), (ALIGN, dict(out=EIGHT)), (ALIGN, dict(scale=TWO))])
def test_norm(code, changed):
    refused("fptq_norm_quantize8", NORM, list(NORM), code, **changed)


@pytest.mark.parametrize("code,changed", [
    (NULL, dict(gate=None)), (NULL, dict(up=None)), (NULL, dict(out=None)), (NULL, dict(scale=None)), (SHAPE, dict(M=0)), (SHAPE, dict(K=-3)),
    (SHAPE, dict(gs=299)), (SHAPE, dict(us=299)), (SHAPE, dict(us=-600)), (SHAPE, dict(gs=1 << 39)), (SIZE, dict(nbytes=1535)),
    (ALIGN, dict(gate=ODD)), (ALIGN, dict(up=ODD)), (ALIGN, dict(out=EIGHT)), (ALIGN, dict(scale=TWO))])
def test_gated(code, changed):
    refused("fptq_gated_quantize8", GATED, list(GATED), code, **changed)


@pytest.mark.parametrize("code,changed", [
    (NULL, dict(x=None)), (NULL, dict(s=None)), (NULL, dict(w=None)), (NULL, dict(ws=None)), (NULL, dict(y=None)),
    (SHAPE, dict(M=0)), (SHAPE, dict(N=0)), (SHAPE, dict(K=0)), (SHAPE, dict(M=1 << 25)), (SHAPE, dict(N=(1 << 24) + 1)), (SHAPE, dict(K=1 << 25)), (SHAPE, dict(M=1 << 24, N=(1 << 12) + 1)),
    (SHAPE, dict(group=0)), (SHAPE, dict(group=-128)), (SHAPE, dict(group=16)), (SHAPE, dict(group=96)), (SHAPE, dict(group=130)), (SHAPE, dict(group=192)),
    (MODE, dict(type=2)), (MODE, dict(type=-1)), (ALIGN, dict(x=EIGHT)), (ALIGN, dict(w=EIGHT)), (ALIGN, dict(y=EIGHT)), (ALIGN, dict(s=TWO)), (ALIGN, dict(ws=TWO)),
    (SIZE, dict(sbytes=-1)), (ALIGN, dict(scratch=EIGHT, sbytes=1 << 20))])
def test_linear(code, changed):
    refused("fptq_w4a8_linear", LINEAR, list(LINEAR), code, **changed)


def test_sizes_and_unpack():
    L = fptq.lib()
    assert L.fptq_packed8_bytes(1, 1) == 128 and L.fptq_packed8_bytes(10, 129) == 2560 and L.fptq_packed8_bytes(8192, 28672) == 8192 * 28672
    assert L.fptq_packed8_bytes(0, 1) == SHAPE and L.fptq_packed8_bytes(1, -1) == SHAPE
    assert L.fptq_unpack8(None, 1, 1, P, None) == NULL and L.fptq_unpack8(P, 1, 1, None, None) == NULL
    assert L.fptq_unpack8(P, 0, 1, P, None) == SHAPE and L.fptq_unpack8(EIGHT, 1, 1, P, None) == ALIGN


def test_kernel_choice_is_host_arithmetic():
    """On 256 CUs: a few-token kernel up to 16 tokens by two lines, then the least of the fitted times."""
    L = fptq.lib()
    for bad in ((-1, 1), (15, 1), (3, 0), (3, 9)):
        assert L.fptq_set_grouped_kernel(*bad) == VALUE
    assert L.fptq_w4a8_linear_scratch_bytes(0, 1, 1, 128) == SHAPE and L.fptq_w4a8_linear_scratch_bytes(64, 64, 64, 100) == SHAPE
    for M, N, K in ((1, 4096, 14336), (16, 4096, 14336), (64, 28672, 4096), (4096, 28672, 4096), (1000, 4096, 14336)):
        assert L.fptq_w4a8_linear_scratch_bytes(M, N, K, 128) == 0
    of = L.fptq_grouped_kernel
    assert of(0, 1, 1, 32) == SHAPE and of(1, 1, 1, 0) == SHAPE
    assert of(1, 4096, 4096, 128) == 11 and of(1, 6144, 4096, 128) == 12 and of(8, 128256, 4096, 64) == 13 and of(12, 28672, 14336, 128) == 12
    assert of(16, 28672, 14336, 128) == 8 and of(16, 28672, 14336, 32) == 10 and of(3, 4096, 512, 128) == 14
    assert of(4096, 28672, 4096, 128) == 1 and of(333, 32003, 2504, 64) == 2 and of(1000, 4096, 14336, 128) == 5 and of(32, 28672, 4096, 128) == 8
    for M in (17, 64, 65, 500, 3000):
        for N in (64, 1000, 5000, 40000):
            for K in (128, 1000, 8000):
                assert of(M, N, K, 32) not in (1, 3, 5) and 1 <= of(M, N, K, 128) <= (13 if M <= 64 else 10)


@pytest.mark.parametrize("M,N,K,group", [(4, 5, 300, 33), (4, 5, 300, 96), (4, 5, 300, 130), ((1 << 24) + 1, 5, 300, 64), (4, 1 << 25, 300, 64), (4, 5, 1 << 25, 64), (1 << 24, (1 << 12) + 1, 300, 64),
                                         (1 << 40, 1, 300, 64)])
def test_no_kernel_is_named_for_a_call_that_is_refused(M, N, K, group):
    L = fptq.lib()
    assert L.fptq_w4a8_linear(*[dict(LINEAR, M=M, N=N, K=K, group=group)[k] for k in LINEAR]) == SHAPE
    assert L.fptq_grouped_kernel(M, N, K, group) == SHAPE and b"fptq_grouped_kernel" in L.fptq_last_error()
