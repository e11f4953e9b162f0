"""Products of 8-bit codes with packed 4-bit weights in groups, against the oracle's in 64 bits.

How far an output may be: the integer sums are exact; each of the terms (a group's sum, or 128 values') goes into the fp32 sum by one fused multiply-add, and up to 16 waves' sums are added:
(terms + 16) roundings of 2^-24 of at most `mass`, what the magnitudes of the terms add up to; the token's scale once more; bf16 rounds by 2^-8 of the result."""
import numpy as np
import pytest
import torch

from oracle import grouped
from paper_2506_04985_amd import binding as fptq

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def draw(M, N, K, group, seed=0, zeros=False):
    rng = np.random.default_rng([M, N, K, group, seed])
    codes = rng.integers(-127, 128, (M, K), dtype=np.int8)
    w = rng.integers(-8, 8, (N, K), dtype=np.int8)
    s = np.exp(rng.normal(-4, 1, M)).astype(np.float32)
    ws = (np.exp(rng.normal(-5, 1, (-(-K // group), N))) * rng.choice([-1.0, 1.0, 1.0, 1.0], (-(-K // group), N))).astype(np.float32)
    return codes, s, w, ws


def tolerance(y, mass, K, group, bf16):
    terms = -(-K // min(group, 128))
    return 1.01 * ((terms + 18) * 2.0 ** -24 * mass + (2.0 ** -8 * np.abs(y) if bf16 else 0)) + 1e-37


def run(codes, s, w, ws, group, dtype=torch.float32, out=None, scratch=None):
    (M, K), N = codes.shape, w.shape[0]
    return fptq.fptq_w4a8_linear(dev(grouped.lay_out(codes)), dev(s), fptq.fptq_pack_weights(dev(w)), M, N, K, group, dev(ws), out=out, out_dtype=dtype, scratch=scratch)


def check(got, y, mass, K, group):
    bf16 = got.dtype == torch.bfloat16
    far = np.abs(got.cpu().double().numpy() - y) / tolerance(y, mass, K, group, bf16)
    assert got.shape == y.shape and far.max() <= 1.0, f"{far.max()} of the bound at {np.unravel_index(far.argmax(), far.shape)}"


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 17, 130), (2, 3, 31), (5, 40, 33), (16, 64, 256), (17, 100, 1000), (1, 6144, 4096), (31, 33, 65), (33, 48, 640), (64, 257, 2504),
          (65, 65, 129), (100, 300, 383), (128, 128, 128), (129, 256, 1024), (200, 520, 96), (256, 256, 512), (257, 130, 1111), (300, 1000, 777), (513, 264, 1536), (777, 333, 500)]


@pytest.mark.parametrize("group", [32, 64, 128, 256, 384])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_products(M, N, K, group):
    case = draw(M, N, K, group)
    y, mass = grouped.linear(*case[:3], group, case[3])
    check(run(*case, group), y, mass, K, group)
    check(run(*case, group, torch.bfloat16), y, mass, K, group)


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("M,N,K", [(2600, 5200, 200), (3500, 3601, 100), (300, 26000, 129)])
def test_products_of_many_tiles(M, N, K, group):
    case = draw(M, N, K, group)
    y, mass = grouped.linear(*case[:3], group, case[3])
    check(run(*case, group), y, mass, K, group)
    check(run(*case, group, torch.bfloat16), y, mass, K, group)


@pytest.fixture
def forced():
    yield fptq.fptq_set_grouped_kernel
    fptq.fptq_set_grouped_kernel(0)


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("kernel", range(1, 15))
def test_every_kernel(kernel, group, forced):
    """Each kernel on sizes that cut its tiles, sets of K tiles and groups; a single K tile, fewer than it has sets, and many."""
    for M, N, K in ((1, 1, 1), (70, 90, 100), (33, 257, 640), (300, 520, 1100), (257, 129, 2600), (5, 64, 129)):
        case = draw(M, N, K, group, kernel)
        y, mass = grouped.linear(*case[:3], group, case[3])
        forced(kernel)
        if group == 32 and kernel in (1, 3, 5):
            with pytest.raises(fptq.FptqError):
                run(*case, group)
            continue
        check(run(*case, group), y, mass, K, group)
        check(run(*case, group, torch.bfloat16), y, mass, K, group)


@pytest.mark.parametrize("splits", [2, 3, 8])
@pytest.mark.parametrize("kernel,group", [(k, g) for k in range(1, 11) for g in (32, 64, 128, 256) if g != 32 or k not in (1, 3, 5)])
def test_ranges_of_k(kernel, group, splits, forced):
    """K cut between workgroups: ranges of several K tiles, of one, and without any; a caller's scratch, more than needed and full of NaN."""
    for M, N, K in ((70, 90, 100), (33, 257, 1100), (257, 129, 2600)):
        case = draw(M, N, K, group, kernel)
        y, mass = grouped.linear(*case[:3], group, case[3])
        forced(kernel, splits)
        need = fptq.fptq_w4a8_linear_scratch_bytes(M, N, K, group)
        assert need == (splits * M * ((N + 3) // 4 * 16) if splits <= -(-K // 128) else 0)
        got = run(*case, group)
        check(got, y, mass, K, group)
        check(run(*case, group, torch.bfloat16), y, mass, K, group)
        scratch = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
        assert torch.equal(run(*case, group, scratch=scratch), got) and bool((scratch[need:] == 255).all())
        check(run(*case, group, scratch=scratch[:256]), y, mass, K, group)          # too small: as without


@pytest.mark.parametrize("M", [1, 40, 300])
def test_one_scale_a_channel(M):
    N, K = 96, 700
    case = draw(M, N, K, 768)
    y, mass = grouped.linear(*case[:3], 768, case[3])
    for group in (768, 1 << 20, (1 << 63) - 128):
        check(run(*case, group), y, mass, K, 768)


@pytest.mark.parametrize("M,N,K,group", [(1, 64, 512, 128), (8, 80, 300, 32), (50, 96, 640, 64), (200, 130, 1000, 64), (600, 520, 2000, 128), (300, 264, 999, 32)])
def test_results_are_exact_where_fp32_holds_them(M, N, K, group):
    """Scales that are powers of two within 2^4 of each other: every partial sum is a multiple of one unit below 2^24 of it, so no rounding may be seen anywhere.  Also
    the ends of both grids."""
    rng = np.random.default_rng(K)
    codes, w = rng.integers(-2, 3, (M, K), dtype=np.int8), rng.integers(-8, 8, (N, K), dtype=np.int8)
    ws = np.exp2(rng.integers(-2, 2, (-(-K // group), N))).astype(np.float32)
    s = np.exp2(rng.integers(-3, 3, M)).astype(np.float32)
    y, _ = grouped.linear(codes, s, w, group, ws)
    assert np.array_equal(run(codes, s, w, ws, group).cpu().double().numpy(), y)
    codes[:], w[:] = 127, -8
    w[::2] = 7
    codes[::3] = -127
    y, mass = grouped.linear(codes, s, w, group, ws)
    check(run(codes, s, w, ws, group), y, mass, K, group)


@pytest.mark.parametrize("M,N,K,group", [(3, 40, 256, 64), (40, 40, 256, 128), (300, 200, 384, 32)])
def test_rows_that_are_not_numbers_stay_by_themselves(M, N, K, group):
    codes, s, w, ws = draw(M, N, K, group)
    want = run(codes, s, w, ws, group, torch.bfloat16)
    s[1] = np.nan
    got = run(codes, s, w, ws, group, torch.bfloat16)
    assert bool(torch.isnan(got[1]).all())
    keep = torch.arange(M, device="cuda") != 1
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("M,N,K,group", [(1, 33, 200, 64), (30, 65, 300, 32), (130, 70, 500, 128), (515, 391, 260, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nothing_is_written_behind_the_last_row(M, N, K, group, dtype):
    case = draw(M, N, K, group)
    whole = torch.full((M * N + 4096,), 7.0, dtype=dtype, device="cuda")
    got = run(*case, group, dtype, out=whole[:M * N].view(M, N))
    assert bool((whole[M * N:] == 7.0).all()) and torch.equal(got, run(*case, group, dtype))


@pytest.mark.parametrize("kernel,M,N,K", [(12, 3, 131077, 65664), (5, 40, 131077, 65664), (1, 70001, 32003, 130), (10, 70001, 35, 61500)])
def test_arrays_beyond_32_bits(kernel, M, N, K, forced):
    """More than 2^32 bytes of weights, of outputs or of codes: the first and last rows and channels are what the same kernel makes of them alone, bit by bit."""
    tiles = -(-K // 128)
    x = torch.randint(-127, 128, (tiles, M, 128), dtype=torch.int8, device="cuda")
    w = torch.randint(0, 256, (tiles, N, 64), dtype=torch.uint8, device="cuda")
    s, ws = torch.rand((M,), device="cuda"), torch.rand((tiles, N), device="cuda")
    forced(kernel)
    y = fptq.fptq_w4a8_linear(x, s, w, M, N, K, 128, ws)
    assert max(x.numel(), w.numel(), 2 * y.numel()) > 2 ** 32
    for rows in (slice(0, min(M, 300)), slice(max(M - 300, 0), M)):
        for channels in (slice(0, min(N, 600)), slice(max(N - 600, 0), N)):
            xs, wss, scales = x[:, rows].contiguous(), w[:, channels].contiguous(), ws[:, channels].contiguous()
            part = fptq.fptq_w4a8_linear(xs, s[rows].clone(), wss, xs.shape[1], wss.shape[1], K, 128, scales)
            assert torch.equal(y[rows, channels], part)


def test_the_same_call_gives_the_same_bits():
    for M, N, K, group in ((1, 500, 4096, 128), (48, 300, 3000, 32), (400, 500, 2000, 64)):
        case = draw(M, N, K, group)
        first = run(*case, group)
        assert all(torch.equal(first, run(*case, group)) for _ in range(5))


def test_a_run_of_them_as_a_layer_makes_it():
    """Norm to 8 bits, gate+up, gated activation to 8 bits, down: each step against the oracle on what the step before it gave."""
    g = torch.Generator(device="cuda").manual_seed(0)
    host = lambda t: t.detach().cpu().float().numpy()
    for M in (1, 33, 300):
        K, F, group = 320, 448, 64
        x, r = (torch.randn((M, K), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
        gain = (1 + 0.1 * torch.randn((K,), device="cuda", generator=g)).to(torch.bfloat16)
        w1, w2 = (torch.randint(-8, 8, s, dtype=torch.int8, device="cuda", generator=g) for s in ((2 * F, K), (K, F)))
        s1, s2 = (0.01 * torch.rand(s, device="cuda", generator=g) for s in ((-(-K // group), 2 * F), (-(-F // group), K)))
        codes, scale, z = fptq.fptq_norm_quantize8(x, r, gain, eps=1e-5)
        h = fptq.fptq_w4a8_linear(codes, scale, fptq.fptq_pack_weights(w1), M, 2 * F, K, group, s1)
        c2, t2 = fptq.fptq_gated_quantize8(*h.split(F, 1))
        y = fptq.fptq_w4a8_linear(c2, t2, fptq.fptq_pack_weights(w2), M, K, F, group, s2)
        want, mass = grouped.linear(fptq.fptq_unpack8(codes, M, K).cpu().numpy(), scale.cpu().numpy(), w1.cpu().numpy(), group, s1.cpu().numpy())
        check(h, want, mass, K, group)
        q, t = grouped.quantize_rows(grouped.gated(host(h[:, :F]), host(h[:, F:])))
        assert np.array_equal(fptq.fptq_unpack8(c2, M, F).cpu().numpy(), q) and np.array_equal(t2.cpu().numpy(), t)
        want, mass = grouped.linear(q, t, w2.cpu().numpy(), group, s2.cpu().numpy())
        check(y, want, mass, F, group)


@pytest.mark.parametrize("kernel,splits", [(k, 1) for k in range(1, 15)] + [(1, 2), (8, 3)])
@pytest.mark.parametrize("group", [64, 128])
def test_subnormal_scales_keep_their_bits(kernel, splits, group, forced):
    """Token scales of 2^-130 and below with bits down to fp32's last, against sums of 2^16 and more: every output is a number that fp32 holds.  And sums that are tiny behind large scales."""
    M, N, K = 70, 96, 640
    rng = np.random.default_rng(kernel)
    codes, w = np.zeros((M, K), np.int8), np.zeros((N, K), np.int8)
    codes[:, 3], codes[np.arange(M), 128 + np.arange(M)] = 1, rng.integers(-3, 4, M)
    w[:, 3], w[:, 128:128 + M] = rng.integers(1, 4, N), 1
    ws = np.full((-(-K // group), N), 2.0 ** 16, np.float32)
    s = (2.0 ** -130 * (1 + rng.integers(0, 1 << 19, M) * 2.0 ** -19)).astype(np.float32)
    s[::7], s[1::7], s[2::7] = 2.0 ** -149, 2.0 ** -122, 2.0 ** -122 * (1 + 2.0 ** -20)
    y, _ = grouped.linear(codes, s, w, group, ws)
    assert np.array_equal(y, y.astype(np.float32))
    forced(kernel, splits)
    assert np.array_equal(run(codes, s, w, ws, group).cpu().double().numpy(), y)
    s, ws = np.full(M, 2.0 ** 100, np.float32), np.full_like(ws, 2.0 ** -140)
    y, _ = grouped.linear(codes, s, w, group, ws)
    assert np.array_equal(run(codes, s, w, ws, group).cpu().double().numpy(), y)


@pytest.mark.parametrize("M,N,K,group", [(24, 4096, 14336, 128), (64, 2048, 16384, 64), (100, 1000, 16000, 32), (130, 2048, 28672, 128), (33, 300, 16384, 128)])
def test_scratch_that_is_too_small_counts_as_none(M, N, K, group):
    """Bit by bit, however little is missing: no call takes as many ranges as happen to fit."""
    tiles, g = -(-K // 128), torch.Generator(device="cuda").manual_seed(M)
    x = torch.randint(-127, 128, (tiles * M * 128,), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(0, 256, (tiles * N * 64,), dtype=torch.uint8, device="cuda", generator=g)
    s, ws = torch.rand((M,), device="cuda", generator=g), torch.rand((-(-K // group), N), device="cuda", generator=g)
    need = fptq.fptq_w4a8_linear_scratch_bytes(M, N, K, group)
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    assert need > 0

    def call(bytes, null=False):
        y = torch.empty((M, N), device="cuda")
        fptq._check(fptq.lib().fptq_w4a8_linear(fptq._ptr(x), fptq._ptr(s), fptq._ptr(w), M, N, K, group, fptq._ptr(ws), fptq._ptr(y), 1, None if null else fptq._ptr(scratch), bytes,
                                                fptq._stream()))
        return y
    without = call(0, null=True)
    assert torch.equal(call(need, null=True), without) and torch.equal(call(0), without)
    for bytes in (need - 1, need - 1 - need // 4, need // 2, need // 3):
        assert torch.equal(call(bytes), without)
    assert not bool(scratch.any())
    call(need)
    assert bool(scratch.any())
