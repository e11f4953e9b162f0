"""fptq_cached_attention against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from attention_util import PAGE, check, device, host, paged, projection, starts
from oracle import attention as oracle
from paper_2506_04985_amd import binding as fptq

pytestmark = pytest.mark.gpu


def filled(lengths, J, D, seed, poison=True):
    """A cache of random codes; what lies past the lengths is NaN, pages of no sequence too."""
    rng = np.random.default_rng(seed)
    table, pool = paged(lengths, seed=seed)
    codes = rng.integers(0, 256, (2, pool, J, PAGE, D), dtype=np.uint8)
    codes[(codes & 127) == 127] ^= 1
    scales = np.exp2(rng.integers(-8, -5, (2, pool, J))).astype(np.float32)
    used = np.zeros(pool, int)
    for b, n in enumerate(lengths):
        for p in range(-(-n // PAGE)):
            used[table[b, p]] = min(PAGE, n - p * PAGE)
    if poison:
        for p in range(pool):
            codes[:, p, :, used[p]:] = 127
            if used[p] == 0:
                scales[:, p] = np.nan
    return table, codes, scales


def cache_of(codes, scales):
    k = np.stack([[oracle.keys_page(x) for x in page] for page in codes[0]])
    v = np.stack([[oracle.values_page(x) for x in page] for page in codes[1]])
    return fptq.Cache(*(torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (k, v, scales[0], scales[1])))


def tokens_of(table_row, codes, scales, length):
    """keys and values [length, J, D] in 64 bits"""
    x = oracle.e4m3_values()[codes[:, table_row[:-(-length // PAGE)]]] * scales[:, table_row[:-(-length // PAGE)], :, None, None].astype(np.float64)
    x = x.transpose(0, 1, 3, 2, 4).reshape(2, -1, codes.shape[2], codes.shape[4])
    return x[0, :length], x[1, :length]


def expected(q, new, lengths, table, codes, scales, scale):
    parts = []
    for b, (s, e) in enumerate(zip(starts(new), starts(new)[1:])):
        k, v = tokens_of(table[b], codes, scales, lengths[b])
        parts.append(oracle.attention(host(q[s:e]), k, v, scale))
    return [np.concatenate([p[i] for p in parts]) for i in range(3)]


def run(new, lengths, H, J, D, seed=0, with_cu=True, **more):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, _, _ = projection(g, sum(new), H, J, D)
    table, codes, scales = filled(lengths, J, D, seed)
    out = fptq.fptq_cached_attention(q, cache_of(codes, scales), device(table), device(lengths), device(starts(new)) if with_cu else None, **more)
    check(out, *expected(q, new, lengths, table, codes, scales, D ** -0.5), D)


@pytest.mark.parametrize("H,J,D", [(4, 2, 128), (3, 3, 64), (7, 1, 64), (16, 1, 128), (40, 1, 64), (40, 2, 128)])
@pytest.mark.parametrize("lengths", [[1], [63, 64, 65], [2, 300, 129, 1]])
def test_one_token_each(lengths, H, J, D):
    run([1] * len(lengths), lengths, H, J, D, seed=H + len(lengths), with_cu=False)


@pytest.mark.parametrize("H,J,D", [(4, 2, 128), (5, 1, 64), (16, 1, 128)])
@pytest.mark.parametrize("new,lengths", [([4], [4]), ([2, 0, 5], [200, 70, 5]), ([1, 9], [64, 65]), ([0, 3], [0, 67]), ([70], [130])])
def test_several_tokens_each(new, lengths, H, J, D):
    run(new, lengths, H, J, D, seed=H + sum(new))


@pytest.mark.parametrize("H,J,D,new,lengths", [(4, 1, 64, [1], [5000]), (8, 2, 128, [1, 1, 1], [4200, 40, 6000]), (4, 1, 64, [6, 2], [4097, 9000]),
                                               (16, 1, 128, [5, 1, 0], [4500, 5000, 90]), (6, 2, 128, [1] * 70, [1100] * 69 + [2100])])
def test_long_sequences_shared_out_and_not(H, J, D, new, lengths):
    """More than 16 pages are cut into parts where there are few.  Without scratch they are not; both are within the bound, and the parts' own order is the same every time."""
    run(new, lengths, H, J, D, seed=1)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, _, _ = projection(g, sum(new), H, J, D)
    table, codes, scales = filled(lengths, J, D, 1)
    cache, cu = cache_of(codes, scales), device(starts(new))
    n = fptq.fptq_cached_attention_scratch_bytes(sum(new), len(new), H, J, D, table.shape[1])
    assert n > 0
    want = expected(q, new, lengths, table, codes, scales, D ** -0.5)
    whole = fptq.fptq_cached_attention(q, cache, device(table), device(lengths), cu, scratch=torch.empty(256, dtype=torch.uint8, device="cuda"))
    check(whole, *want, D)
    scratch = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")               # NaN wherever it is read unwritten
    outs = [fptq.fptq_cached_attention(q, cache, device(table), device(lengths), cu, scratch=scratch) for _ in range(3)]
    check(outs[0], *want, D)
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_very_many_short_and_long_sequences():
    rng = np.random.default_rng(3)
    lengths = [int(n) for n in rng.integers(1, 200, 150)]
    lengths[70], lengths[149] = 4500, 4700
    run([1] * 150, lengths, 4, 2, 64, seed=3, with_cu=False)


@pytest.mark.parametrize("H,J,D,tokens", [(8, 8, 64, 1), (16, 1, 128, 2)])
def test_a_wide_table_of_short_sequences(H, J, D, tokens):
    """Room for many more parts than there are."""
    lengths, new = [100, 70, 1, 4100] * 4, [tokens] * 16
    g = torch.Generator(device="cuda").manual_seed(3)
    q, _, _ = projection(g, sum(new), H, J, D)
    table, codes, scales = filled(lengths, J, D, 3)
    wide = np.full((16, 5000), -1, np.int32)
    wide[:, :table.shape[1]] = table
    out = fptq.fptq_cached_attention(q, cache_of(codes, scales), device(wide), device(lengths), device(starts(new)) if tokens > 1 else None)
    check(out, *expected(q, new, lengths, table, codes, scales, D ** -0.5), D)


@pytest.mark.parametrize("H,J,D,B", [(8, 1, 64, 5), (12, 4, 128, 33), (9, 3, 64, 70), (20, 1, 128, 3), (40, 40, 64, 2)])
@pytest.mark.parametrize("tokens", [1, 3])
def test_no_row_behind_the_tokens_is_written(H, J, D, B, tokens):
    """The host's bound of row tiles is higher than their number where a tile is not full: there is no sequence, and no output, behind the last."""
    lengths, new = [7 + 13 * b % 90 for b in range(B)], [tokens] * B
    g = torch.Generator(device="cuda").manual_seed(B)
    q, _, _ = projection(g, sum(new), H, J, D)
    table, codes, scales = filled(lengths, J, D, B)
    out = torch.full((4 * B * tokens + 64, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    fptq.fptq_cached_attention(q, cache_of(codes, scales), device(table), device(lengths), device(starts(new)) if tokens > 1 else None, out=out)
    check(out[:sum(new)], *expected(q, new, lengths, table, codes, scales, D ** -0.5), D)
    assert (out[sum(new):] == 7).all()


def test_tokens_before_the_first_key_get_zeros():
    g = torch.Generator(device="cuda").manual_seed(4)
    q, _, _ = projection(g, 9, 4, 2, 64)
    lengths, new = [3, 0, 2], [5, 2, 2]
    table, codes, scales = filled(lengths, 2, 64, 4)
    out = fptq.fptq_cached_attention(q, cache_of(codes, scales), device(table), device(lengths), device(starts(new)))
    check(out, *expected(q, new, lengths, table, codes, scales, 0.125), 64)
    assert (out[:2] == 0).all() and (out[5:7] == 0).all() and (out[2:5] != 0).any()


@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_value_reaches_only_those_who_see_it(D):
    g = torch.Generator(device="cuda").manual_seed(5)
    q, _, _ = projection(g, 40, 4, 1, D)
    table, codes, scales = filled([100], 1, D, 5)
    codes[1, table[0, 1], 0, 80 - PAGE, 9] = 0xFF                       # the value of token 80: tokens 60 .. 79 do not see it
    out = host(fptq.fptq_cached_attention(q, cache_of(codes, scales), device(table), device([100]), device([0, 40])))
    assert np.isnan(out[20:, :, 9]).all() and np.isfinite(out[:20]).all()
    assert np.isfinite(np.delete(out[20:], 9, axis=2)).all()
    codes[0, table[0, 1], 0, 90 - PAGE, 3] = 0x7F                       # a key
    out = host(fptq.fptq_cached_attention(q, cache_of(codes, scales), device(table), device([100]), device([0, 40])))
    assert np.isnan(out[30:]).all() and np.isfinite(out[:20]).all()


def test_page_numbers_outside_the_pool_are_not_seen():
    g = torch.Generator(device="cuda").manual_seed(6)
    q, _, _ = projection(g, 2, 4, 2, 64)
    lengths = [300, 130]
    table, codes, scales = filled(lengths, 2, 64, 6)
    pool = codes.shape[1]
    bad = table.copy()
    bad[0, 1], bad[0, 3], bad[1, 0] = -1, pool, 0x7FFFFFFF
    out = fptq.fptq_cached_attention(q, cache_of(codes, scales), device(bad), device(lengths))
    for b, keep in ((0, [0, 2, 4]), (1, [1, 2])):
        k, v = tokens_of(table[b], codes, scales, lengths[b])
        seen = np.isin(np.arange(lengths[b]) // PAGE, keep)
        check(out[b:b + 1], *oracle.attention(host(q[b:b + 1]), k[seen], v[seen], 0.125), 64)


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), 0.0])
@pytest.mark.parametrize("H,J,D,tokens,more", [(4, 2, 64, 1, 0), (16, 1, 128, 1, 0), (8, 1, 64, 4, 0), (40, 2, 128, 1, 0), (4, 1, 64, 1, 40)])
def test_page_numbers_outside_the_pool_whatever_the_first_page_holds(scale, H, J, D, tokens, more):
    """Page 0 belongs to nobody, and neither its codes nor its scales were ever written: pages that are not there take nothing of it."""
    g = torch.Generator(device="cuda").manual_seed(12)
    q, _, _ = projection(g, 2 * tokens, H, J, D)
    lengths = [300 + more * PAGE, 130]
    table, codes, scales = filled(lengths, J, D, 12)
    codes = np.concatenate([np.full_like(codes[:, :1], 127), codes], 1)
    scales = np.concatenate([np.full_like(scales[:, :1], scale), scales], 1)
    table += 1
    pool = codes.shape[1]
    bad = table.copy()
    bad[0, 1], bad[0, 3], bad[1, 0] = -1, pool, 0x7FFFFFFF
    out = fptq.fptq_cached_attention(q, cache_of(codes, scales), device(bad), device(lengths), device([0, tokens, 2 * tokens]) if tokens > 1 else None)
    for b, gone in ((0, [1, 3]), (1, [0])):
        k, v = tokens_of(table[b], codes, scales, lengths[b])
        seen = ~np.isin(np.arange(lengths[b]) // PAGE, gone)
        rows = slice(b * tokens, (b + 1) * tokens)
        check(out[rows], *oracle.attention(host(q[rows]), k[seen], v[seen], D ** -0.5), D)


def test_a_length_beyond_the_table():
    g = torch.Generator(device="cuda").manual_seed(7)
    q, _, _ = projection(g, 1, 2, 2, 64)
    table, codes, scales = filled([128], 2, 64, 7)
    out = fptq.fptq_cached_attention(q, cache_of(codes, scales), device(np.ascontiguousarray(table[:, :2])), device([100000]))
    k, v = tokens_of(table[0], codes, scales, 128)
    check(out, *oracle.attention(host(q), k, v, 0.125), 64)


def test_pages_past_32_bits():
    """A pool of more than 4 GB of codes each, of which the last pages are used."""
    J, D, pool = 8, 128, 66000
    lengths = [200]
    table, codes, scales = filled(lengths, J, D, 8)
    small = cache_of(codes, scales)
    big = fptq.Cache.empty(pool, J, D)
    n = small.key_codes.shape[0]
    for to, x in ((big.key_codes, small.key_codes), (big.value_codes, small.value_codes), (big.key_scales, small.key_scales), (big.value_scales, small.value_scales)):
        to[pool - n:] = x
    g = torch.Generator(device="cuda").manual_seed(8)
    q, _, _ = projection(g, 1, 16, J, D)
    high = np.where((table >= 0) & (table < n), table + (pool - n), table + pool).astype(np.int32)
    out = fptq.fptq_cached_attention(q, big, device(high), device(lengths))
    check(out, *expected(q, [1], lengths, table, codes, scales, D ** -0.5), D)


def test_replays_of_a_captured_call_follow_growing_lengths():
    J, D, H = 2, 128, 8
    table, codes, scales = filled([4800, 700], J, D, 9, poison=False)
    cache = cache_of(codes, scales)
    q = torch.empty((2, H, D), dtype=torch.bfloat16, device="cuda")
    t, lengths, out = device(table), device([1, 1]), torch.empty((2, H, D), dtype=torch.bfloat16, device="cuda")
    fptq.fptq_init()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        fptq.fptq_cached_attention(q, cache, t, lengths, out=out)
    g = torch.Generator(device="cuda").manual_seed(9)
    for a, b in ((1, 700), (4097, 64), (4800, 0), (4799, 699)):
        q.copy_(torch.randn(q.shape, device="cuda", generator=g).to(torch.bfloat16))
        lengths.copy_(device([a, b]))
        want = fptq.fptq_cached_attention(q, cache, t, lengths)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        check(out, *expected(q, [1, 1], [a, b], table, codes, scales, D ** -0.5), D)


@pytest.mark.parametrize("H,D,tokens", [(1, 64, 1), (4, 128, 1), (8, 64, 5), (20, 128, 3)])
@pytest.mark.parametrize("order", ["rising", "falling"])
def test_the_largest_scores_served(order, H, D, tokens):
    """Scores of up to 4.9 * 10^8, all of e4m3's positive values apart: all weight is on the largest one seen.  Its weight is rounded to bf16, its sum is not, and
    the output is rounded."""
    length = 126
    table, codes, scales = filled([length], 1, D, 14)
    flat = np.zeros((2, 1, PAGE, D), np.uint8)
    flat[0, 0, :, 5], flat[1, 0, :62, 5] = np.arange(1, 65), np.arange(65, 127)
    if order == "falling":
        flat[0, 0, :, 5], flat[1, 0, :62, 5] = np.arange(126, 62, -1), np.arange(62, 0, -1)
    codes[0, table[0, :2]], scales[0] = flat, 1.0
    q = torch.zeros((tokens, H, D), dtype=torch.bfloat16, device="cuda")
    q[..., 5] = 2.0 ** 20
    out = host(fptq.fptq_cached_attention(q, cache_of(codes, scales), device(table), device([length]), device([0, tokens]) if tokens > 1 else None, scale=1.04))
    _, v = tokens_of(table[0], codes, scales, length)
    want = v[length - tokens:] if order == "rising" else np.broadcast_to(v[:1], (tokens, 1, D))
    np.testing.assert_allclose(out, np.broadcast_to(want, (tokens, H, D)), rtol=1.01 * 2 * 2.0 ** -8)
