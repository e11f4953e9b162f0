"""Calls of the attention operators with more of something than one turn of a kernel's loop takes: pages of a wave, units, cut units, parts of a unit, tokens.
Against the oracle in 64 bits; sequences share pages here (which a cache that is only read allows), so that the host has little to make."""
import numpy as np
import pytest
import torch

from attention_util import PAGE, check, device, host, projection, starts
from oracle import attention as oracle
from paper_2506_04985_amd import binding as fptq
from test_gpu_cache_append import run as run_append
from test_gpu_cached_attention import cache_of, run as run_cached

pytestmark = pytest.mark.gpu

POOL = 24


@pytest.fixture(autouse=True, scope="module")
def memory_given_back():
    """Scratch of 50 MiB here would stay in torch's cache, and a small tensor of a later test in such a segment keeps it: tests/test_gpu_binding.py, which limits
    the memory, counts on no segment in use having that much left."""
    yield
    torch.cuda.empty_cache()


def pool_of(J, D, seed):
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 256, (2, POOL, J, PAGE, D), dtype=np.uint8)
    codes[(codes & 127) == 127] ^= 1
    return codes, np.exp2(rng.integers(-8, -5, (2, POOL, J))).astype(np.float32)


def table_of(lengths, width, seed):
    rng = np.random.default_rng(seed)
    table = np.full((len(lengths), width), -1, np.int32)
    for b, n in enumerate(lengths):
        need = -(-n // PAGE)
        table[b, :need] = rng.integers(0, POOL, need)
    return table


def expected(q, row, length, codes, scales):
    """Attention of a sequence's last tokens q [n, H, D] over the pages of its table's row: a token of the pool counts as often as it is seen."""
    (n, H, D), J = q.shape, codes.shape[2]
    k, v = oracle.e4m3_values()[codes] * scales[..., None, None].astype(np.float64)          # [POOL, J, PAGE, D]
    out, mass, terms = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H))
    for i in range(n):
        seen = length - n + 1 + i
        times = np.repeat(np.bincount(row[:seen // PAGE], minlength=POOL)[:, None], PAGE, 1).astype(np.float64)
        if seen % PAGE:
            times[row[seen // PAGE], :seen % PAGE] += 1
        times = times.reshape(-1)
        for h in range(H):
            kk, vv = k[:, h // (H // J)].reshape(-1, D), v[:, h // (H // J)].reshape(-1, D)
            s = D ** -0.5 * (kk @ q[i, h])
            p = np.where(times > 0, times * np.exp(s - s[times > 0].max()), 0.0)
            out[i, h], mass[i, h] = p @ vv / p.sum(), p @ np.abs(vv) / p.sum()
            terms[i, h] = D ** -0.5 * (np.abs(kk) @ np.abs(q[i, h]))[times > 0].max()
    return out, mass, terms


def test_the_oracle_of_shared_pages():
    """Counting what is seen several times is the same as listing it."""
    codes, scales = pool_of(2, 64, 0)
    row, q = table_of([300], 6, 0)[0], np.random.default_rng(0).normal(size=(3, 4, 64))
    k, v = (oracle.e4m3_values()[codes[w, row[:5]]] * scales[w, row[:5], :, None, None].astype(np.float64) for w in (0, 1))
    k, v = (x.transpose(0, 2, 1, 3).reshape(-1, 2, 64)[:300] for x in (k, v))
    for a, b in zip(expected(q, row, 300, codes, scales), oracle.attention(q, k, v, 0.125)):
        np.testing.assert_allclose(a, b, rtol=1e-12, atol=1e-14)


def few(kinds, B, lengths, width, tokens, H, J, D, with_cu, seed, scratch=None):
    """A call of B sequences of `kinds` kinds in turn: the first of each kind against the oracle, the others, which see the same pages in the same
    parts, bit by bit against the first."""
    codes, scales = pool_of(J, D, seed)
    table = table_of(lengths[:kinds], width, seed)[np.arange(B) % kinds]
    lengths = [lengths[b % kinds] for b in range(B)]
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = projection(g, kinds * tokens, H, J, D)[0].reshape(kinds, tokens, H, D)
    all_q = q[torch.arange(B, device="cuda") % kinds].reshape(B * tokens, H, D)
    cu = device([tokens * b for b in range(B + 1)]) if with_cu else None
    out = fptq.fptq_cached_attention(all_q, cache_of(codes, scales), device(table), device(lengths), cu, scratch=scratch).reshape(B, tokens, H, D)
    for i in range(kinds):
        check(out[i], *expected(host(q[i]), table[i], lengths[i], codes, scales), D)
    assert torch.equal(out, out[torch.arange(B, device="cuda") % kinds])


@pytest.mark.parametrize("H,J,D,tokens,length", [(3, 1, 64, 1, 40001), (4, 2, 128, 1, 40001), (40, 1, 64, 1, 17000), (20, 1, 128, 2, 20011)])
@pytest.mark.parametrize("cut", [False, True])
def test_more_than_64_pages_of_a_wave(H, J, D, tokens, length, cut):
    """Uncut, a wave has 67 to 79 pages, whose numbers it looks up 64 at a time."""
    few(1, 1, [length], -(-length // PAGE), tokens, H, J, D, tokens > 1, 1, None if cut else torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("H,J,D", [(3, 1, 64), (2, 1, 128), (20, 1, 64), (20, 1, 128)])
@pytest.mark.parametrize("width,long", [(8, 400), (200, 400), (200, 4500)])
@pytest.mark.parametrize("with_cu", [False, True])
def test_more_units_than_workgroups(H, J, D, width, long, with_cu):
    """1100 units, and where the table has room for long sequences and some are, their parts: workgroups go on to second ones.  (Seven kinds: the units of a workgroup
    differ.)"""
    few(7, 1100, [long, 64, 300, 1, 65, 128, 17], width, 1, H, J, D, with_cu, 2)


@pytest.mark.parametrize("H,J,D", [(1, 1, 64), (2, 1, 128), (20, 1, 64), (20, 1, 128)])
def test_more_cut_units_than_the_join_has_workgroups(H, J, D):
    """530 units of three parts each."""
    few(7, 530, [4200, 4989, 4611, 4161, 5100, 4352, 4400], 80, 1, H, J, D, False, 3)


def test_more_parts_than_a_wave_has_lanes():
    """76 parts of one unit, joined by a wave a row."""
    few(40, 40, [38431] + [1 + 37 * b % 600 for b in range(39)], 640, 1, 16, 1, 64, False, 4)


@pytest.mark.parametrize("D", [64, 128])
def test_more_parts_than_a_workgroup_has_threads(D):
    """625 parts of one unit, joined by eight waves a row."""
    few(1, 1, [20000 * PAGE - 17], 20000, 1, 2, 1, D, False, 5)


@pytest.mark.parametrize("H,J,D,new,lengths", [(6, 2, 128, [300, 0, 211], [1000, 5, 340]), (3, 1, 64, [300, 0, 211], [1000, 5, 340]), (4, 1, 64, [200], [9000]),
                                               (4, 1, 128, [130, 1, 1], [4777, 4200, 3])])
def test_hundreds_of_new_tokens_behind_a_prefix(H, J, D, new, lengths):
    run_cached(new, lengths, H, J, D, seed=6)


@pytest.mark.parametrize("H,J,D", [(20, 1, 64), (20, 1, 128), (9, 3, 128)])
def test_an_append_of_many_tokens_and_heads(H, J, D):
    """From 4096 groups of query heads on a wave takes all heads of a token, a group after the other."""
    run_append([2000, 100, 0, 5], [10, 0, 70, 63], H, J, D, D, False, seed=7)
    run_append([2000, 100, 0, 5], [10, 0, 70, 63], H, J, D, D // 2, True, seed=8)
