"""fptq_prompt_attention against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from attention_util import check, device, host, projection, starts
from oracle import attention as oracle
from paper_2506_04985_amd import binding as fptq

pytestmark = pytest.mark.gpu


def expected(q, k, v, new, scale):
    parts = []
    for a, b in zip(starts(new), starts(new)[1:]):
        parts.append(oracle.attention(host(q[a:b]), host(k[a:b]), host(v[a:b]), scale))
    return [np.concatenate([p[i] for p in parts]) for i in range(3)]


@pytest.mark.parametrize("H,J,D", [(4, 2, 128), (3, 3, 64), (8, 1, 64), (7, 1, 128), (8, 8, 128)])
@pytest.mark.parametrize("new", [[1], [2, 31, 32], [33, 0, 63, 64, 65], [127, 128, 129], [0, 0, 5], [260]])
def test_packed_prompts(new, H, J, D):
    g = torch.Generator(device="cuda").manual_seed(sum(new) + H)
    q, k, v = projection(g, sum(new), H, J, D, 1.5)
    out = fptq.fptq_prompt_attention(q, k, v, device(starts(new)))
    check(out, *expected(q, k, v, new, D ** -0.5), D)


@pytest.mark.parametrize("B", [8, 9, 32, 33, 64, 65, 130])
def test_many_prompts(B):
    """Up to 32 sequences are sorted by length, more are taken in their order, 64 at a time."""
    new = [int(n) for n in np.random.default_rng(B).integers(0, 150, B)]
    new[B // 2] = 300
    g = torch.Generator(device="cuda").manual_seed(B)
    q, k, v = projection(g, sum(new), 3, 1, 64)
    out = fptq.fptq_prompt_attention(q, k, v, device(starts(new)))
    check(out, *expected(q, k, v, new, 0.125), 64)


@pytest.mark.parametrize("D", [64, 128])
def test_a_long_prompt_with_large_scores(D):
    """Scores far apart, so that the running maximum grows often and by much."""
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = projection(g, 1100, 2, 1, D, 1.0)
    k = k * (torch.arange(1100, device="cuda")[:, None, None] / 100).to(torch.bfloat16)
    out = fptq.fptq_prompt_attention(q, k, v, device([0, 1100]), scale=0.3)
    check(out, *expected(q, k, v, [1100], float(np.float32(0.3))), D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_value_that_is_not_finite_reaches_only_those_who_see_it(bad, D):
    g = torch.Generator(device="cuda").manual_seed(6)
    q, k, v = projection(g, 300, 2, 2, D)
    v[100, 1, 7] = bad
    v[233, 0, D - 1] = bad
    out = host(fptq.fptq_prompt_attention(q, k, v, device([0, 170, 300])))
    want = expected(q, k, v, [170, 130], D ** -0.5)[0]
    np.testing.assert_array_equal(np.isnan(out), np.isnan(want))
    np.testing.assert_array_equal(np.isposinf(out), np.isposinf(want))
    np.testing.assert_array_equal(np.isneginf(out), np.isneginf(want))
    assert np.isfinite(out[:100]).all() and not np.isfinite(out[100:170, 1, 7]).any() and np.isfinite(out[170:233]).all()


def test_keys_that_are_not_finite():
    """NaN for the tokens that see a NaN key; a key whose score is the lowest there is has no weight; a token that sees only such keys gets zeros."""
    g = torch.Generator(device="cuda").manual_seed(7)
    q, k, v = projection(g, 200, 1, 1, 64)
    q, k = q.abs() + 0.1, k.clone()
    k[:40] = float("-inf")
    k[150, 0, 3] = float("nan")
    out = host(fptq.fptq_prompt_attention(q, k, v, device([0, 200])))
    assert (out[:40] == 0).all() and np.isnan(out[150:]).all()
    out2, mass, terms = oracle.attention(host(q[40:150]), host(k[40:150]), host(v[40:150]), 0.125)
    check(torch.from_numpy(out[40:150]), out2, mass, terms, 64)


def test_strided_rows_an_output_of_the_callers_and_another_stream():
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v = projection(g, 150, 4, 2, 128)
    kt = k.transpose(0, 1).contiguous().transpose(0, 1)                 # heads outermost
    out = torch.full((160, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    cu = device([0, 90, 150])
    want = fptq.fptq_prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), cu)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        assert fptq.fptq_prompt_attention(q, kt, v, cu, out=out) is out
    stream.synchronize()
    assert torch.equal(out[:150], want) and (out[150:] == 7).all()


def test_rows_of_no_sequence_and_starts_out_of_range():
    g = torch.Generator(device="cuda").manual_seed(9)
    q, k, v = projection(g, 100, 2, 1, 64)
    out = torch.full((100, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    fptq.fptq_prompt_attention(q, k, v, device([10, 50, 80]), out=out)
    check(out[10:80], *expected(q[10:80], k[10:80], v[10:80], [40, 30], 0.125), 64)
    assert (out[:10] == 7).all() and (out[80:] == 7).all()
    out = fptq.fptq_prompt_attention(q, k, v, device([-5, 60, 1 << 30]))             # 0, 60, 100
    check(out, *expected(q, k, v, [60, 40], 0.125), 64)


def test_no_tokens():
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert fptq.fptq_prompt_attention(q, q, q, device([0, 0])).shape == (0, 4, 64)


def test_offsets_past_32_bits():
    """Rows that lie 32 MB apart: more than 4 GB from the first to the last."""
    stride, T, D = (1 << 24) - 8, 150, 64
    room = torch.zeros(stride * T, dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((T, 3, D), (stride, D, 1))
    g = torch.Generator(device="cuda").manual_seed(10)
    x.copy_(torch.randn((T, 3, D), device="cuda", generator=g).to(torch.bfloat16))
    out = fptq.fptq_prompt_attention(x[:, :1], x[:, 1:2], x[:, 2:], device([0, T]))
    check(out, *expected(x[:, :1], x[:, 1:2], x[:, 2:], [T], 0.125), D)


def test_replays_of_a_captured_call_match_eager_ones():
    g = torch.Generator(device="cuda").manual_seed(11)
    q, k, v = (t.contiguous() for t in projection(g, 200, 4, 2, 128))
    cu, out = device([0, 70, 200]), torch.empty((200, 4, 128), dtype=torch.bfloat16, device="cuda")
    fptq.fptq_init()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fptq.fptq_prompt_attention(q, k, v, cu, out=out)
    for middle in (70, 1, 200, 128):
        q.copy_(torch.randn(q.shape, device="cuda", generator=g).to(torch.bfloat16))
        cu[1] = middle
        want = fptq.fptq_prompt_attention(q, k, v, cu)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("order", ["rising", "falling"])
def test_the_largest_scores_served(order, D):
    """Scores of up to 4.9 * 10^8, 2^22 apart: all weight is on the largest one seen.  Its weight is rounded to bf16, its sum is not, and the output is rounded."""
    n = 117
    g = torch.Generator(device="cuda").manual_seed(14)
    q, k, v = (torch.zeros((n, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    q[:, 0, 5] = 2048
    k[:, 0, 5] = (torch.arange(1, n + 1, device="cuda") if order == "rising" else torch.arange(n, 0, -1, device="cuda")) * 2048.0
    v.copy_(torch.randn(v.shape, device="cuda", generator=g))
    out = host(fptq.fptq_prompt_attention(q, k, v, device([0, n]), scale=1.0))
    want = host(v) if order == "rising" else np.broadcast_to(host(v)[:1], (n, 1, D))
    np.testing.assert_allclose(out, want, rtol=1.01 * 2 * 2.0 ** -8)
