"""What the attention entry points refuse, before anything is launched: no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2506_04985_amd import binding as fptq

P = 4096


def heads(data=P, token=1024, head=128):
    return fptq._Heads(data, token, head)


def cache(**change):
    return fptq._Cache(**{"key_codes": P, "value_codes": P, "key_scales": P, "value_scales": P, "pages": 10, **change})


def append(**change):
    a = {"q": heads(), "k": heads(), "v": heads(), "tokens": 4, "sequences": 4, "heads": 8, "kv_heads": 2, "head_dim": 128, "rope": P, "positions": 100,
         "rope_dims": 128, "interleaved": 0, "cache": cache(), "table": P, "width": 4, "lengths": P, "cu": None, "q_out": P, "k_out": None, "stream": None, **change}
    return fptq.lib().fptq_cache_append(*a.values())


def cached(**change):
    a = {"q": heads(), "tokens": 4, "sequences": 4, "heads": 8, "kv_heads": 2, "head_dim": 128, "scale": 0.1, "cache": cache(), "table": P, "width": 4,
         "lengths": P, "cu": None, "out": P, "scratch": None, "bytes": 0, "stream": None, **change}
    return fptq.lib().fptq_cached_attention(*a.values())


def prompt(**change):
    a = {"q": heads(), "k": heads(), "v": heads(), "tokens": 4, "sequences": 1, "heads": 8, "kv_heads": 2, "head_dim": 128, "scale": 0.1, "cu": P, "out": P,
         "stream": None, **change}
    return fptq.lib().fptq_prompt_attention(*a.values())


SHAPES = [({"tokens": -1}, -2), ({"tokens": (1 << 24) + 1}, -2), ({"sequences": 0}, -2), ({"heads": 0}, -2), ({"heads": 7}, -2), ({"kv_heads": 0}, -2),
          ({"heads": 8192, "kv_heads": 8192}, -2), ({"head_dim": 96}, -2), ({"head_dim": 256}, -2), ({"q": None}, -1), ({"q": heads(0)}, -1), ({"q": heads(P + 8)}, -7),
          ({"q": heads(P, 1020)}, -7), ({"q": heads(P, -8)}, -2), ({"q": heads(P, 1 << 24)}, -2), ({"q": heads(P, 1024, 4)}, -7)]
PAGED = [({"cache": None}, -1), ({"cache": cache(key_codes=0)}, -1), ({"cache": cache(value_scales=0)}, -1), ({"cache": cache(pages=0)}, -2),
         ({"cache": cache(pages=1 << 31)}, -2), ({"cache": cache(key_codes=P + 8)}, -7), ({"cache": cache(key_scales=P + 2)}, -7), ({"table": None}, -1),
         ({"lengths": None}, -1), ({"width": 0}, -2), ({"sequences": 3}, -2), ({"table": P + 1}, -7), ({"lengths": P + 2}, -7), ({"cu": P + 2, "sequences": 3}, -7)]
SCALES = [({"scale": s}, -6) for s in (0.0, -1.0, float("inf"), float("nan"))]


@pytest.mark.parametrize("change,code", SHAPES + PAGED + [
    ({"k": heads(P, 1020)}, -7), ({"v": None}, -1), ({"rope": None}, -1), ({"rope": P + 4}, -7), ({"rope_dims": 24}, -2), ({"rope_dims": 144}, -2), ({"rope_dims": -16}, -2),
    ({"positions": 0}, -2), ({"q_out": None}, -1), ({"q_out": P + 2}, -7), ({"k_out": P + 2}, -7)])
def test_cache_append(change, code):
    assert append(**change) == code
    assert b"fptq_cache_append" in fptq.lib().fptq_last_error()


@pytest.mark.parametrize("change,code", SHAPES + PAGED + SCALES + [({"out": None}, -1), ({"out": P + 2}, -7), ({"bytes": -1}, -3), ({"scratch": P + 128}, -7)])
def test_cached_attention(change, code):
    assert cached(**change) == code
    assert b"fptq_cached_attention" in fptq.lib().fptq_last_error()


@pytest.mark.parametrize("change,code", SHAPES + SCALES + [({"k": None}, -1), ({"v": heads(P + 2)}, -7), ({"cu": None}, -1), ({"cu": P + 2}, -7), ({"out": None}, -1),
                                                          ({"out": P + 8}, -7)])
def test_prompt_attention(change, code):
    assert prompt(**change) == code
    assert b"fptq_prompt_attention" in fptq.lib().fptq_last_error()


# Sizes that are within their own limits each and together ask for more workgroups than a launch may have (include/fptq.h states how many), refused
# before the device is asked for anything.  No call here is just within them: its pointers are made up, and it would be launched where there is a GPU.
BIG = 1 << 24


@pytest.mark.parametrize("change", [{"tokens": 1 << 20, "sequences": 1 << 20, "heads": 8, "kv_heads": 8}, {"tokens": BIG, "sequences": BIG},
                                    {"tokens": BIG, "sequences": 1, "heads": 32, "kv_heads": 32, "cu": P}, {"tokens": 4096, "sequences": 4096, "heads": 4096, "kv_heads": 4096}])
def test_cache_append_of_too_much(change):
    assert append(**change) == -2
    assert b"fptq_cache_append: too many" in fptq.lib().fptq_last_error()


@pytest.mark.parametrize("more", [{}, {"scratch": P, "bytes": 1 << 40}])
@pytest.mark.parametrize("change", [{"tokens": 1 << 21, "sequences": 1 << 21, "heads": 8, "kv_heads": 8, "width": 100}, {"tokens": BIG, "sequences": 1, "heads": 64, "kv_heads": 8, "cu": P},
                                    {"tokens": BIG, "sequences": 1, "heads": 4096, "kv_heads": 1, "cu": P}])
def test_cached_attention_of_too_much(change, more):
    assert cached(**change, **more) == -2
    assert b"fptq_cached_attention: too many" in fptq.lib().fptq_last_error()


def test_the_parts_of_cached_attention_count_too():
    """Without scratch nothing is cut, and 2^23 rows are served; with it there can be 3072 parts beside them."""
    assert cached(tokens=1 << 20, sequences=1 << 20, heads=8, kv_heads=8, width=100, scratch=P, bytes=1 << 40) == -2
    assert b"fptq_cached_attention: too many" in fptq.lib().fptq_last_error()


@pytest.mark.parametrize("change", [{"tokens": BIG, "heads": 64}, {"tokens": BIG, "sequences": BIG}, {"tokens": 1 << 20, "sequences": 1 << 20, "heads": 16},
                                    {"tokens": 4096, "sequences": 4096, "heads": 4096}])
def test_prompt_attention_of_too_much(change):
    assert prompt(**change) == -2
    assert b"fptq_prompt_attention: too many" in fptq.lib().fptq_last_error()


def test_no_tokens_are_nothing_to_do():
    assert append(tokens=0, cu=P) == 0 and cached(tokens=0, cu=P) == 0 and prompt(tokens=0) == 0


def test_scratch_bytes():
    f = fptq.fptq_cached_attention_scratch_bytes
    assert f(1, 1, 8, 2, 128, 16) == 0                      # 16 pages are never cut
    assert f(1, 1, 8, 2, 128, 17) == 3072 * 16 * 130 * 4
    assert f(8, 1, 8, 2, 64, 4096) == 3072 * 32 * 66 * 4    # 32 rows a tile
    for bad in ((1, 1, 8, 3, 128, 16), (1, 1, 8, 2, 100, 16), (1, 1, 8, 2, 128, 0), (-1, 1, 8, 2, 128, 16)):
        with pytest.raises(fptq.FptqError) as e:
            f(*bad)
        assert e.value.code == -2


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros((4, 8, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        fptq.fptq_prompt_attention(x, x, x, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        fptq.Cache(torch.zeros((1, 2, 64 * 64), dtype=torch.uint8), None, None, None)
