"""Performance cases of what a decoder block does between its QKV and its O projection: rotating queries and keys by their
positions and appending keys and values to a paged 8-bit cache, attention over that cache, and attention over whole prompts.

A case has a kind:
  append   `tokens` new tokens, packed one sequence after the other, of `sequences` sequences that hold up to `context` tokens
           already: q and k are rotated (`rope` of the head's values, pairs of neighbours or of halves), k and v go into the pages
  prompt   causal attention among the `tokens` of `sequences` packed prompts, on the rows that the QKV projection wrote
  cached   attention of each sequence's last tokens (one each where `tokens` equals `sequences`) over its cache of up to `context` tokens

The cache: a page holds 64 tokens of one sequence, for each of its heads as e4m3 codes with one power of two as scale, the smallest s
with max |x| <= 448 s (at least 2^-100).  A page-head's keys lie as [D / 64][64 tokens][64 values], its values as [4][D][16 tokens].  `lengths` counts a sequence's
tokens with the new ones; new tokens that begin in the middle of a page keep its scale or raise it, and then the older codes are
rounded again.  Codes are rounded once, from the keys as they were rotated and not from their bf16 form.  What a sequence's length is
follows from the case alone (`lengths` is a seed).
"""
import math
import random

import torch

own = False

PAGE = 64
HEADS = [(32, 8, 128), (64, 8, 128), (32, 32, 128), (20, 4, 128), (40, 40, 128), (32, 4, 64), (12, 4, 64), (28, 4, 128), (16, 1, 128), (9, 3, 64)]


def listed():
    return [
        # one token of one sequence, heads of a Llama-3-8B-shaped layer: what a call costs at its smallest
        _case("append_token_8b", "append", 1, 1, 1000, (32, 8, 128), 128, False, False, 1),
        # a token of each of 32 sequences at odd places of their pages, Llama-3-70B-shaped layer
        _case("append_tokens_70b_32", "append", 32, 32, 2048, (64, 8, 128), 128, False, False, 2),
        # a chunk of seven prompts behind what is cached of them: neighbouring pairs, half of the head rotated, narrow heads
        _case("append_ragged_1000", "append", 7, 1000, 777, (12, 4, 64), 32, True, True, 3),
        # a prompt of 4096 tokens into an empty cache, rotated keys wanted for the attention over it
        _case("append_prompt_8b_4096", "append", 1, 4096, 0, (32, 8, 128), 128, False, True, 4),
        # the tokens of five short prompts, odd lengths
        _case("prompt_ragged_333", "prompt", 5, 333, 0, (32, 8, 128), 0, False, False, 5),
        # nine prompts in a batch, a head of keys for each head of queries (Llama-2-7B-shaped layer)
        _case("prompt_7b_packed_6000", "prompt", 9, 6000, 0, (32, 32, 128), 0, False, False, 6),
        # one prompt of 4096 tokens, Llama-3-8B-shaped layer
        _case("prompt_8b_4096", "prompt", 1, 4096, 0, (32, 8, 128), 0, False, False, 7),
        # one prompt of 8192 tokens, Llama-3-70B-shaped layer: the largest
        _case("prompt_70b_8192", "prompt", 1, 8192, 0, (64, 8, 128), 0, False, False, 8),
        # the token loop of one short conversation
        _case("token_8b_333", "cached", 1, 1, 333, (32, 8, 128), 0, False, False, 9),
        # a batch of 32 sequences of different lengths
        _case("tokens_8b_32", "cached", 32, 32, 4096, (32, 8, 128), 0, False, False, 10),
        # four tokens to verify behind one very long context, narrow heads
        _case("verify_4_long_131072", "cached", 1, 4, 131072, (32, 4, 64), 0, False, False, 11),
        # a full batch of long sequences, Llama-3-70B-shaped layer
        _case("tokens_70b_64_long", "cached", 64, 64, 32768, (64, 8, 128), 0, False, False, 12),
    ]


def _case(name, kind, sequences, tokens, context, heads, rope, interleaved, keys, lengths):
    c = {"name": name, "kind": kind, "sequences": sequences, "tokens": tokens, "context": context, "heads": heads[0], "kv_heads": heads[1],
         "head_dim": heads[2], "lengths": lengths}
    if kind == "append":
        c.update(rope=rope, interleaved=interleaved, keys=keys)
    if name is None:
        del c["name"]
    return c


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind, heads, seed = rng.choice(["append", "prompt", "prompt", "cached", "cached"]), rng.choice(HEADS), rng.randrange(1 << 30)
    h, j, d = heads
    if kind == "append":
        sequences = _log_int(rng, 1, 128)
        tokens = sequences if rng.random() < 0.5 else _log_int(rng, 1, 8192 * 32 // h)
        rope = rng.choice([d, d, d, d // 2, d // 4])
        return _case(None, kind, sequences, tokens, rng.choice([0, _log_int(rng, 1, 2048)]), heads, rope, rng.random() < 0.4, rng.random() < 0.5, seed)
    if kind == "prompt":
        tokens = _log_int(rng, 1, 8192)
        return _case(None, kind, _log_int(rng, 1, max(1, min(64, tokens))), tokens, 0, heads, 0, False, False, seed)
    context = _log_int(rng, 1, 131072)
    most = max(1, 2 * 10**9 // (2 * context * j * d))                # cached bytes below those of the largest listed case
    sequences = min(_log_int(rng, 1, 256), most)
    tokens = sequences if rng.random() < 0.7 else sequences * rng.randrange(2, 9)
    return _case(None, kind, sequences, tokens, context, heads, 0, False, False, seed)


def _lengths(case):
    """(new tokens, tokens with the new ones) of every sequence."""
    rng, b, t, c = random.Random(case["lengths"]), case["sequences"], case["tokens"], case["context"]
    if case["kind"] == "cached" or t == b:
        new = [t // b] * b
    else:                                                            # cut at random: some may be empty
        cuts = sorted(rng.randrange(t + 1) for _ in range(b - 1))
        new = [y - x for x, y in zip([0] + cuts, cuts + [t])]
    if case["kind"] == "cached":
        return new, [c if b == 1 else rng.randint(max(1, c // 4), c) for _ in range(b)]      # a few may be shorter than their new tokens
    before = [0 if c == 0 else c if b == 1 else rng.randint(c // 4, c) for _ in range(b)]
    return new, [n + p for n, p in zip(new, before)]


# ---------------------------------------------------------------------------------------------------------- inputs

def _qkv(case, g):
    """A row of the QKV projection for every token: unit variance, some channels of the keys larger, queries that make some tokens matter more."""
    h, j, d = case["heads"], case["kv_heads"], case["head_dim"]
    x = torch.randn((case["tokens"], (h + 2 * j) * d), device="cuda", generator=g)
    x[:, :h * d] *= 1.5
    x[:, h * d:(h + j) * d] *= torch.exp(0.3 * torch.randn((j * d,), device="cuda", generator=g))
    return x.to(torch.bfloat16)


def _views(case, qkv):
    h, j, d = case["heads"], case["kv_heads"], case["head_dim"]
    q, k, v = qkv.split([h * d, j * d, j * d], 1)
    return q.unflatten(1, (h, d)), k.unflatten(1, (j, d)), v.unflatten(1, (j, d))


def _codes(g, pages, j, d):
    """Pages full of codes as older tokens leave them, and their scales."""
    x = torch.empty((pages, j, PAGE * d), dtype=torch.float8_e4m3fn, device="cuda")
    for i in range(0, pages, 1024):
        x[i:i + 1024] = torch.randn((min(1024, pages - i), j, PAGE * d), device="cuda", generator=g).mul_(80.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
    return x.view(torch.uint8), torch.exp2(torch.randint(-8, -5, (pages, j), device="cuda", generator=g).float())


def _rope_table(positions, rope):
    """fp32 [positions, 2, rope / 2]: cosines and sines of angles taken in 64 bits, base 500000."""
    freq = 500000.0 ** (-torch.arange(0, rope, 2, dtype=torch.float64, device="cuda") / rope)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, lengths = _lengths(case)
    s = {"case": case, "new": new, "lens": lengths}
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["starts"] = starts
    s["qkv"] = _qkv(case, g)
    s["q"], s["k"], s["v"] = _views(case, s["qkv"])
    s["cu"] = i32(starts)
    s["one_each"] = all(n == 1 for n in new)
    if case["kind"] == "prompt":
        if own:
            from paper_2506_04985_amd import binding as fptq
            fptq.fptq_init()
        return s
    j, d = case["kv_heads"], case["head_dim"]
    pages = [max(1, -(-n // PAGE)) for n in lengths]
    pool = sum(pages) + 3
    order = torch.randperm(pool, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros((len(pages), max(pages)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"], s["length"] = table, i32(lengths)
    s["ck"], s["sk"] = _codes(g, pool, j, d)
    s["cv"], s["sv"] = _codes(g, pool, j, d)
    if case["kind"] == "append":
        s["rope"] = _rope_table(max(lengths) + 1, case["rope"])
    if own:
        from paper_2506_04985_amd import binding as fptq
        fptq.fptq_init()
        s["cache"] = fptq.Cache(s["ck"], s["cv"], s["sk"], s["sv"])
    return s


# ----------------------------------------------------------------------------------------------------- plain forms

def _rotate(x, rope, interleaved):
    """x [T, heads, D] in fp32 by the rows [T, 2, R / 2] of the table, in fp32."""
    r = rope.shape[2] * 2
    c, s = rope[:, 0, None], rope[:, 1, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    p, q = a * c - b * s, b * c + a * s
    y = torch.stack([p, q], -1).flatten(-2) if interleaved else torch.cat([p, q], -1)
    return torch.cat([y, x[..., r:]], -1)


def _scale_for(largest):
    """The smallest power of two s with largest <= 448 s, 2^-100 at least: 448 is 1.75 * 2^8."""
    bits = ((largest.view(torch.int32) + 0x1fffff) >> 23) - 8
    return (bits.clamp(min=27) << 23).view(torch.float32)


def _plain_append(s):
    case = s["case"]
    d = case["head_dim"]
    dev = s["q"].device
    new, length = s["cu"][1:] - s["cu"][:-1], s["length"]
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=dev), new.long(), output_size=case["tokens"])
    pos = (length - new)[seq].long() + torch.arange(case["tokens"], device=dev) - s["cu"][:-1].long()[seq]
    page, off = s["table"][seq, pos // PAGE].long(), pos % PAGE
    rows = s["rope"][pos]
    q = _rotate(s["q"].float(), rows, case["interleaved"])
    k = _rotate(s["k"].float(), rows, case["interleaved"])
    touched, of = torch.unique(page, return_inverse=True)
    first = torch.full((len(touched),), PAGE, dtype=torch.long, device=dev).scatter_reduce(0, of, off, "amin")
    for x, codes, scales, keys in ((k, s["ck"], s["sk"], True), (s["v"].float(), s["cv"], s["sv"], False)):
        j = x.shape[1]
        largest = torch.zeros((len(touched), j), device=dev).scatter_reduce(0, of[:, None].expand(-1, j), x.abs().amax(2), "amax")
        old = torch.where((first > 0)[:, None], scales[touched], torch.zeros((), device=dev))
        scale = torch.maximum(_scale_for(largest), old)
        c = codes[touched].view(torch.float8_e4m3fn)
        c = c.view(len(touched), j, d // 64, PAGE, 64).permute(0, 1, 3, 2, 4) if keys else c.view(len(touched), j, 4, d, 16).permute(0, 1, 2, 4, 3)
        c = c.reshape(len(touched), j, PAGE, d).float()
        older = torch.arange(PAGE, device=dev) < first[:, None]
        ratio = torch.where(older[:, None, :], (old / scale)[:, :, None], torch.ones((), device=dev))
        c = c * ratio[..., None]
        c[of, :, off] = x / scale[of][..., None]
        c = c.to(torch.float8_e4m3fn).view(torch.uint8)
        c = c.view(len(touched), j, PAGE, d // 64, 64).permute(0, 1, 3, 2, 4) if keys else c.view(len(touched), j, 4, 16, d).permute(0, 1, 2, 4, 3)
        codes[touched] = c.reshape(len(touched), j, PAGE * d)
        scales[touched] = scale
    return q.to(torch.bfloat16), k.to(torch.bfloat16) if case["keys"] else None


def _attend(q, k, v, out, scale):
    """q [n, H, D] over k, v [m, J, D] in fp32, the last query at the last key; queries before the first key get zeros."""
    n, h, d = q.shape
    m, j, _ = k.shape
    g = h // j
    kt, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
    step = max(1, (1 << 29) // (h * m))
    for i in range(0, n, step):
        rows = min(step, n - i)
        x = q[i:i + rows].reshape(rows, j, g, d).permute(1, 2, 0, 3).reshape(j, g * rows, d).contiguous()
        p = (x @ kt).mul_(scale).view(j, g, rows, m)
        masked = torch.arange(m, device=q.device) > torch.arange(i, i + rows, device=q.device)[:, None] + (m - n)
        p.masked_fill_(masked, float("-inf"))
        largest = p.amax(3, keepdim=True)
        p.sub_(torch.where(largest == float("-inf"), torch.zeros_like(largest), largest)).exp_()
        total = p.sum(3, keepdim=True)
        o = (p.view(j, g * rows, m) @ v).view(j, g, rows, d) / torch.where(total == 0, torch.ones_like(total), total)
        out[i:i + rows] = o.permute(2, 0, 1, 3).reshape(rows, h, d).to(out.dtype)


def _plain_prompt(s):
    out = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
    for a, b in zip(s["starts"], s["starts"][1:]):
        if b > a:
            _attend(s["q"][a:b].float(), s["k"][a:b].float(), s["v"][a:b].float(), out[a:b], s["case"]["head_dim"] ** -0.5)
    return out


def _values(s, b, n, dtype):
    """The first n keys and values [n, J, D] of sequence b."""
    j, d = s["case"]["kv_heads"], s["case"]["head_dim"]
    pages = s["table"][b, :-(-n // PAGE)].long()
    k = s["ck"][pages].view(torch.float8_e4m3fn).to(dtype) * s["sk"][pages].to(dtype)[..., None]
    v = s["cv"][pages].view(torch.float8_e4m3fn).to(dtype) * s["sv"][pages].to(dtype)[..., None]
    k = k.view(-1, j, d // 64, PAGE, 64).permute(0, 3, 1, 2, 4).reshape(-1, j, d)
    v = v.view(-1, j, 4, d, 16).permute(0, 2, 4, 1, 3).reshape(-1, j, d)
    return k[:n], v[:n]


def _plain_cached(s):
    out = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
    for b, n in enumerate(s["lens"]):
        k, v = _values(s, b, n, torch.float32)
        a, e = s["starts"][b], s["starts"][b + 1]
        _attend(s["q"][a:e].float(), k, v, out[a:e], s["case"]["head_dim"] ** -0.5)
    return out


# ------------------------------------------------------------------------------------------------------------- run

def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2506_04985_amd import binding as fptq
        cu = None if s["one_each"] else s["cu"]
        if case["kind"] == "prompt":
            return {"out": fptq.fptq_prompt_attention(s["q"], s["k"], s["v"], s["cu"])}
        if case["kind"] == "cached":
            return {"out": fptq.fptq_cached_attention(s["q"], s["cache"], s["table"], s["length"], cu)}
        q, k = fptq.fptq_cache_append(s["q"], s["k"], s["v"], s["rope"], s["cache"], s["table"], s["length"], cu, interleaved=case["interleaved"],
                                      want_k=case["keys"])
    else:
        if case["kind"] == "prompt":
            return {"out": _plain_prompt(s)}
        if case["kind"] == "cached":
            return {"out": _plain_cached(s)}
        q, k = _plain_append(s)
    fp8 = torch.float8_e4m3fn
    out = {"q": q, "key_codes": s["ck"].view(fp8), "value_codes": s["cv"].view(fp8), "key_scales": s["sk"], "value_scales": s["sv"]}
    if case["keys"]:
        out["k"] = k
    return out


# ---------------------------------------------------------------------------------------------------- work, checks

def work(case):
    h, j, d, t = case["heads"], case["kv_heads"], case["head_dim"], case["tokens"]
    new, lengths = _lengths(case)
    if case["kind"] == "append":          # rows in, rotated queries (and keys) and codes out, the table's row of each token
        nbytes = 2 * t * (h + 2 * j) * d + 2 * t * h * d + (2 * t * j * d if case["keys"] else 0) + 2 * t * j * d + 4 * t * case["rope"]
        return {"bytes": nbytes, "flops": 3 * t * (h + j) * case["rope"] + 2 * t * j * d}
    if case["kind"] == "prompt":
        return {"bytes": 2 * t * (h + 2 * j) * d + 2 * t * h * d, "flops": sum(2 * n * (n + 1) for n in new) * h * d}
    pairs = sum(n * m - n * (n - 1) // 2 if m >= n else m * (m + 1) // 2 for n, m in zip(new, lengths))
    return {"bytes": sum(lengths) * 2 * j * d + 4 * t * h * d + sum(-(-m // PAGE) for m in lengths) * (8 * j + 4), "flops": 4 * pairs * h * d}


def _softmax_rows(q, k, v, scale):
    """One head in 64 bits: q [n, D], k, v [m, D], causal from the end."""
    n, m = q.shape[0], k.shape[0]
    out = torch.zeros_like(q)
    for i in range(max(0, n - m), n, 1024):
        rows = min(1024, n - i)
        keys = m - n + i + rows
        x = scale * (q[i:i + rows] @ k[:keys].t())
        x += torch.triu(torch.full((rows, keys), -math.inf, dtype=torch.float64, device=q.device), keys - rows + 1)
        out[i:i + rows] = torch.softmax(x, 1) @ v[:keys]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    h, j, d = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] != "append":
        out = torch.zeros((case["tokens"], h, d), dtype=torch.float64, device="cuda")
        for b, (a, e) in enumerate(zip(s["starts"], s["starts"][1:])):
            if e == a:
                continue
            k, v = (s["k"][a:e].double(), s["v"][a:e].double()) if case["kind"] == "prompt" else _values(s, b, s["lens"][b], torch.float64)
            for head in range(h):
                o = head // (h // j)
                out[a:e, head] = _softmax_rows(s["q"][a:e, head].double(), k[:, o].contiguous(), v[:, o].contiguous(), d ** -0.5)
        return {"out": out}
    # append, a sequence and a page at a time; codes as what they round, x / s
    q, k = s["q"].double(), s["k"].double()
    r = case["rope"]
    first = torch.arange(0, r, 2, device="cuda") if case["interleaved"] else torch.arange(r // 2, device="cuda")
    second = first + 1 if case["interleaved"] else first + r // 2
    codes = {n: s[n].view(torch.float8_e4m3fn).double() for n in ("ck", "cv")}
    keys, values = codes["ck"].view(-1, j, d // 64, PAGE, 64), codes["cv"].view(-1, j, 4, d, 16)
    scales = {n: s[n].double() for n in ("sk", "sv")}
    for b, (a, e) in enumerate(zip(s["starts"], s["starts"][1:])):
        if e == a:
            continue
        begin = s["lens"][b] - (e - a)
        cos, sin = s["rope"][begin:s["lens"][b]].double().unbind(1)
        for x in (q[a:e], k[a:e]):
            u, w = x[..., first].clone(), x[..., second].clone()
            x[..., first] = u * cos[:, None] - w * sin[:, None]
            x[..., second] = w * cos[:, None] + u * sin[:, None]
        pages = s["table"][b].tolist()
        p = begin
        while p < s["lens"][b]:
            page, o = pages[p // PAGE], p % PAGE
            n = min(PAGE - o, s["lens"][b] - p)
            for name, x in (("k", k), ("v", s["v"].double())):
                x = x[a + p - begin:a + p - begin + n]
                largest = x.abs().amax((0, 2))
                scale = torch.exp2(torch.ceil(torch.log2(largest / 448)).clamp(min=-100))
                if o:
                    old = scales["s" + name][page]
                    scale = torch.maximum(scale, old)
                    if name == "k":
                        keys[page, :, :, :o] *= (old / scale)[:, None, None, None]
                    else:
                        t = torch.arange(o, device="cuda")
                        values[page][:, t // 16, :, t % 16] *= (old / scale)[None, :, None]
                scales["s" + name][page] = scale
                x = x / scale[None, :, None]
                t = torch.arange(o, o + n, device="cuda")
                if name == "k":
                    keys[page][:, :, t] = x.view(n, j, d // 64, 64).permute(1, 2, 0, 3)
                else:
                    values[page][:, t // 16, :, t % 16] = x
            p += n
    out = {"q": q, "key_codes": codes["ck"], "value_codes": codes["cv"], "key_scales": scales["sk"], "value_scales": scales["sv"]}
    if case["keys"]:
        out["k"] = k
    return out
