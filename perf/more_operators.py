"""Performance cases of a layer's linears with 8-bit activations and 4-bit weights in groups: the residual's addition with the norm and an 8-bit
output, the gated activation with an 8-bit output, and the products.

A case has a kind:
  norm    `tokens` rows of `width` values: z = x + r (where there is a `residual` r), which is also the new residual; u = z * gain (where there
          is a `gain`); codes of u, and the scale of a row with 1 / sqrt(mean z^2 + eps) in it (where `rms`)
  gated   codes of silu(gate) * up; gate and up are the halves of the rows of one projection, `width` values each
  linear  y[t, n] = scale[t] * sum over groups of w_scale[group, n] * sum over the group's k of code[t, k] * w[n, k], with `group` values of
          k to a group; `logits`: y in fp32 and not in bf16

Codes are 8-bit integers, code = rne(u * (127 / max |u|)) in fp32, and a row's values are code * scale.  They lie in tiles of 128 values of k, tile after
tile, 128 bytes a row, the last tile filled up with zeros; of every eight values the even ones come first.  silu is rounded once, from 64 bits, so that codes
are the same wherever they are computed.
"""
import math
import random

import torch

own = False

TILE = 128
EPS = 1e-5


def listed():
    return [
        # the norm of one token, Llama-3-8B-shaped layer: what a call costs at its smallest
        _norm("norm_token_8b", 1, 4096, True, True, True),
        # the quantizer alone on rows of odd width, as before a projection that has no norm in front
        _norm("quantize_ragged_777", 777, 3601, False, False, False),
        # the norm of a long prompt, Llama-3-70B-shaped layer
        _norm("norm_70b_8192", 8192, 8192, True, True, True),
        # the gated activation of 16 tokens, Llama-3-8B-shaped layer
        _gated("gated_tokens_8b_16", 16, 14336),
        # of five short prompts, odd width
        _gated("gated_ragged_333", 333, 7391),
        # of a long prompt, Llama-3-8B-shaped layer
        _gated("gated_8b_4096", 4096, 14336),
        # one token against the QKV projection: the matrix-vector product
        _linear("token_qkv_8b", 1, 6144, 4096, 128, False),
        # a batch of 32 tokens against gate+up
        _linear("tokens_gate_up_8b_32", 32, 28672, 4096, 128, False),
        # eight tokens against the head of a large vocabulary, fine groups, fp32 logits
        _linear("head_8", 8, 128256, 4096, 64, True),
        # short prompts in a batch against an odd number of channels, a width that ends inside a group
        _linear("ragged_333", 333, 32003, 2504, 64, False),
        # a prompt against the down projection
        _linear("prompt_down_8b_1000", 1000, 4096, 14336, 128, False),
        # a long prompt against gate+up: the largest
        _linear("prompt_gate_up_8b_4096", 4096, 28672, 4096, 128, False),
    ]


def _case(name, **values):
    return values if name is None else {"name": name, **values}


def _norm(name, tokens, width, residual, gain, rms):
    return _case(name, kind="norm", tokens=tokens, width=width, residual=residual, gain=gain, rms=rms)


def _gated(name, tokens, width):
    return _case(name, kind="gated", tokens=tokens, width=width)


def _linear(name, tokens, channels, width, group, logits):
    return _case(name, kind="linear", tokens=tokens, channels=channels, width=width, group=group, logits=logits)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of the sizes are multiples of 64, the others whatever comes."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.5 else max(64, n // 64 * 64)


def draw(rng):
    kind, tokens = rng.choice(["norm", "gated", "linear", "linear"]), _log_int(rng, 1, 8192)
    if kind == "norm":
        width = _size(rng, 64, 16384)
        return _norm(None, min(tokens, 8192 * 8192 // width), width, rng.random() < 0.6, rng.random() < 0.6, rng.random() < 0.7)
    if kind == "gated":
        width = _size(rng, 64, 28672)
        return _gated(None, min(tokens, 4096 * 14336 // width), width)
    width, group, logits = _size(rng, 64, 16384), rng.choice([32, 64, 128, 128, 128, 256]), rng.random() < 0.25
    channels = min(_size(rng, 64, 131072), 128256 * 4096 // width)
    most = 4096 * 28672 * 4096 // (width * channels)                     # products of the largest listed case
    return _linear(None, max(1, min(tokens, most)), channels, width, group, logits)


# ---------------------------------------------------------------------------------------------------------- inputs

def _rows(g, tokens, width):
    """What a residual stream holds: unit variance, about one channel in two hundred of them twenty times as large."""
    x = torch.randn((tokens, width), device="cuda", generator=g)
    x *= 1.0 + 19.0 * (torch.rand((width,), device="cuda", generator=g) < 0.005)
    return x.to(torch.bfloat16)


def _lay_out(codes):
    """int8 [tokens, width] as the products read it."""
    tokens, width = codes.shape
    tiles = -(-width // TILE)
    if width % TILE:
        codes = torch.cat([codes, codes.new_zeros((tokens, tiles * TILE - width))], 1)
    return codes.view(tokens, tiles, TILE // 8, 4, 2).permute(1, 0, 2, 4, 3).reshape(-1)


def _quantize_weights(g, channels, width, group):
    """Normal weights rounded to 4 bits on a grid for each group, a slab of channels at a time."""
    groups = -(-width // group)
    w = torch.empty((channels, width), dtype=torch.int8, device="cuda")
    scales = torch.empty((groups, channels), device="cuda")
    step = max(1, (1 << 28) // (groups * group))
    for i in range(0, channels, step):
        n = min(step, channels - i)
        x = torch.randn((n, groups * group), device="cuda", generator=g).mul_(0.02).view(n, groups, group)
        s = x.abs().amax(2).div_(7.5)
        scales[:, i:i + n] = s.t()
        w[i:i + n] = (x / s[:, :, None]).round_().clamp_(-8, 7).to(torch.int8).view(n, -1)[:, :width]
    return w, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, k, s = case["tokens"], case["width"], {"case": case}
    if case["kind"] == "norm":
        s["x"] = _rows(g, t, k)
        s["residual"] = _rows(g, t, k) if case["residual"] else None
        s["gain"] = (1.0 + 0.3 * torch.randn((k,), device="cuda", generator=g)).to(torch.bfloat16) if case["gain"] else None
    elif case["kind"] == "gated":
        s["gate_up"] = torch.randn((t, 2 * k), device="cuda", generator=g).mul_(1.5).to(torch.bfloat16)
        s["gate"], s["up"] = s["gate_up"].split(k, 1)
    else:
        s["codes"], s["scale"] = _codes(_rows(g, t, k).float(), None)
        s["laid_out"] = _lay_out(s["codes"])
        s["w"], s["w_scales"] = _quantize_weights(g, case["channels"], k, case["group"])
    if own:
        from paper_2506_04985_amd import binding as fptq
        fptq.fptq_init()
        if case["kind"] == "linear":
            s["packed"] = fptq.fptq_pack_weights(s["w"])
    return s


# ----------------------------------------------------------------------------------------------------- plain forms

def _codes(u, inv):
    """Codes [tokens, width] of fp32 rows, and their scales."""
    largest = u.abs().amax(1)
    a = largest.clamp(min=2.0 ** -100)
    codes = (u * torch.div(torch.full_like(a, 127.0), a)[:, None]).round_().to(torch.int8)
    scale = (a if inv is None else a * inv) * (1.0 / 127.0)
    return codes, torch.where(largest == 0, torch.zeros_like(scale), scale)


def _plain_norm(s):
    z, case = s["x"].float(), s["case"]
    if case["residual"]:
        z = z + s["residual"].float()
    inv = None
    if case["rms"]:
        inv = (1.0 / torch.sqrt(z.double().square().sum(1) / case["width"] + EPS)).float()
    codes, scale = _codes(z * s["gain"].float() if case["gain"] else z, inv)
    out = {"codes": _lay_out(codes), "scale": scale}
    if case["residual"]:
        out["residual"] = z.to(torch.bfloat16)
    return out


def _plain_gated(s):
    g = s["gate"].double()
    codes, scale = _codes((g / (1.0 + torch.exp(-g))).float() * s["up"].float(), None)
    return {"codes": _lay_out(codes), "scale": scale}


def _plain_linear(s):
    case = s["case"]
    w = s["w"].float() * s["w_scales"].t().repeat_interleave(case["group"], 1)[:, :case["width"]]
    y = (s["codes"].float() @ w.t()) * s["scale"][:, None]
    return {"y": y if case["logits"] else y.to(torch.bfloat16)}


# ------------------------------------------------------------------------------------------------------------- run

def run(state):
    s, case = state, state["case"]
    if not own:
        return {"norm": _plain_norm, "gated": _plain_gated, "linear": _plain_linear}[case["kind"]](s)
    from paper_2506_04985_amd import binding as fptq
    if case["kind"] == "linear":
        y = fptq.fptq_w4a8_linear(s["laid_out"], s["scale"], s["packed"], case["tokens"], case["channels"], case["width"], case["group"], s["w_scales"],
                                  out_dtype=torch.float32 if case["logits"] else torch.bfloat16)
        return {"y": y}
    if case["kind"] == "gated":
        codes, scale = fptq.fptq_gated_quantize8(s["gate"], s["up"])
        return {"codes": codes, "scale": scale}
    mode = fptq.SCALE_RMS if case["rms"] else fptq.SCALE_NONE
    codes, scale, residual = fptq.fptq_norm_quantize8(s["x"], s["residual"], s["gain"], mode, EPS)
    out = {"codes": codes, "scale": scale}
    if case["residual"]:
        out["residual"] = residual
    return out


# ---------------------------------------------------------------------------------------------------- work, checks

def work(case):
    t, k = case["tokens"], case["width"]
    if case["kind"] == "norm":
        return {"bytes": t * k * (7 if case["residual"] else 3) + 4 * t + (2 * k if case["gain"] else 0), "flops": 6 * t * k}
    if case["kind"] == "gated":
        return {"bytes": 5 * t * k + 4 * t, "flops": 8 * t * k}
    n, groups = case["channels"], -(-k // case["group"])
    return {"bytes": n * ((k + 1) // 2) + 4 * n * groups + t * k + 4 * t + t * n * (4 if case["logits"] else 2), "flops": 2 * t * n * k}


def exact(case, seed):
    """From the definition in 64 bits; codes have no such value."""
    s = prepare(case, seed)
    t, k = case["tokens"], case["width"]
    if case["kind"] == "norm":
        z = s["x"].double()
        if case["residual"]:
            z = z + s["residual"].double()
        u = z if s["gain"] is None else z * s["gain"].double()
        largest = u.abs().max(1).values
        if case["rms"]:
            largest = largest / (z.pow(2).mean(1) + EPS).sqrt()
        out = {"codes": None, "scale": largest / 127}
        if case["residual"]:
            out["residual"] = z
        return out
    if case["kind"] == "gated":
        z = s["gate"].double() * torch.sigmoid(s["gate"].double()) * s["up"].double()
        return {"codes": None, "scale": z.abs().max(1).values / 127}
    y = torch.empty((t, case["channels"]), dtype=torch.float64, device="cuda")
    x = s["codes"].double() * s["scale"].double()[:, None]
    step = max(1, (1 << 27) // k)
    for i in range(0, case["channels"], step):
        of = torch.arange(k, device="cuda") // case["group"]
        y[:, i:i + step] = x @ (s["w"][i:i + step].double() * s["w_scales"][of, i:i + step].t().double()).t()
    return {"y": y}
