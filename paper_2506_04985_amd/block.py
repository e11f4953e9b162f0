"""A decoder layer on the library's calls.  Its attention half: quantizer, W4A4 QKV projection, rotation and paged 8-bit cache, attention,
quantizer, W4A4 O projection.  Its MLP half, with activations of 8 bits and weights of 4 bits in groups: residual and RMS norm, gate+up, gated activation, down.
`python -m paper_2506_04985_amd.block` runs prompts and a token loop on random weights (a Llama-3-8B-shaped layer) and prints how long each takes.
"""
import math

import torch

from . import binding as fptq

PAGE = 64


def rope_table(positions, rope_dims, base=500000.0, scale=1.0, device="cuda"):
    """fp32 [positions, 2, rope_dims / 2] cosines and sines of position / scale * base^(-2 i / rope_dims), angles taken in 64 bits."""
    freq = base ** (-torch.arange(0, rope_dims, 2, dtype=torch.float64, device=device) / rope_dims)
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] / scale * freq
    return torch.stack([angle.cos(), angle.sin()], 1).float()


class Attention:
    """w_qkv int8 [(heads + 2 kv_heads) * head_dim, K] and w_o int8 [N, heads * head_dim] in [-8, 7] with fp32 scales of their rows; s_x and s_o: the static
    quantizers' scales of the layer's normed input and of the attention's output."""

    def __init__(self, w_qkv, s_qkv, w_o, s_o_rows, heads, kv_heads, head_dim, s_x, s_o, rope, interleaved=False, eps=1e-5):
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.K, self.N = w_qkv.shape[1], w_o.shape[0]
        if w_qkv.shape[0] != (heads + 2 * kv_heads) * head_dim or w_o.shape[1] != heads * head_dim:
            raise ValueError(f"weights {tuple(w_qkv.shape)} and {tuple(w_o.shape)} do not go with {heads} + 2 * {kv_heads} heads of {head_dim}")
        self.w_qkv, self.w_o = fptq.fptq_pack_weights(w_qkv), fptq.fptq_pack_weights(w_o)
        self.s_qkv, self.s_o_rows, self.s_x, self.s_o = s_qkv, s_o_rows, float(s_x), float(s_o)
        self.rope, self.interleaved, self.eps = rope, interleaved, eps

    def _qkv(self, x):
        """The projection's rows [T, (heads + 2 kv_heads) * head_dim] as views of queries, keys and values."""
        H, J, D = self.heads, self.kv_heads, self.head_dim
        xq, _ = fptq.fptq_quantize_act(x, self.s_x, fptq.SCALE_RMS, self.eps, want_row_scale=False)
        y = fptq.fptq_w4a4_linear(xq, self.w_qkv, x.shape[0], (H + 2 * J) * D, self.K, self.s_x, self.s_qkv)
        q, k, v = y.split([H * D, J * D, J * D], 1)
        return q.unflatten(1, (H, D)), k.unflatten(1, (J, D)), v.unflatten(1, (J, D))

    def _o(self, out):
        rows = out.view(out.shape[0], self.heads * self.head_dim)
        oq, _ = fptq.fptq_quantize_act(rows, self.s_o, fptq.SCALE_NONE, want_row_scale=False)
        return fptq.fptq_w4a4_linear(oq, self.w_o, rows.shape[0], self.N, rows.shape[1], self.s_o, self.s_o_rows)

    def prompt(self, x, cache, table, lengths, cu):
        """Whole prompts, x bf16 [T, K] packed by cu, into empty sequences of the cache: bf16 [T, N]."""
        q, k, v = self._qkv(x)
        q, k = fptq.fptq_cache_append(q, k, v, self.rope, cache, table, lengths, cu, interleaved=self.interleaved, want_k=True)
        return self._o(fptq.fptq_prompt_attention(q, k, v, cu))

    def tokens(self, x, cache, table, lengths, cu=None):
        """The sequences' next tokens, one each or packed by cu, behind what the cache holds of them; lengths count the new ones."""
        q, k, v = self._qkv(x)
        q, _ = fptq.fptq_cache_append(q, k, v, self.rope, cache, table, lengths, cu, interleaved=self.interleaved)
        return self._o(fptq.fptq_cached_attention(q, cache, table, lengths, cu))


class Mlp:
    """w_gate_up int8 [2 F, K] (gate's rows, then up's) and w_down int8 [N, F] in [-8, 7], with fp32 scales [ceil(K / group), 2 F] and [ceil(F / group), N] of groups of `group`
    values of a row; gain bf16 [K] of the norm, or None where it is folded into the weights."""

    def __init__(self, w_gate_up, s_gate_up, w_down, s_down, group, gain=None, eps=1e-5):
        self.F, self.K, self.N, self.group = w_gate_up.shape[0] // 2, w_gate_up.shape[1], w_down.shape[0], group
        if w_gate_up.shape[0] % 2 or w_down.shape[1] != self.F:
            raise ValueError(f"weights {tuple(w_gate_up.shape)} and {tuple(w_down.shape)} do not go together")
        if tuple(s_gate_up.shape) != (-(-self.K // group), 2 * self.F) or tuple(s_down.shape) != (-(-self.F // group), self.N):
            raise ValueError(f"scales {tuple(s_gate_up.shape)} and {tuple(s_down.shape)} do not go with groups of {group}")
        self.w_gate_up, self.w_down = fptq.fptq_pack_weights(w_gate_up), fptq.fptq_pack_weights(w_down)
        self.s_gate_up, self.s_down, self.gain, self.eps = s_gate_up, s_down, gain, eps

    def __call__(self, x, residual):
        """x bf16 [T, K], the attention half's output, and the residual stream in front of it: (bf16 [T, N], the residual stream with x in it)."""
        codes, scale, residual = fptq.fptq_norm_quantize8(x, residual, self.gain, fptq.SCALE_RMS, self.eps)
        h = fptq.fptq_w4a8_linear(codes, scale, self.w_gate_up, x.shape[0], 2 * self.F, self.K, self.group, self.s_gate_up)
        codes, scale = fptq.fptq_gated_quantize8(*h.split(self.F, 1))
        return fptq.fptq_w4a8_linear(codes, scale, self.w_down, x.shape[0], self.N, self.F, self.group, self.s_down), residual


def main(prompt=4096, steps=64, sequences=4, heads=32, kv_heads=8, head_dim=128, width=4096, mlp_width=None, group=128):
    g = torch.Generator(device="cuda").manual_seed(0)
    weights = lambda n, k: torch.randint(-8, 8, (n, k), dtype=torch.int8, device="cuda", generator=g)
    rows = (heads + 2 * kv_heads) * head_dim
    s_x = 0.4
    s_qkv = torch.full((rows,), 1.0 / (s_x * math.sqrt(21.5 * 7.0 * width)), device="cuda")              # rows of about unit variance
    s_rows = torch.full((width,), 0.01, device="cuda")
    total = prompt // sequences + steps
    layer = Attention(weights(rows, width), s_qkv, weights(width, heads * head_dim), s_rows, heads, kv_heads, head_dim, s_x, 0.05, rope_table(total, head_dim))
    if mlp_width:
        unit = lambda n, k: torch.full((-(-k // group), n), 1.0 / math.sqrt(21.5 * k), device="cuda")
        mlp = Mlp(weights(2 * mlp_width, width), unit(2 * mlp_width, width), weights(width, mlp_width), unit(width, mlp_width), group,
                  torch.ones(width, dtype=torch.bfloat16, device="cuda"))
    pages = -(-total // PAGE)
    cache = fptq.Cache.empty(sequences * pages, kv_heads, head_dim)
    table = torch.randperm(sequences * pages, device="cuda", generator=g).to(torch.int32).view(sequences, pages)
    lengths = torch.full((sequences,), prompt // sequences, dtype=torch.int32, device="cuda")
    cu = torch.arange(0, prompt + 1, prompt // sequences, dtype=torch.int32, device="cuda")
    x = torch.randn((prompt, width), device="cuda", generator=g).to(torch.bfloat16)
    token = torch.randn((sequences, width), device="cuda", generator=g).to(torch.bfloat16)

    def timed(call, n):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(n):
            y = call()
        end.record()
        end.synchronize()
        return y, begin.elapsed_time(end) * 1e3 / n

    def step():
        lengths.add_(1)
        return layer.tokens(token, cache, table, lengths)

    layer.prompt(x, cache, table, lengths, cu)
    y, us = timed(lambda: layer.prompt(x, cache, table, lengths, cu), 10)
    print(f"prompts of {sequences} x {prompt // sequences} tokens: {us:.1f} us, output {tuple(y.shape)}, finite: {bool(torch.isfinite(y).all())}")
    if mlp_width:
        mlp(y, x)
        (y, _), us = timed(lambda: mlp(y, x), 10)
        print(f"their MLP half: {us:.1f} us, output {tuple(y.shape)}, finite: {bool(torch.isfinite(y).all())}")
    # the token loop as a server runs it: one captured step, replayed on growing lengths
    before = lengths.clone()
    for what, call in [("", step)] + [(", with its MLP half", lambda: mlp(step(), token)[0])] * bool(mlp_width):
        lengths.copy_(before)
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            y = call()
        _, us = timed(graph.replay, steps)
        print(f"a token of {sequences} sequences behind {prompt // sequences} to {total}{what}: {us:.1f} us, output {tuple(y.shape)}, finite: {bool(torch.isfinite(y).all())}")


if __name__ == "__main__":
    main(mlp_width=14336)
