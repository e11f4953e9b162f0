"""The MLP half of a decoder layer, step by step against the oracle on what the step before it gave, and captured as a server runs it."""
import numpy as np
import pytest
import torch

from oracle import grouped
from paper_2506_04985_amd import binding as fptq
from paper_2506_04985_amd import block
from test_gpu_grouped_linear import check

pytestmark = pytest.mark.gpu
host = lambda t: t.detach().cpu().float().numpy()


def layer(K, F, N, group, gain, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = [torch.randint(-8, 8, s, dtype=torch.int8, device="cuda", generator=g) for s in ((2 * F, K), (N, F))]
    s = [0.02 * torch.rand((-(-k // group), n), device="cuda", generator=g) for n, k in ((2 * F, K), (N, F))]
    gain = (1 + 0.2 * torch.randn((K,), device="cuda", generator=g)).to(torch.bfloat16) if gain else None
    return w, s, block.Mlp(w[0], s[0], w[1], s[1], group, gain)


@pytest.mark.parametrize("T,K,F,N,group,gain", [(1, 256, 640, 256, 128, True), (37, 320, 333, 96, 64, False), (300, 512, 1000, 512, 32, True)])
def test_steps(T, K, F, N, group, gain, monkeypatch):
    (w1, w2), (s1, s2), mlp = layer(K, F, N, group, gain)
    seen = []
    for name in ("fptq_norm_quantize8", "fptq_w4a8_linear", "fptq_gated_quantize8"):
        def spy(*args, call=getattr(fptq, name)):
            seen.append(call(*args))
            return seen[-1]
        monkeypatch.setattr(fptq, name, spy)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn((T, K), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    y, residual = mlp(x, r)
    (c1, t1, z), h, (c2, t2), out = seen
    assert y is out and residual is z and torch.equal(z, (x.float() + r.float()).to(torch.bfloat16))
    _, u, inv = grouped.residual_norm(host(x), host(r), None if mlp.gain is None else host(mlp.gain), 1e-5)
    q, t = grouped.quantize_rows(u, inv)
    assert np.array_equal(c1.cpu().numpy(), grouped.lay_out(q)) and np.abs(t1.cpu().numpy().view(np.int32) - t.view(np.int32)).max() <= 1
    check(h, *grouped.linear(q, t1.cpu().numpy(), w1.cpu().numpy(), group, s1.cpu().numpy()), K, group)
    q, t = grouped.quantize_rows(grouped.gated(host(h[:, :F]), host(h[:, F:])))
    assert np.array_equal(c2.cpu().numpy(), grouped.lay_out(q)) and np.array_equal(t2.cpu().numpy(), t)
    check(out, *grouped.linear(q, t, w2.cpu().numpy(), group, s2.cpu().numpy()), F, group)


def test_weights_and_scales_that_do_not_go_together():
    w = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda")
    f = lambda *s: torch.zeros(s, device="cuda")
    for a in ((w(64, 32), f(1, 64), w(32, 31), f(1, 32)), (w(63, 32), f(1, 63), w(32, 31), f(1, 32)), (w(64, 32), f(64, 1), w(32, 32), f(1, 32)), (w(64, 32), f(1, 64), w(32, 32), f(2, 32))):
        with pytest.raises(ValueError):
            block.Mlp(*a, 128)


@pytest.mark.parametrize("T", [1, 24, 200])
def test_captured(T):
    """Two graphs of two layers, replayed in turn on changing inputs with eager calls between them; scratch (a long F against few outputs) comes from the captures' pools."""
    K, F, N, group = 128, 6000, 128, 128
    layers = [layer(K, F, N, group, True, seed)[2] for seed in (0, 1)]
    xs, rs = [[torch.empty((T, K), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    fptq.fptq_init()
    graphs, outs = [], []
    for l, x, r in zip(layers, xs, rs):
        x.zero_(), r.zero_()
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            outs.append(l(x, r))
        graphs.append(graph)
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        want = []
        for i in (0, 1):
            xs[i].copy_(torch.randn((T, K), device="cuda", generator=g)), rs[i].copy_(torch.randn((T, K), device="cuda", generator=g))
            want.append(tuple(v.clone() for v in layers[i](xs[i], rs[i])))
        graphs[0].replay(), graphs[1].replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])


def test_the_command_runs_it(capsys):
    block.main(prompt=256, steps=3, sequences=2, heads=4, kv_heads=2, head_dim=64, width=256, mlp_width=500, group=64)
    lines = capsys.readouterr().out.strip().splitlines()
    assert len(lines) == 4 and all("finite: True" in l for l in lines)


def test_the_command_times_no_first_call(monkeypatch, capsys):
    """What it prints holds no call that allocates: each half runs once before its prompts are timed."""
    events, record = [], torch.cuda.Event.record
    monkeypatch.setattr(torch.cuda.Event, "record", lambda self, *a: (events.append("time"), record(self, *a))[1])
    for kind, name in ((block.Attention, "prompt"), (block.Mlp, "__call__")):
        def spy(self, *a, call=getattr(kind, name), kind=kind):
            events.append(kind.__name__)
            return call(self, *a)
        monkeypatch.setattr(kind, name, spy)
    block.main(prompt=256, steps=3, sequences=2, heads=4, kv_heads=2, head_dim=64, width=256, mlp_width=500, group=64)
    half = lambda name: [name, "time"] + 10 * [name] + ["time"]
    assert events[:26] == half("Attention") + half("Mlp")
