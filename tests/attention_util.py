"""Shared by the tests of the attention operators: inputs, and how far outputs may be from the oracle's."""
import numpy as np
import torch

PAGE = 64


def device(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def host(t):
    """A bf16 tensor's values in 64 bits."""
    return t.detach().cpu().double().numpy()


def projection(g, tokens, H, J, D, spread=1.0):
    """Rows of a QKV projection and the three views of them."""
    x = torch.randn((tokens, (H + 2 * J) * D), device="cuda", generator=g) * spread
    x = x.to(torch.bfloat16)
    q, k, v = x.split([H * D, J * D, J * D], 1)
    return q.unflatten(1, (H, D)), k.unflatten(1, (J, D)), v.unflatten(1, (J, D))


def starts(new):
    return [0, *np.cumsum(new).tolist()]


def paged(lengths, spare=3, seed=0):
    """(table with pages in a shuffled order and numbers outside the pool where no page is needed, pages of the pool)"""
    rng = np.random.default_rng(seed)
    need = [-(-max(n, 0) // PAGE) for n in lengths]
    pool = sum(need) + spare
    order, table, at = rng.permutation(pool), np.full((len(lengths), max(1, *need) + 1), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    table[:, -1] = pool + 7
    return table, pool


def tolerance(out, mass, terms, D):
    """Bound of the error of a bf16 output, value by value.  Weights are rounded to bf16 (2^-8 of each term, so of `mass`, the mean |v|), and so is the output
    (2^-8).  A score is a sum of D fp32 products: D 2^-24 of `terms`, their absolute sum, twice that for the maximum that it is taken from; the weight's
    exponential 2^-20.  Sums of weights and outputs in fp32 stay below 2^-16 (up to 2^8 page or tile sums in a row)."""
    weight = 2.0 ** -8 + 2 * D * 2.0 ** -24 * terms[..., None] + 2.0 ** -20 + 2.0 ** -16
    return 1.01 * (2 * weight * mass + 2.0 ** -8 * np.abs(out)) + 1e-30


def check(got, out, mass, terms, D):
    got = host(got)
    assert got.shape == out.shape
    finite = np.isfinite(out)
    assert np.array_equal(finite, np.isfinite(got)), "where outputs are finite"
    far = np.abs(got - out)[finite] / tolerance(out, mass, terms, D)[finite]
    assert far.size == 0 or far.max() <= 1.0, f"{far.max()} of the bound"

