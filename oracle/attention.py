"""What a decoder layer does between its QKV and its O projection, in float64 and from the definitions: rotation by position (the pair maps of
oracle.transforms' RoPE), the paged 8-bit cache with a power of two as scale of each page and head, and causal attention with grouped heads.

The paper keeps these products out of its quantized path; its RoPE is that of PAPER.md:283-302.  A head's page of the cache is kept here as
plain arrays [64 tokens, D]; `keys_page` and `values_page` put it into the library's layout."""
import numpy as np

PAGE = 64


def e4m3_values():
    """The 256 values of e4m3 (no infinities; 0x7f and 0xff are NaN)."""
    c = np.arange(256)
    s, e, m = np.where(c & 128, -1.0, 1.0), c >> 3 & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    return np.where((c & 127) == 127, np.nan, s * v)


def e4m3(x):
    """Codes of x, rounded to nearest, ties to the even code; NaN where x is not finite."""
    x = np.asarray(x, np.float64)
    grid = e4m3_values()[:127]
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0)
    i = np.clip(np.searchsorted(grid, a), 1, 126)
    low, high = a - grid[i - 1], grid[i] - a
    code = np.where((high < low) | ((high == low) & (i % 2 == 0)), i, i - 1)
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_for(largest):
    """The smallest power of two s with largest <= 448 s, 2^-100 at least."""
    mantissa, exponent = np.frexp(np.asarray(largest, np.float64) / 448.0)          # in [0.5, 1)
    return np.exp2(np.maximum(np.where(largest > 0, exponent - (mantissa == 0.5), -100), -100.0))


def rotate(x, cos, sin, interleaved):
    """x [..., D], the first 2 n values by n angles: pair i is (2 i, 2 i + 1) or (i, i + n)."""
    n = len(cos)
    first = 2 * np.arange(n) if interleaved else np.arange(n)
    second = first + 1 if interleaved else first + n
    y = np.array(x, np.float64)
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def append_page(values, scale, first, new):
    """A page-head of `first` older values [first, D] with their scale, and new ones [n, D] behind them: (all of them in 64 bits, the page's scale).  What the
    codes are is these, rounded."""
    finite = np.abs(np.where(np.isfinite(new), new, 0.0))
    s = float(scale_for(finite.max(initial=0.0)))
    if first:
        s = max(s, scale)
    return np.concatenate([values[:first], new]), s


def keys_page(codes):
    """[64, D] -> the library's [D / 64][64][64]"""
    return codes.reshape(PAGE, -1, 64).transpose(1, 0, 2).reshape(-1)


def values_page(codes):
    """[64, D] -> the library's [4][D][16]"""
    return codes.reshape(4, 16, -1).transpose(0, 2, 1).reshape(-1)


def from_keys_page(flat, D):
    return flat.reshape(D // 64, PAGE, 64).transpose(1, 0, 2).reshape(PAGE, D)


def from_values_page(flat, D):
    return flat.reshape(4, D, 16).transpose(0, 2, 1).reshape(PAGE, D)


def attention(q, k, v, scale, keys=None):
    """q [n, H, D], k and v [m, J, D]: the last query is at the last key, or token i sees the first keys[i]; a query that sees nothing gets zeros.
    Returns (out, the mean of |v| under the softmax, the
    largest sum |q k| scale of a row): what error bounds are made of."""
    n, H, D = q.shape
    m, J = k.shape[0], k.shape[1]
    keys = np.arange(n) + (m - n) + 1 if keys is None else np.asarray(keys)
    out, mass, terms = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H))
    for h in range(H):
        j = h // (H // J)
        for i in range(n):
            seen = int(keys[i])
            if seen <= 0:
                continue
            kk, vv = k[:seen, j], v[:seen, j]
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (kk @ q[i, h])
                top = s.max()
                p = np.exp(s - (top if top != -np.inf else 0.0))
                if p.sum() == 0:
                    continue
                out[i, h] = (p @ vv) / p.sum()
                mass[i, h] = (p @ np.abs(vv)) / p.sum()
                terms[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, mass, terms
