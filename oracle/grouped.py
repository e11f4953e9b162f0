"""Activations of 8 bits with a scale for each token and weights of 4 bits with a scale for each group of K values, from the definitions, in NumPy.

The paper keeps to 4 bits on both sides; its dynamic quantization (a scale for each token at run time) is that of the paper's App. B, here on a grid of
[-127, 127].  `quantize_rows` follows the stated fp32 recipe, whose codes are unique; `residual_norm` and `gated` give its input, and the products are taken in
integers within a group and in 64 bits between groups."""
import numpy as np

KT = 128


def lay_out(codes):
    """int8 [rows, K] -> the library's layout: 128-value tiles outermost, 128 bytes a row, of every eight values the even ones first, zero-padded."""
    rows, K = codes.shape
    tiles = -(-K // KT)
    padded = np.zeros((rows, tiles * KT), np.int8)
    padded[:, :K] = codes
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    return np.ascontiguousarray(padded.reshape(rows, tiles, KT // 8, 8)[..., order].transpose(1, 0, 2, 3)).reshape(-1)


def quantize_rows(u, inv=None):
    """(codes int8, scales fp32) of fp32 rows u: a = max |u| (at least 2^-100), code = rne(u (127 / a)), scale = (a inv) (1 / 127), all fp32.  A row of zeros has scale
    0; one with a value that is not finite has codes 0 and scale NaN."""
    u = np.asarray(u, np.float32)
    finite = np.isfinite(u).all(1)
    safe = np.where(finite[:, None], u, np.float32(0))
    largest = np.abs(safe).max(1)
    a = np.maximum(largest, np.float32(2.0 ** -100))
    codes = np.rint(safe * (np.float32(127) / a)[:, None]).astype(np.int8)
    scale = (a if inv is None else a * np.asarray(inv, np.float32)) * np.float32(1.0 / 127.0)
    scale = np.where(largest == 0, np.float32(0), scale)
    return codes, np.where(finite, scale, np.float32(np.nan)).astype(np.float32)


def residual_norm(x, residual=None, gain=None, eps=None):
    """(z, u, inv) in fp32 of rows that bf16 holds: z = x + residual, u = z gain, inv = 1 / sqrt(mean z^2 + eps) with the mean in 64 bits (None without eps)."""
    with np.errstate(over="ignore", invalid="ignore"):
        z = np.asarray(x, np.float32)
        if residual is not None:
            z = z + np.asarray(residual, np.float32)
        u = z if gain is None else z * np.asarray(gain, np.float32)
        inv = None
        if eps is not None:
            inv = (1.0 / np.sqrt((z.astype(np.float64) ** 2).sum(1) / z.shape[1] + float(np.float32(eps)))).astype(np.float32)
    return z, u, inv


def silu(g):
    """g / (1 + e^-g) of what bf16 holds, rounded once to fp32."""
    g = np.asarray(g, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        return (g / (1.0 + np.exp(-g))).astype(np.float32)


def gated(gate, up):
    with np.errstate(over="ignore", invalid="ignore"):
        return silu(gate) * np.asarray(up, np.float32)


def linear(codes, token_scale, w, group, w_scales):
    """(y, mass) in 64 bits: y[t, n] = token_scale[t] sum_g w_scales[g, n] (sum_k codes w), and what the magnitudes of its terms add up to, a term being a group's or at most 128
    values' integer sum."""
    codes, w = np.asarray(codes, np.float64), np.asarray(w, np.float64)
    (T, K), N = codes.shape, w.shape[0]
    y, mass = np.zeros((T, N)), np.zeros((T, N))
    for k in range(0, K, min(group, KT)):
        part = codes[:, k:k + min(group, KT)] @ w[:, k:k + min(group, KT)].T            # integers below 2^53: exact
        term = part * np.asarray(w_scales, np.float64)[k // group]
        y, mass = y + term, mass + np.abs(term)
    s = np.asarray(token_scale, np.float64)[:, None]
    return s * y, np.abs(s) * mass
