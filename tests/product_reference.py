"""Plain forms of the products and of the quantisation in front of them, on the host, and what their results are held to.

Integer products are exact, so their results are compared bit for bit: one conversion of the sum to fp32, two fp32
products, one rounding.  fp32 and bf16 products are compared bit for bit on small whole numbers, whose sums fp32 holds
exactly in any order, and within a bound on drawn ones."""
import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}       # half a step, relative to the value


def quantize(x: np.ndarray):
    """float32 [rows][K] -> codes, scales by the definition, in IEEE fp32."""
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        amax = np.abs(x).max(axis=1)
        fine = np.isfinite(x).all(axis=1)
        scale = np.maximum(amax / np.float32(127.0), np.float32(2.0 ** -126))
        scale = np.where(amax > 0, scale, np.float32(1.0)).astype(np.float32)
        codes = np.rint((x / scale[:, None]).astype(np.float32))
        codes = np.where(fine[:, None], codes, 0.0)
    assert np.abs(codes).max(initial=0) <= 127
    return codes.astype(np.int8), np.where(fine, scale, np.float32(np.nan)).astype(np.float32)


def rows_of(sizes, off, M):
    """(group, first, last) of the groups that have rows; offsets outside [0, M] count as the nearer end."""
    for g in range(len(off) - 1):
        lo = min(max(int(off[g]), 0), M)
        hi = min(max(int(off[g + 1]), lo), M)
        if hi > lo:
            yield g, lo, hi


def _rounded(x: np.ndarray, dtype) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype)


def product(x, w, xs=None, ws=None):
    """One group's product.  int8: (fp32 result, None); otherwise (float64 result, bound of its fp32 sums)."""
    if x.dtype == np.int8:
        # whole numbers below 2^53: exact in float64, whatever the order
        acc = (x.astype(np.float64) @ w.astype(np.float64).T).astype(np.int64)
        with np.errstate(over="ignore", invalid="ignore"):
            return acc.astype(np.float32) * xs[:, None] * ws[None, :], None
    x, w = x.astype(np.float64), w.astype(np.float64)
    # each of up to K additions is off by at most a unit in the last place of a partial sum, 2^-23 of the sum of magnitudes
    return x @ w.T, x.shape[1] * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)


def gated(g, eg, u, eu, dtype):
    """silu(g) * u in 64 bits and its bound.  Integer products hold g and u to the last bit; fp32 ones to eg and eu.
    silu(g) = g / (1 + exp(-g)) in fp32: exp(-g) is off by |g| + 2 half steps (its argument's product with log2(e), the
    power), the sum, the division and the product with u by one each; silu changes by at most 1.1 of a change of g.  Where
    exp(-g) passes the largest fp32 number (g < -128 ln 2 = -88.7) silu is 0 in place of |g| exp(g) < 88.8 / 2^128 < 2^-121."""
    g, u = g.astype(np.float64), u.astype(np.float64)
    silu = g / (1.0 + np.exp(np.minimum(-g, 700.0)))
    y = silu * u
    bound = np.abs(y) * (U[dtype] * (1 + 2.0 ** -8) + 2.0 ** -24 * (2 * np.abs(g) + 10)) + 2.0 ** -126 + np.where(g < -88.0, 2.0 ** -121, 0.0) * np.abs(u)
    if eg is not None:
        bound = bound + 1.1 * eg * np.abs(u) + np.abs(silu) * eu + 1.1 * eg * eu
    return y, bound
