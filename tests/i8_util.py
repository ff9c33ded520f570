"""Model of the operators of 8-bit linear layers: codes by single float32 operations (numpy rounds each of them as
IEEE 754 says, so codes are compared to the bit), products in whole numbers, scales and outputs in 64 bits."""
import numpy as np

TINY = np.float32(2.0 ** -119)


def up(n, to):
    return -(-n // to) * to


def tile(codes):
    """Row-major int8 [R, K] as the padded tiles of 16 rows x 64 columns, by the formula of each element's place."""
    R, K = codes.shape
    kt = up(K, 64) // 64
    out = np.zeros(up(R, 16) * kt * 64, np.int8)
    r, k = np.arange(R)[:, None], np.arange(K)[None, :]
    out[((r // 16) * kt + k // 64) * 1024 + (k % 64 // 16) * 256 + (r % 16) * 16 + k % 16] = codes
    return out


def codes_of(t):
    """(int8 codes, 127 / m applied, float32 m / 127) of float32 rows t."""
    t = np.asarray(t, np.float32)
    with np.errstate(all="ignore"):
        m = np.abs(t).max(1)
        fine = np.isfinite(t).all(1)
        ok = fine & (m >= TINY)
        inv = np.where(ok, np.float32(127) / np.where(ok, m, 1), np.float32(0)).astype(np.float32)
        codes = np.where(ok[:, None], np.rint(t * inv[:, None]), 0)
        unit = np.where(ok, np.where(ok, m, 0) / np.float32(127), np.float32(0)).astype(np.float32)
    return codes.astype(np.int8), np.where(fine, unit, np.float32(np.nan))


def norm_rows(x, rows, g, eps):
    """(float32 x * g of the rows, 64-bit 1 / sqrt(mean(x^2) + eps)); zeros where rows has none of x's."""
    x = np.asarray(x, np.float32)
    if rows is not None:
        rows = np.asarray(rows)
        ok = (rows >= 0) & (rows < len(x))
        x = np.where(ok[:, None], x[np.where(ok, rows, 0)], np.float32(0))
    with np.errstate(all="ignore"):
        return x * np.asarray(g, np.float32)[None, :], 1 / np.sqrt((x.astype(np.float64) ** 2).mean(1) + eps)


def product(a, sa, b, sb):
    """64-bit (a . b^T) sa sb; the whole numbers are exact (below 2^53)."""
    acc = a.astype(np.float64) @ b.astype(np.float64).T
    return acc * np.asarray(sa, np.float64)[:, None] * np.asarray(sb, np.float64)


def silu(z):
    with np.errstate(over="ignore"):
        return z / (1 + np.exp(-z))
