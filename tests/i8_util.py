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


# (rows, output columns, K) that take the instances of the product's kernels: tile heights, widths, wavefronts, weights
# read once or more often, K cut or whole, K shared out inside a workgroup
PLANS = [
    (1, 1, 248), (1, 4097, 40), (1, 4103, 13218), (1, 4098, 1895), (1, 9067, 19122), (17, 1, 1536),
    (17, 1, 64), (17, 1, 6144), (17, 1, 640), (18, 10888, 3358), (65, 1, 28), (49, 1, 5012), (33, 1, 460),
    (1346, 1046, 36), (1539, 1, 8094), (33, 4099, 54), (33, 1, 5964), (39, 4112, 763), (227, 13202, 289),
    (225, 2207, 16830), (33, 8215, 5778), (130, 16234, 1940), (2305, 1, 7048), (194, 21758, 6000),
    (195, 4206, 10829), (791, 12340, 839), (200, 8306, 14610), (173, 16343, 3870), (2689, 1, 8084),
    (2087, 2305, 10), (324, 2730, 16238), (65, 5429, 11580), (2265, 4624, 365), (262, 8294, 14608),
    (196, 16340, 10420), (2245, 132, 12217), (2507, 2322, 501), (195, 4533, 16942), (2977, 4231, 14),
    (292, 8194, 14682), (2310, 1544, 178), (2046, 268, 15030), (65, 16404, 5), (72, 5418, 12630),
    (2635, 2604, 399), (244, 4151, 16985), (97, 8249, 9360), (2906, 5258, 24), (228, 10971, 17061),
    (2307, 1667, 264), (129, 5489, 6624), (257, 30016, 5681), (264, 4367, 17053), (2890, 5638, 56),
    (259, 16440, 16499), (2003, 2314, 49), (145, 4123, 13978), (2250, 4125, 1457), (291, 8328, 14291),
    (129, 8307, 12002), (873, 6491, 126), (162, 4137, 14093), (868, 12864, 984), (337, 8362, 16023),
    (2702, 2078, 204), (181, 4367, 15882), (2702, 4174, 2256), (178, 8233, 14213), (610, 21699, 1615),
    (2594, 5180, 5702), (194, 8325, 16105), (1154, 12872, 3766), (727, 21562, 53), (228, 11360, 17800)]
