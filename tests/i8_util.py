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
    (1, 1, 248), (1, 4097, 40), (1, 4101, 11172), (1, 4098, 1895), (1, 16396, 7593), (17, 1, 1600),
    (17, 1, 64), (17, 1, 6144), (17, 1, 448), (17, 10881, 3436), (65, 1, 28), (49, 1, 4948), (33, 1, 460),
    (1346, 1032, 50), (1539, 1, 8094), (33, 4101, 52), (33, 1, 5900), (33, 4108, 813), (436, 8259, 865),
    (65, 5380, 7281), (33, 8215, 5778), (130, 16115, 2067), (2305, 1, 7048), (195, 21603, 5712),
    (194, 4106, 12028), (792, 12385, 719), (197, 8302, 13867), (163, 16378, 4101), (2689, 1, 8084),
    (2087, 2305, 10), (329, 2714, 16539), (65, 5440, 10993), (2311, 4740, 283), (261, 8289, 14620),
    (199, 16313, 8954), (2245, 132, 12217), (777, 7711, 438), (197, 5497, 17244), (2977, 4231, 14),
    (294, 8299, 16539), (2309, 1537, 192), (2018, 257, 16597), (68, 16530, 358), (71, 5438, 11401),
    (2835, 2352, 327), (248, 4105, 15147), (97, 8245, 8788), (2896, 5263, 29), (354, 8323, 17151),
    (2201, 1801, 208), (135, 3209, 16114), (257, 30677, 4016), (257, 4367, 15698), (2902, 5635, 35),
    (259, 16440, 16499), (2001, 2309, 8), (153, 4097, 13112), (725, 12989, 1596), (291, 4391, 18744),
    (132, 8330, 11634), (866, 6450, 32), (162, 4396, 14454), (483, 21592, 627), (343, 8236, 14639),
    (2429, 2309, 204), (177, 5385, 12776), (566, 21691, 543), (354, 9007, 18407), (161, 9005, 14284),
    (587, 21578, 825), (386, 9332, 17758), (644, 21612, 620), (193, 8798, 15479), (678, 21683, 1251),
    (722, 21739, 799), (227, 10882, 16461),
    (1, 32804, 60), (17, 33119, 17), (33, 33616, 64), (67, 33345, 33), (97, 33354, 20), (148, 83564, 50),
    (165, 90599, 64), (436, 4379, 31400), (201, 89937, 48), (459, 4381, 29230), (482, 4401, 37888),
    (242, 83836, 63)]
