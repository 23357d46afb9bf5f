"""Inputs of the operators in 8 and 4 bits whose results are exact in fp32, whatever the order of the sums.

Weight gradient, "one row": a feature has one non-zero value, a power of two, in a row of its own, so dW is that value
times J of the row: fp32's 24 bits in three parts of 8, added without a rounding.  "Integers": values and gradients are
integers and sum |v J| stays below 2^23, with the parts of J, which are integers too and together at most |J| (1 + 2^-6),
below 2^24.  Product: terms are multiples of 1/16 and sum |a b| stays below 2^20.  So a result that lacks a part, a
row or a block, or counts one twice, is another one."""
import numpy as np

from oracle import mx


def bf16(x):
    """x rounded to bf16, nearest even (finite, no overflow)."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def parts(x):
    """Three bf16 parts of fp32 numbers: the high half, what is left rounded to nearest, and the rest."""
    x = np.asarray(x, np.float32)
    a = (x.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32).astype(np.float64)
    b = bf16(x - a)
    return a, b, x - a - b


def mask(rng, rows, cols):
    return np.maximum(rng.standard_normal((rows, cols)), 0)


def one_row(seed, rows, f_in, f_out):
    """(code, s, J): feature i is non-zero in row at[i] alone, the first and the last row among them."""
    rng = np.random.default_rng(seed)
    at = rng.integers(0, rows, f_in)
    at[0], at[-1] = 0, rows - 1
    if f_in > 4:                                    # around the slabs of 16 rows and the ends of the matrix
        at[1:4] = np.clip([15, 16, rows - 2], 0, rows - 1)
    v = np.zeros((rows, f_in))
    v[at, np.arange(f_in)] = (2.0 ** rng.integers(-3, 4, rows))[at] * rng.choice([-1.0, 1.0], f_in)
    code, s = mx.quantize(v, "int8")
    assert np.array_equal(mx.values(code, s, f_in, "int8"), v)
    J = (1e-3 * rng.standard_normal((rows, f_out))).astype(np.float32)
    return code, s, (J.view(np.uint32) | np.uint32(1)).view(np.float32).astype(np.float64)


def integers(seed, rows, f_in, f_out, dtype):
    """(code, s, J), no value zero."""
    rng = np.random.default_rng(seed)
    budget = (1 << 23) // rows
    top_v = int(np.clip(budget ** 0.4, 1, 127))
    top_j = min(budget // top_v, 256 if dtype == "bf16" else 1 << 20)
    sign = lambda n: rng.choice([-1, 1], n)
    code = np.zeros((rows, mx.blocks(f_in) * 32), np.int64)
    code[:, :f_in] = rng.integers(1, top_v + 1, (rows, f_in)) * sign((rows, f_in))
    s = np.full((rows, mx.blocks(f_in)), 133)       # steps of 1
    J = (rng.integers(1, top_j + 1, (rows, f_out)) * sign((rows, f_out))).astype(np.float64)
    assert (np.abs(code[:, :f_in]).T @ np.abs(J)).max() <= 1 << 23
    return code, s, J


def rows_in_4_bits(rng, rows, k, signed):
    """(code, s) of rows without zeros among their k elements, scales 1/2, 1 and 2."""
    code = np.zeros((rows, mx.blocks(k) * 32), np.int64)
    code[:, :k] = rng.integers(1, 8, (rows, k)) + (8 * rng.integers(0, 2, (rows, k)) if signed else 0)
    return code, rng.integers(126, 129, (rows, mx.blocks(k)))


def product(seed, m, n, k, signed):
    rng = np.random.default_rng(seed)
    a, b = rows_in_4_bits(rng, m, k, signed), rows_in_4_bits(rng, n, k, signed)
    assert (np.abs(mx.values(*a, k, "fp4")) @ np.abs(mx.values(*b, k, "fp4")).T).max() < 1 << 20
    return a, b


# rows, f_in, f_out: one row to many splits, rows behind the last slab, each tile height and both widths
WGRAD = [(1, 1, 1), (1, 33, 7), (15, 5, 100), (16, 32, 16), (17, 129, 65), (33, 96, 128), (100, 602, 41), (257, 256, 256), (1500, 100, 130),
         (4099, 300, 47), (3000, 513, 260), (700, 1025, 8), (64, 40, 1500), (20000, 128, 128), (2000, 300, 130), (999, 540, 200),
         (50, 384, 100), (35, 257, 65), (9001, 602, 256)]

# m, n, k: every number of slabs around the stages, long rows in parts, tiles of 64, 128 and 256 with ragged edges
PRODUCT = [(1, 1, 1), (1, 100, 4096), (3, 513, 1000), (16, 16, 128), (17, 31, 127), (64, 64, 512), (65, 130, 515), (129, 257, 96), (700, 47, 100),
           (513, 769, 1030), (2050, 2100, 290), (2049, 2176, 1200), (4100, 4000, 600), (4090, 4200, 70)]
SLABS = [32, 256, 257, 512, 600, 768, 1000, 1024, 1030, 1280, 1500, 1800, 2048, 2100, 2400]
LONG = [(1, 40, 20000), (1, 1, 70000), (9, 130, 9001), (16, 33, 16384), (100, 90, 9000), (17, 5, 40000), (129, 200, 4100), (64, 64, 2048)]
