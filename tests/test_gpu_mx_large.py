"""Rows in 8 and 4 bits past 32-bit offsets: matrices of more than 4 GiB, of which the last rows hold something.

Bounds as in the operators' own tests: a product of k terms is off by at most 2 (k + 64) u sum |a b|, a weight gradient of
rows by (2 rows + 260) u sum |v J|, where only the rows that hold something count; u = 2^-24."""
import numpy as np
import pytest
import torch

from mx_helpers import U, dequantize, host, matmul, matrix, quantize, upload, wgrad
from oracle import mx

pytestmark = pytest.mark.gpu


def tall(rows, ld, last, filled):
    """A byte matrix of zeros, with `last` in its last rows."""
    t = torch.zeros(rows, ld, dtype=torch.uint8, device="cuda")
    t[rows - filled:, :last.shape[1]] = torch.from_numpy(last.astype(np.uint8)).cuda()
    return t


def sides(rows, k, filled, rng):
    code, s = mx.quantize(rng.standard_normal((filled, k)), "fp4")
    b = mx.to_bytes(code, "fp4")
    return code, s, tall(rows, b.shape[1], b, filled), tall(rows, (s.shape[1] + 3) // 4 * 4, s, filled)


def check(C, a, b, k):
    want, size = mx.product(a, b), np.abs(a) @ np.abs(b).T
    assert (np.abs(C - want) <= 2 * (k + 64) * U * size + 2.0 ** -120).all()


@pytest.mark.parametrize("m", [3, 40])
def test_product_with_more_than_4_gib_of_b(m):
    k, n, filled = 100_000, 90_000, 20
    rng = np.random.default_rng(m)
    code, s, Bq, SB = sides(n, k, filled, rng)
    assert Bq.numel() > 1 << 32
    a = mx.quantize(rng.standard_normal((m, k)), "fp4")
    C = matmul(*upload(*a, "fp4"), Bq, SB, m, n, k, "f32")
    torch.cuda.synchronize()
    check(host(C[:m, n - filled:n]), mx.values(*a, k, "fp4"), mx.values(code, s, k, "fp4"), k)
    assert (C[:m, :n - filled] == 0).all()


def test_product_with_more_than_4_gib_of_a_and_of_c():
    k, m, n, filled = 9_000, 1_000_000, 1_100, 20
    rng = np.random.default_rng(7)
    code, s, A, SA = sides(m, k, filled, rng)
    assert A.numel() > 1 << 32
    b = mx.quantize(rng.standard_normal((n, k)), "fp4")
    C = matmul(A, SA, *upload(*b, "fp4"), m, n, k, "f32")
    assert C.numel() * 4 > 1 << 32
    torch.cuda.synchronize()
    check(host(C[m - filled:m], n), mx.values(code, s, k, "fp4"), mx.values(*b, k, "fp4"), k)
    assert (C[:m - filled, :n] == 0).all() and (C[m:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_gradient_of_more_than_4_gib(dtype):
    rows, f_in, f_out, filled = 1_500_000, 70, 40, 25
    rng = np.random.default_rng(3)
    code, s = mx.quantize(rng.standard_normal((filled, f_in)), "int8")
    Q = tall(rows, 2912, mx.to_bytes(code, "int8"), filled)      # a wide stride
    S = tall(rows, 4, s, filled)
    assert Q.numel() > 1 << 32
    J = torch.ones(rows, 720, device="cuda")                           # 4.3 GB; its rows meet zeros but for the last
    last = rng.standard_normal((filled, f_out)).astype(np.float32)
    J[rows - filled:, :f_out] = torch.from_numpy(last).cuda()
    H = torch.ones(rows, f_out, device="cuda")
    H[rows - 3:] = 0.0
    dW = wgrad(Q, S, J, H, rows, f_in, f_out, dtype)
    torch.cuda.synchronize()
    v, j = mx.values(code, s, f_in, "int8"), last.astype(np.float64)
    j[-3:] = 0.0
    if dtype == "bf16":
        j = torch.from_numpy(j).float().to(torch.bfloat16).double().numpy()
    got = dW[:f_in * f_out].view(f_in, f_out).cpu().numpy().astype(np.float64)
    assert (np.abs(got - mx.wgrad(v, j)) <= (2 * rows + 260) * U * (np.abs(v).T @ np.abs(j)) + 2.0 ** -126).all()
    assert np.abs(got - mx.wgrad(v, j)).max() < 1e-3                   # the zeros round nothing


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
def test_rows_of_more_than_4_gib_written_and_read(fmt):
    rows, cols, filled = 2_200_000, 500, 30
    X = torch.zeros(rows, 504, device="cuda")
    assert X.numel() * 4 > 1 << 32
    x = np.random.default_rng(5).standard_normal((filled, cols)).astype(np.float32).astype(np.float64)
    X[rows - filled:, :cols] = torch.from_numpy(x.astype(np.float32)).cuda()
    Q, S = quantize(X, cols, fmt)
    y = dequantize(Q, S, rows, cols, fmt)
    torch.cuda.synchronize()
    assert np.array_equal(host(y[rows - filled:rows], cols), mx.values(*mx.quantize(x, fmt), cols, fmt))
    assert (y[:rows - filled, :cols] == 0).all() and (y[:, cols:] == 77).all()


def test_transpose_of_more_than_4_gib():
    rows, cols = 270_000, 8_200
    X = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    assert X.numel() * 2 > 1 << 32
    x = np.random.default_rng(6).standard_normal((40, cols))
    X[rows - 40:] = torch.from_numpy(x).cuda().to(torch.bfloat16)
    Q, S = quantize(X, cols, "fp4", "bf16", transpose=True)
    y = dequantize(Q, S, cols, rows, "fp4", "bf16", out=torch.empty(cols, (rows + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    first = rows - 40 - (rows - 40) % 32                               # whole blocks from here on
    want = np.zeros((cols, rows - first))
    want[:, -40:] = host(X[rows - 40:]).T
    assert np.array_equal(host(y[:, first:rows]), mx.values(*mx.quantize(want, "fp4"), rows - first, "fp4"))
    assert (y[:, :first] == 0).all()


def test_matrix_helper_is_exact():
    x = np.random.default_rng(1).standard_normal((3, 5)).astype(np.float32).astype(np.float64)
    assert np.array_equal(host(matrix(x), 5), x)
