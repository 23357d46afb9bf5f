"""The weight gradient from 8 bits and the product of rows in 4 bits on inputs whose results are exact in fp32
(``mx_exact``): every bit has to be there, where a bound over long sums lets a lost part, row or block pass."""
import numpy as np
import pytest
import torch

import mx_exact as E
from mx_helpers import host, matmul, matrix, upload, wgrad
from oracle import mx
from paper_2203_10428_amd import binding as B

pytestmark = pytest.mark.gpu


def check_wgrad(code, s, J, H, f_in, f_out, dtype):
    Q, S = upload(code, s, "int8")
    dW = wgrad(Q, S, matrix(J), None if H is None else matrix(H, pad=16), len(J), f_in, f_out, dtype)
    torch.cuda.synchronize()
    if H is not None:
        J = np.where(H > 0, J, 0.0)
    want = mx.wgrad(mx.values(code, s, f_in, "int8"), E.bf16(J) if dtype == "bf16" else J)
    assert np.array_equal(dW[:f_in * f_out].view(f_in, f_out).cpu().numpy(), want)
    assert (dW[f_in * f_out:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("rows,f_in,f_out", E.WGRAD)
def test_every_bit_of_the_gradient_is_used(rows, f_in, f_out, masked, dtype):
    code, s, J = E.one_row(rows + f_out, rows, f_in, f_out)
    H = E.mask(np.random.default_rng(rows), rows, f_out) if masked else None
    check_wgrad(code, s, J, H, f_in, f_out, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("rows,f_in,f_out", E.WGRAD)
def test_every_row_counts_once(rows, f_in, f_out, masked, dtype):
    code, s, J = E.integers(rows + f_out, rows, f_in, f_out, dtype)
    H = E.mask(np.random.default_rng(rows), rows, f_out) if masked else None
    check_wgrad(code, s, J, H, f_in, f_out, dtype)


def check_product(m, n, k, dtype, signed, relu):
    a, b = E.product(m + n + k, m, n, k, signed)
    C = matmul(*upload(*a, "fp4"), *upload(*b, "fp4", (0, 0)), m, n, k, dtype, relu)
    torch.cuda.synchronize()
    want = mx.product(mx.values(*a, k, "fp4"), mx.values(*b, k, "fp4"), relu)
    assert np.array_equal(host(C[:m], n), E.bf16(want) if dtype == "bf16" else want)
    assert (C[:m, n:] == 77).all() and (C[m:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", E.PRODUCT)
def test_products_are_exact(m, n, k, dtype):
    check_product(m, n, k, dtype, True, (m + n) % 2 == 0)


@pytest.mark.parametrize("k", E.SLABS)
@pytest.mark.parametrize("m,n", [(70, 3), (1, 90), (16, 16)])
def test_every_block_counts_once(m, n, k):
    check_product(m, n, k, "f32", False, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("signed", [False, True])
@pytest.mark.parametrize("m,n,k", E.LONG)
def test_every_block_of_a_long_row_counts_once(m, n, k, signed, dtype):
    assert B.pgcn_mx_matmul_workspace_size(B.PGCN_F32, m, n, k) >= 2 * 4 * m * n
    check_product(m, n, k, dtype, signed, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(64, 64), (200, 100), (2100, 2050), (2048, 2176), (4096, 4096), (4100, 4090)])
def test_results_of_every_tile_are_in_their_place(m, n, dtype):
    """Rows of a tile go through LDS, which one lane writes and another reads, and the next rows after them: products of
    one term, a sign and a power of two that tell neighbouring rows and columns apart, several times over the same output."""
    rng = np.random.default_rng(m)
    side = lambda rows: (np.concatenate((rng.choice([1, 2, 4, 10], (rows, 1)), np.zeros((rows, 31), np.int64)), axis=1),
                         rng.integers(100, 150, (rows, 1)))
    a, b = side(m), side(n)
    held = upload(*a, "fp4"), upload(*b, "fp4")
    want = torch.from_numpy(mx.product(mx.values(*a, 1, "fp4"), mx.values(*b, 1, "fp4"))).cuda()
    C = None
    for _ in range(5):
        C = matmul(*held[0], *held[1], m, n, 1, dtype, out=C)
        torch.cuda.synchronize()
        assert torch.equal(C[:m, :n].double(), want)
        C[:m, :n] = 5.0
