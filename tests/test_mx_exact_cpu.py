"""The exact inputs of the operators in 8 and 4 bits tell wrong results from right ones: mistakes planted in the oracle's
sums, on the CPU, change them.  Sums in fp32, in several orders, give the exact results."""
import numpy as np
import pytest

import mx_exact as E
from oracle import mx


def test_parts_add_up_and_have_8_bits():
    x = np.float32(1e-3) * np.random.default_rng(1).standard_normal(4000).astype(np.float32)
    a, b, c = E.parts(x)
    assert np.array_equal(a + b + c, x.astype(np.float64))
    for p in (a, b, c):
        assert np.array_equal(E.bf16(p), p)


@pytest.mark.parametrize("rows,f_in,f_out", E.WGRAD)
def test_a_lost_part_of_the_gradient_shows(rows, f_in, f_out):
    code, s, J = E.one_row(rows + f_out, rows, f_in, f_out)
    v = mx.values(code, s, f_in, "int8")
    want, p = mx.wgrad(v, J), E.parts(J)
    assert np.array_equal(want.astype(np.float32), want)
    acc = np.zeros(want.shape, np.float32)                    # smallest part first, in fp32
    for part in p[::-1]:
        acc = acc + mx.wgrad(v, part).astype(np.float32)
    assert np.array_equal(acc, want)
    assert (mx.wgrad(v, p[0] + p[1]) != want).any() and (mx.wgrad(v, E.bf16(J)) != want).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,f_in,f_out", [x for x in E.WGRAD if x[0] * x[1] * x[2] < 1 << 26])
def test_integers_are_exact_and_every_row_shows(rows, f_in, f_out, dtype):
    code, s, J = E.integers(rows + f_out, rows, f_in, f_out, dtype)
    v = mx.values(code, s, f_in, "int8")
    want = mx.wgrad(v, J)
    assert dtype == "f32" or np.array_equal(E.bf16(J), J)
    acc = np.zeros(want.shape, np.float32)
    parts = E.parts(J)[::-1] if dtype == "f32" else (J,)
    cut = max(1, rows // 7)
    for k in range(0, rows, cut):
        for p in parts:
            acc = acc + mx.wgrad(v[k:k + cut], p[k:k + cut]).astype(np.float32)
    assert np.array_equal(acc, want)
    assert (v[:, 0] * J[:, 0] != 0).all()                     # so is a row that is left out or counted twice


@pytest.mark.parametrize("m,n,k", [x for x in E.LONG if x[0] * x[1] < 20000])
def test_a_lost_block_of_a_long_row_shows(m, n, k):
    a, b = E.product(m + n + k, m, n, k, False)
    x, y = mx.values(*a, k, "fp4"), mx.values(*b, k, "fp4")
    assert (x > 0).all() and (y > 0).all()
    want = mx.product(x, y)
    assert np.array_equal(want.astype(np.float32), want)
    acc = np.zeros(want.shape, np.float32)
    for t in range(0, k, 512):
        acc = acc + mx.product(x[:, t:t + 512], y[:, t:t + 512]).astype(np.float32)
    assert np.array_equal(acc, want)
